// Rotation of queries and keys by position (rsa_rotate, rsa_rotate_bwd).
//
// y = x turned by its token's angles: every element is read and written once, so HBM bounds it.  The angles are the same for all
// heads, and 75 instructions each: a work-group takes a few rows, works out their angles and turns these rows of several
// heads, all of whose loads are in flight meanwhile.  A lane has 16 bytes of a row, its partner's come from another lane.
#include "rsa_kernels.h"
#include "rsa_rotary.h"

namespace rsa {
namespace {

// 16 bytes of a row.
template <typename T> struct RowChunk;
template <> struct RowChunk<bf16_t> {
  static constexpr int W = 8;
  u32x4 r;
  __device__ __forceinline__ float get(int k) const {
    return __builtin_bit_cast(float, k & 1 ? r[k >> 1] & 0xffff0000u : r[k >> 1] << 16);
  }
  __device__ __forceinline__ void set2(int k, float x, float y) { r[k >> 1] = pack_bf16(x, y); }
  // neighbours in exchanged places
  __device__ __forceinline__ RowChunk swapped() const {
    RowChunk c;
#pragma unroll
    for (int i = 0; i < 4; ++i) c.r[i] = (r[i] >> 16) | (r[i] << 16);
    return c;
  }
};
template <> struct RowChunk<float> {
  static constexpr int W = 4;
  u32x4 r;
  __device__ __forceinline__ float get(int k) const {
    const uint32_t x = r[k];
    return __builtin_bit_cast(float, x);
  }
  __device__ __forceinline__ void set2(int k, float x, float y) {
    r[k] = __builtin_bit_cast(uint32_t, x);
    r[k + 1] = __builtin_bit_cast(uint32_t, y);
  }
  __device__ __forceinline__ RowChunk swapped() const {
    RowChunk c;
    c.r = u32x4{r[1], r[0], r[3], r[2]};
    return c;
  }
};
// How the waves of a work-group lie over rows and heads: a lane has a chunk of a row, a wave as many whole rows as it has lanes for,
// one to four waves a head's 8 rows in one piece (4 where a row takes more than half a wave).
struct TurnShape {
  int chunks, wave_rows, waves, rows;  // chunks of a row; rows of a wave; waves of a head; rows of a head
  FastDiv by_chunks, by_half;          // by_half: R / 2 angles of a row
};
TurnShape make_turn_shape(int A, int R, int dtype) {
  TurnShape s;
  s.chunks = A / (dtype == RSA_BF16 ? 8 : 4);
  s.wave_rows = 64 / s.chunks;
  s.waves = s.wave_rows >= 8 ? 1 : s.wave_rows >= 4 ? 2 : 4;
  s.rows = s.wave_rows * s.waves;
  s.by_chunks = make_fast_div(s.chunks); s.by_half = make_fast_div(R > 1 ? R / 2 : 1);
  return s;
}
constexpr int kTurnAngles = 1024;  // of a work-group at most: 8 rows of 128 pairs

// A thread's place in that.
struct Place {
  int lane, group, row, c;  // group: which head; row, c: row of the tile, chunk of the row
  __host__ __device__ __forceinline__ Place(const TurnShape &s, uint32_t thread) {
    const int wave = (int)(thread >> 6);
    lane = (int)(thread & 63);
    const int in = (int)s.by_chunks((uint32_t)lane);
    group = s.waves == 1 ? wave : s.waves == 2 ? wave >> 1 : 0;
    // Lanes behind the wave's whole rows (heads of 192 leave 16) have none: a row behind the tile's, and a chunk behind a row's, whose
    // elements nothing turns.
    const bool some = in < s.wave_rows;
    row = some ? (wave - group * s.waves) * s.wave_rows + in : 1 << 20;
    c = some ? lane - in * s.chunks : lane;
  }
};
// Where the element that e of a row is turned with is, in pairs half the turned part apart.
__host__ __device__ __forceinline__ int partner_of(int e, int R) { return e < R / 2 ? e + R / 2 : e < R ? e - R / 2 : e; }

// What a thread turns by: y = x co + partner si.
// WHOLE: a chunk is turned as a whole or not, and its partner in a half is one lane's chunk.
bool whole_chunks(int dtype, int R, int adjacent) {
  const int w = dtype == RSA_BF16 ? 8 : 4;
  return R % (adjacent ? w : 2 * w) == 0;
}
template <typename T, bool WHOLE> struct Turn : Place {
  static constexpr int W = RowChunk<T>::W;
  float co[W], si[W];

  __device__ __forceinline__ explicit Turn(const TurnShape &s) : Place(s, threadIdx.x) {}
  // the angles of this thread's elements, from those of its row
  __device__ __forceinline__ void take(const Rotary &ro, const float2 *angles) {
    const int half = ro.R / 2;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const int e = c * W + k, i = ro.adjacent ? e >> 1 : e < half ? e : e - half;
      const bool first = ro.adjacent ? (k & 1) == 0 : e < half;
      const float2 cs = e < ro.R ? angles[i] : make_float2(1.f, 0.f);
      co[k] = cs.x;
      si[k] = first ? -cs.y : cs.y;
    }
  }
  // The turned chunk.  All lanes of the wave have to come here; scratch: 1 KB of LDS of this wave's own (not WHOLE).
  __device__ __forceinline__ RowChunk<T> turned(const Rotary &ro, const RowChunk<T> &x, u32x4 *scratch) const {
    const int half = ro.R / 2;
    RowChunk<T> p, y;
    if (ro.adjacent) {
      p = x.swapped();
    } else if (WHOLE) {
      const int from = c * W < half ? lane + half / W : c * W < ro.R ? lane - half / W : lane;
#pragma unroll
      for (int i = 0; i < 4; ++i) p.r[i] = __shfl(x.r[i], from);
    } else {
      scratch[lane] = x.r;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const unsigned char *mine = reinterpret_cast<const unsigned char *>(scratch + (lane - c));
#pragma unroll
      for (int k = 0; k < W; k += 2) {
        float v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int from = partner_of(c * W + k + j, ro.R);
          T z;
          __builtin_memcpy(&z, mine + from * sizeof(T), sizeof(T));
          v[j] = (float)z;
        }
        p.set2(k, v[0], v[1]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
#pragma unroll
    for (int k = 0; k < W; k += 2) y.set2(k, x.get(k) * co[k] + p.get(k) * si[k], x.get(k + 1) * co[k + 1] + p.get(k + 1) * si[k + 1]);
    // elements from R on are copies (a product by 0 would not be one next to an infinity)
    if (WHOLE) return c * W < ro.R ? y : x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = c * W + i * (W / 4);  // the first of this word's one or two; R is even, so both are turned or neither
      y.r[i] = e < ro.R ? y.r[i] : x.r[i];
    }
    return y;
  }
};

struct Side {  // Q or K
  const void *x;
  void *y;
  int64_t st[3];
  uint32_t rows, tiles;  // of a sequence
};
struct RotateArgs {
  Side side[2];
  Rotary ro;
  TurnShape shape;
  RowMap map;  // rows of Q
  FastDiv by_Z;
  int heads;  // of all sequences
};
constexpr int kAhead = 4;  // heads of a wave

// PAST: results go past the caches
template <typename T, bool WHOLE, bool PAST>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs args) {
  __shared__ float2 angles[kTurnAngles];
  __shared__ u32x4 scratch[WHOLE ? 1 : 256];
  const TurnShape &sh = args.shape;
  Turn<T, WHOLE> turn(sh);
  const uint32_t tile = blockIdx.z * gridDim.x + blockIdx.x;
  if (tile >= args.side[0].tiles + args.side[1].tiles) return;
  const bool keys = tile >= args.side[0].tiles;
  const Side &s = args.side[keys ? 1 : 0];
  const uint32_t n0 = (tile - (keys ? args.side[0].tiles : 0u)) * sh.rows, n = n0 + turn.row;
  const bool have = turn.row < sh.rows && n < s.rows;
  const int64_t at = (int64_t)n * s.st[2] + turn.c * turn.W;
  const auto offset = [&](int h) { return head_offset((uint32_t)h, args.by_Z, s.st) + at; };
  const int groups = 4 / sh.waves, h = (int)blockIdx.y * kAhead * groups + turn.group;
  RowChunk<T> x[kAhead] = {};
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (have && h + k * groups < args.heads) x[k].r = *reinterpret_cast<const u32x4 *>(static_cast<const T *>(s.x) + offset(h + k * groups));
  for (uint32_t e = threadIdx.x; e < sh.rows * sh.by_half.d; e += 256) {
    const uint32_t r = sh.by_half(e);
    if (n0 + r >= s.rows) break;
    const int64_t pos = keys ? (int64_t)(n0 + r) : args.map((int64_t)(n0 + r));
    const float2 cs = angle_of(pos, args.ro.inv_freq[e - r * sh.by_half.d]);
    angles[e] = make_float2(cs.x, args.ro.sign * cs.y);
  }
  barrier_lds();
  turn.take(args.ro, angles + (have ? turn.row * (int)sh.by_half.d : 0));
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const RowChunk<T> y = turn.turned(args.ro, x[k], scratch + (WHOLE ? 0 : threadIdx.x & 192));
    if (have && h + k * groups < args.heads) {
      u32x4 *to = reinterpret_cast<u32x4 *>(static_cast<T *>(s.y) + offset(h + k * groups));
      if constexpr (PAST) __builtin_nontemporal_store(y.r, to);
      else *to = y.r;
    }
  }
}

template <typename T>
void launch(const RotateArgs &a, bool whole, bool past, dim3 grid, hipStream_t st) {
  if (whole) past ? rotate_kernel<T, true, true><<<grid, 256, 0, st>>>(a) : rotate_kernel<T, true, false><<<grid, 256, 0, st>>>(a);
  else past ? rotate_kernel<T, false, true><<<grid, 256, 0, st>>>(a) : rotate_kernel<T, false, false><<<grid, 256, 0, st>>>(a);
}

}  // namespace

hipError_t rotate_rows(const Dims &d, int dtype, int R, int adjacent, const float *inv_freq, bool back, const void *Q,
                       const void *K, void *Qr, void *Kr, hipStream_t st) {
  RotateArgs a{};
  a.ro = {R, adjacent, inv_freq, back ? -1.f : 1.f};
  a.shape = make_turn_shape(d.A, R, dtype);
  a.map = make_row_map(d);
  a.by_Z = make_fast_div(d.Z);
  a.heads = d.B * d.Z;
  for (int i = 0; i < 2; ++i) {
    Side &s = a.side[i];
    s.x = i ? K : Q; s.y = i ? Kr : Qr;
    for (int k = 0; k < 3; ++k) s.st[k] = i ? d.ks[k] : d.qs[k];
    s.rows = s.x ? (uint32_t)(i ? d.L : d.Lq) : 0;
    s.tiles = (s.rows + a.shape.rows - 1) / a.shape.rows;
  }
  const uint32_t tiles = a.side[0].tiles + a.side[1].tiles, each = kAhead * (4 / a.shape.waves);
  const uint32_t x = tiles < (1u << 22) ? tiles : (1u << 22);  // (a dimension of a grid has less than 2^32 threads)
  const dim3 grid(x, (a.heads + each - 1) / each, (tiles + x - 1) / x);
  // Results of 16 MB and more are written past the caches: a pass over B8 Z16 L2048 (67 MB) 25.0 -> 21.3 us, in fp32 over
  // B2 Z12 L4608 (57 MB) 21.6 -> 17.6, a layer's projections, rotation and attention of B16 Z12 L512 (25 MB) 89 -> 86 and of the large ones
  // the same.  Small ones stay where the next kernel finds them: a layer of B2 Z16 L512 (4 MB) 37.1, past the caches 37.6.
  const bool past = (int64_t)(a.side[0].rows + (int64_t)a.side[1].rows) * a.heads * d.A * (dtype == RSA_BF16 ? 2 : 4) >= 16 << 20;
  const bool whole = whole_chunks(dtype, R, adjacent);
  if (dtype == RSA_BF16) launch<bf16_t>(a, whole, past, grid, st);
  else launch<float>(a, whole, past, grid, st);
  return hipGetLastError();
}

}  // namespace rsa
