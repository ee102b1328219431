// The paged cache of keys and values: appending to it, attention of one new token per sequence to it, and the join of
// results over shares of it (rsa_cache_append, rsa_cache_attend, rsa_cache_join).
#include "rsa_kernels.h"
#include "rsa_rotary.h"

namespace rsa {
namespace {

constexpr int kCUs = 256;

// Uneven sequences, each of some items of work (none for b outside [0, B)), as every wave counts them for itself: lane l has
// sequences [l per, (l + 1) per), per <= 64.
struct Count {
  uint32_t mine, upto;  // items of this lane's sequences; of theirs and all before
  __device__ __forceinline__ static uint32_t scan(uint32_t x) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(x, o);
      if ((int)(threadIdx.x & 63) >= o) x += y;
    }
    return x;
  }
  template <class F> __device__ __forceinline__ Count(int B, int per, F items) : mine(0) {
    const int b0 = (int)(threadIdx.x & 63) * per, b1 = b0 + per < B ? b0 + per : B;
    if (per == 1) mine = b0 < b1 ? items(b0) : 0u;
    else for (int b = b0; b < b1; b += 8) {  // (eight loads on their way at a time)
      uint32_t n[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) n[k] = items(b + k < b1 ? b + k : b);
#pragma unroll
      for (int k = 0; k < 8; ++k) mine += b + k < b1 ? n[k] : 0u;
    }
    upto = scan(mine);
  }
  __device__ __forceinline__ uint32_t all() const { return __builtin_amdgcn_readlane(upto, 63); }
  // The sequence of item x < all(), and the items before it
  template <class F> __device__ __forceinline__ int find(uint32_t x, int B, int per, F items, uint32_t &before) const {
    const int l = __builtin_ctzll(__ballot(x < upto)), lane = (int)(threadIdx.x & 63), b = l * per + lane;
    before = __builtin_amdgcn_readlane(upto - mine, l);
    if (per == 1) return l;
    const uint32_t n = lane < per && b < B ? items(b) : 0u, s = scan(n);
    const int k = __builtin_ctzll(__ballot(x < before + s));
    before += __builtin_amdgcn_readlane(s - n, k);
    return l * per + k;
  }
};

// ---------------------------------------------------------------- append ----
// W consecutive elements in fp32.
template <typename T, int W> struct Chunk;
template <> struct Chunk<bf16_t, 8> {
  u32x4 r;
  __device__ __forceinline__ void load(const bf16_t *p) { r = *reinterpret_cast<const u32x4 *>(p); }
  __device__ __forceinline__ void load_once(const bf16_t *p) { r = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)); }
  __device__ __forceinline__ void store(bf16_t *p) const { *reinterpret_cast<u32x4 *>(p) = r; }
  __device__ __forceinline__ float get(int k) const {
    return __builtin_bit_cast(float, k & 1 ? r[k >> 1] & 0xffff0000u : r[k >> 1] << 16);
  }
  __device__ __forceinline__ void set2(int k, float x, float y) { r[k >> 1] = pack_bf16(x, y); }
};
template <> struct Chunk<bf16_t, 4> {
  u32x2 r;
  __device__ __forceinline__ void load(const bf16_t *p) { r = *reinterpret_cast<const u32x2 *>(p); }
  __device__ __forceinline__ void store(bf16_t *p) const { *reinterpret_cast<u32x2 *>(p) = r; }
  __device__ __forceinline__ float get(int k) const {
    return __builtin_bit_cast(float, k & 1 ? r[k >> 1] & 0xffff0000u : r[k >> 1] << 16);
  }
  __device__ __forceinline__ void set2(int k, float x, float y) { r[k >> 1] = pack_bf16(x, y); }
};
template <> struct Chunk<bf16_t, 2> {
  uint32_t r;
  __device__ __forceinline__ void load(const bf16_t *p) { r = *reinterpret_cast<const uint32_t *>(p); }
  __device__ __forceinline__ void store(bf16_t *p) const { *reinterpret_cast<uint32_t *>(p) = r; }
  __device__ __forceinline__ float get(int k) const { return __builtin_bit_cast(float, k & 1 ? r & 0xffff0000u : r << 16); }
  __device__ __forceinline__ void set2(int, float x, float y) { r = pack_bf16(x, y); }
};
template <> struct Chunk<float, 4> {
  f32x4 r;
  __device__ __forceinline__ void load(const float *p) { r = *reinterpret_cast<const f32x4 *>(p); }
  __device__ __forceinline__ void load_once(const float *p) { r = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p)); }
  __device__ __forceinline__ void store(float *p) const { *reinterpret_cast<f32x4 *>(p) = r; }
  __device__ __forceinline__ float get(int k) const { return r[k]; }
  __device__ __forceinline__ void set2(int k, float x, float y) { r[k] = x; r[k + 1] = y; }
};
template <typename T> struct Chunk<T, 1> {
  T r;
  __device__ __forceinline__ void load(const T *p) { r = *p; }
  __device__ __forceinline__ void store(T *p) const { *p = r; }
};

// Two chunks of a head: what one thread turns (or copies) at a time.
template <typename T, int W> struct Pair {
  Chunk<T, W> a, b;
  // element offsets of unit u's chunks
  __device__ static __forceinline__ int2 place(const Rotary &ro, int u) {
    const int turning = ro.R / (2 * W);
    if (u >= turning) return make_int2(ro.R + (u - turning) * 2 * W, ro.R + (u - turning) * 2 * W + W);
    return ro.adjacent ? make_int2(2 * u * W, 2 * u * W + W) : make_int2(u * W, ro.R / 2 + u * W);
  }
  __device__ __forceinline__ void load(const T *row, int2 at) { a.load(row + at.x); b.load(row + at.y); }
  __device__ __forceinline__ void store(T *row, int2 at) const { a.store(row + at.x); b.store(row + at.y); }
  // cs: cos and sin of the unit's W angles
  __device__ __forceinline__ void turn(const float2 (&cs)[W], int adjacent) {
    if constexpr (W == 1) {
      const float x = (float)a.r, y = (float)b.r;
      a.r = (T)(x * cs[0].x - y * cs[0].y);
      b.r = (T)(y * cs[0].x + x * cs[0].y);
    } else if (adjacent) {
#pragma unroll
      for (int k = 0; k < W; k += 2) {
        const float x = a.get(k), y = a.get(k + 1), c = cs[k / 2].x, s = cs[k / 2].y;
        a.set2(k, x * c - y * s, y * c + x * s);
        const float z = b.get(k), w = b.get(k + 1), d = cs[W / 2 + k / 2].x, t = cs[W / 2 + k / 2].y;
        b.set2(k, z * d - w * t, w * d + z * t);
      }
    } else {
#pragma unroll
      for (int k = 0; k < W; k += 2) {
        const float x0 = a.get(k), x1 = a.get(k + 1), y0 = b.get(k), y1 = b.get(k + 1);
        a.set2(k, x0 * cs[k].x - y0 * cs[k].y, x1 * cs[k + 1].x - y1 * cs[k + 1].y);
        b.set2(k, y0 * cs[k].x + x0 * cs[k].y, y1 * cs[k + 1].x + x1 * cs[k + 1].y);
      }
    }
  }
};

// How the 256 threads of a work-group lie over rows and heads: groups of `lanes` threads take one head's `rows` rows,
// `units` threads a row, 256 / lanes heads at a time.  The rows' R / 2 angles each are shared through LDS by all heads; there are
// at most lanes * W.
struct AppendShape {
  int lanes, rows;
  FastDiv by_lanes, by_units, by_half;  // threads of a group; of a row; R / 2 angles of a row
};
// The widest chunks that the pairs allow: 16 bytes, a half or a quarter of it, an element.
int chunk_width(int dtype, int R) {
  if (dtype != RSA_BF16) return R % 8 == 0 ? 4 : 1;
  return R % 16 == 0 ? 8 : R % 8 == 0 ? 4 : R % 4 == 0 ? 2 : 1;
}
// heads of a thread whose loads are in flight
template <typename T, int W> constexpr int kPairsAhead = W * (int)sizeof(T) >= 8 ? 2 : 4;
// 32 threads a group, or as many more as a row needs
AppendShape make_append_shape(int A, int R, int W) {
  const int units = A / (2 * W);
  AppendShape s;
  s.lanes = units <= 32 ? 32 : units <= 64 ? 64 : 128;
  s.rows = s.lanes / units;
  s.by_lanes = make_fast_div(s.lanes); s.by_units = make_fast_div(units); s.by_half = make_fast_div(R > 1 ? R / 2 : 1);
  return s;
}

struct AppendArgs {
  const void *Q, *K, *V;
  void *Qr, *Kc, *Vc;
  const int32_t *table, *lengths, *counts, *first;
  int64_t qs[3], ks[3];
  Rotary ro;
  AppendShape shape;
  FastDiv by_T, by_page, by_split;  // by_split: work-groups that share a tile's heads
  int B, Zq, Zkv, A, pages, width;  // Zq: 0 without queries
  uint32_t tokens;                  // B T
  int per;                          // sequences a lane counts; 0: no count, all of the B T tokens in turn
};

// Token t of sequence b: whether it is there, its slot.
struct Token {
  int64_t slot;
  bool there;
};
__device__ __forceinline__ int count_of(const AppendArgs &a, uint32_t b) {
  const int T = (int)a.by_T.d, c = a.counts ? a.counts[b] : T;
  return c < T ? c : T;
}
__device__ __forceinline__ Token token_of(const AppendArgs &a, uint32_t b, uint32_t t) {
  const int count = count_of(a, b);
  return {(int64_t)a.lengths[b] - count + t, (int)t < count};
}

// A work-group takes a few tokens, works out their angles (one a thread), turns their heads of Q and K and moves those of V.
// Where sequences have uneven numbers of tokens, every wave counts the tiles that there are and the work-groups take them in
// turn (work-groups for all B T tokens: of 16384 tokens 7144 there, the other tiles' work-groups took 10 us).
template <typename T, int W>
__global__ __launch_bounds__(256, 4) void append_kernel(AppendArgs args) {
  constexpr int ahead = kPairsAhead<T, W>;
  __shared__ float2 angles[256];
  const AppendShape &sh = args.shape;
  const uint32_t tid = threadIdx.x, head0 = sh.by_lanes(tid), lane = tid - head0 * sh.lanes, rr = sh.by_units(lane), rows = sh.rows;
  const int u = (int)(lane - rr * sh.by_units.d), heads = 256 / sh.lanes, half = args.ro.R / 2;
  const int2 at = Pair<T, W>::place(args.ro, u);
  const uint32_t ar = sh.by_half(tid);  // row of this thread's angle
  const bool turns = u < args.ro.R / (2 * W);
  const auto tiles_of = [&](int b) {
    const int c = count_of(args, b);
    return c > 0 ? (c + rows - 1) / rows : 0u;
  };
  const Count count(args.per ? args.B : 0, args.per, tiles_of);
  const uint32_t tiles = args.per ? count.all() : (args.tokens + rows - 1) / rows;
  const uint32_t items = tiles * args.by_split.d;
  for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t tile = args.by_split(item);
    // sequence and token of a row of the tile
    uint32_t b0 = 0, t0 = tile * rows;
    if (args.per) {
      uint32_t before;
      b0 = count.find(tile, args.B, args.per, tiles_of, before);
      t0 = (tile - before) * rows;
    }
    const auto place = [&](uint32_t r, uint32_t &b, uint32_t &t) {
      b = b0; t = t0 + r;
      if (!args.per) { b = args.by_T(t); t -= b * args.by_T.d; }
      return r < rows && (args.per ? t < args.by_T.d : t0 + r < args.tokens);
    };
    uint32_t b, t;
    const bool row = place(rr, b, t);
    // heads of Q, then of K, then of V; the first are on their way while the page is looked up and the angles are worked out
    const int64_t q = (int64_t)b * args.qs[0] + (int64_t)t * args.qs[2], kv = (int64_t)b * args.ks[0] + (int64_t)t * args.ks[2];
    const int all = args.Zq + 2 * args.Zkv, step = heads * (int)args.by_split.d;
    const auto source = [&](int h) {
      if (h < args.Zq) return static_cast<const T *>(args.Q) + q + h * args.qs[1];
      h -= args.Zq;
      return h < args.Zkv ? static_cast<const T *>(args.K) + kv + h * args.ks[1]
                          : static_cast<const T *>(args.V) + kv + (h - args.Zkv) * args.ks[1];
    };
    int h = (int)((item - tile * args.by_split.d) * heads + head0);
    Pair<T, W> p[ahead], next[ahead];
    Token tok{};
    if (row) tok = token_of(args, b, t);
    if (!__any(tok.there)) continue;  // (a wave sees all rows of the tile: all waves agree)
#pragma unroll
    for (int k = 0; k < ahead; ++k)
      if (tok.there && h + k * step < all) p[k].load(source(h + k * step), at);
    if (item != blockIdx.x) barrier_lds();  // (the angles of the tile before are read)
    uint32_t ab, at_token;
    if (half && place(ar, ab, at_token)) {
      const int64_t slot = token_of(args, ab, at_token).slot;
      angles[tid] = angle_of(slot + (args.first ? args.first[ab] : 0), args.ro.inv_freq[tid - ar * half]);
    }
    // where its keys and values go; -1: nowhere
    int64_t dst = -1;
    const uint32_t page = args.by_page.d;
    if (tok.there && tok.slot >= 0 && tok.slot < (int64_t)args.width * page) {
      const uint32_t pg = args.by_page((uint32_t)tok.slot);
      const int id = args.table[(int64_t)b * args.width + pg];
      if (id >= 0 && id < args.pages) dst = ((int64_t)id * args.Zkv * page + ((uint32_t)tok.slot - pg * page)) * args.A;
    }
    barrier_lds();
    if (!tok.there) continue;
    float2 cs[W];
    if (turns) {
#pragma unroll
      for (int i = 0; i < W; ++i) cs[i] = angles[rr * half + u * W + i];
    }
    for (; h < all; h += ahead * step) {
      // (loads before stores: a wait for loads counts the stores in front of them)
#pragma unroll
      for (int k = 0; k < ahead; ++k)
        if (h + (ahead + k) * step < all) next[k].load(source(h + (ahead + k) * step), at);
#pragma unroll
      for (int k = 0; k < ahead; ++k) {
        const int x = h + k * step, z = x - args.Zq, v = z - args.Zkv;
        if (x < all && (z < 0 || dst >= 0)) {
          T *to = z < 0 ? static_cast<T *>(args.Qr) + q + x * args.qs[1]
                        : (v < 0 ? static_cast<T *>(args.Kc) + dst + (int64_t)z * page * args.A
                                 : static_cast<T *>(args.Vc) + dst + (int64_t)v * page * args.A);
          if (turns && v < 0) p[k].turn(cs, args.ro.adjacent);
          p[k].store(to, at);
        }
        p[k] = next[k];
      }
    }
  }
}

template <typename T>
void launch_append(const AppendArgs &a, int W, uint32_t grid, hipStream_t st) {
  constexpr int wide = sizeof(T) == 2 ? 8 : 4;
  if (W == wide) append_kernel<T, wide><<<grid, 256, 0, st>>>(a);
  else if constexpr (sizeof(T) == 2) {
    if (W == 4) append_kernel<T, 4><<<grid, 256, 0, st>>>(a);
    else if (W == 2) append_kernel<T, 2><<<grid, 256, 0, st>>>(a);
    else append_kernel<T, 1><<<grid, 256, 0, st>>>(a);
  } else append_kernel<T, 1><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- attend ----
// One new token per sequence: S = scale q K^T over the sequence's slots, softmax, O = P V, in one pass with the running
// maximum and sum.  Every key and value is read once and takes part in 2 group products, so HBM bounds it: at 64 and more
// bytes in flight per lane the matrix cores and the vector ALU idle.
//
// A wave takes tiles of 32 (fp32: 16) slots.  Its products need no LDS and no lane exchange:
//   S^T = K Q^T   keys are the rows of a 16x16 tile, queries its columns.  K goes from memory to the operand as it lies: lane l
//                 holds 16 bytes of key l % 16.  Group g = l / 16 receives the scores of keys 4 g .. 4 g + 3 for query l % 16.
//   O^T = V^T P^T the order of the keys in the sum is free, so the probabilities stay in the lanes that have them: group g
//                 takes keys 4 g .. 4 g + 3 (bf16: of both halves of the tile), and loads these rows of V, 16 (or 8) bytes each.  Lane m's
//                 columns are VW m .. VW m + VW - 1, one per product; in bf16 eight rows' elements of one column are put together by
//                 byte permutes, half an instruction an element.
// Every accumulator of a lane belongs to its query l % 16: the rescaling by the running maximum is a product by one number.
// Query heads of one key head are the 16 (or 32) columns; a lone one pays for the unused ones nothing that counts.
struct AttendArgs {
  const void *Q, *Kc, *Vc;
  const int32_t *table, *lengths;
  void *O;
  float *LSE;
  int64_t qs[3], os[3];
  FastDiv by_page, by_tiles;  // by_tiles: query tiles of a key head
  int B, Z, Zkv, group, pages, width, per;  // per: sequences a lane counts
  float c;           // scale log2(e)
  float *part;       // partial results of divided segments (whole segments have none)
  int4 *joins;
  int by_segment;    // one note a segment, else one a share
};

template <typename T> struct AttendShape;
template <> struct AttendShape<bf16_t> { static constexpr int kKeys = 32; };
template <> struct AttendShape<float> { static constexpr int kKeys = 16; };

// Shares of `units` units for `groups` work-groups: the first units % groups have one more.
struct Shares {
  uint32_t q, r;
  __device__ __forceinline__ Shares(uint32_t units, uint32_t groups) : q(units / groups), r(units - units / groups * groups) {}
  __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * q + (w < r ? w : r); }
  __device__ __forceinline__ uint32_t of(uint32_t unit) const {  // (q > 0)
    return unit < r * (q + 1) ? unit / (q + 1) : r + (unit - r * (q + 1)) / q;
  }
};

// The larger of lanes l and l ^ 16: v_permlane16_swap exchanges the odd rows of 16 lanes of its first operand with the even ones of
// its second.
__device__ __forceinline__ float xrow_max(float x) {
  uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// The eight bits of x that a bf16 number has, cut off behind.
__device__ __forceinline__ float first_bits(float x) {
  return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u);
}

template <typename T, int A, int NQ>
struct Attend {
  static constexpr int kKeys = AttendShape<T>::kKeys;
  static constexpr bool kHalf = sizeof(T) == 2;
  static constexpr int VW = kHalf && A % 128 == 0 ? 8 : 4;      // columns of a lane
  static constexpr int NB = A / (16 * VW);                      // blocks of 16 lanes' columns
  static constexpr int KT = kHalf ? 2 : 1;                      // 16-key tiles
  static constexpr int KF = kHalf ? A / 32 : A / 16;            // 16-byte pieces of a key
  static constexpr int VR = kHalf ? 8 : 4;                      // rows of V of a lane
  static constexpr int kDw = kHalf ? VW / 2 : VW;               // dwords of a row of V
  static constexpr int kRow = A + 4;                            // floats of a row in LDS
  typedef __attribute__((__vector_size__(kDw * sizeof(uint32_t)))) uint32_t VReg;

  // registers: tile, operands and accumulators, and about 60 more; of 512 a SIMD has room for these waves
  static constexpr int kRegs = 4 * (KT * KF + NQ * KF + NQ * NB * VW) + VR * NB * kDw + 60;
  static constexpr int kSimd = kRegs <= 128 ? 4 : kRegs <= 256 ? 2 : 1;
  static constexpr int kWaves = 4, kTiles = kWaves, kUnit = kKeys * kTiles;

  struct Lds {
    float o[kWaves][16][kRow];
    float m[kWaves][16], l[kWaves][16];
  };

  const AttendArgs &args;
  Lds &lds;
  int lane, wave, g, n16;

  u32x4 q[NQ][KF];
  f32x4 acc[NQ][NB * VW];
  float m[NQ], l[NQ];
  u32x4 kr[KT][KF];
  VReg vr[VR][NB];

  __device__ __forceinline__ Attend(const AttendArgs &a, Lds &s)
      : args(a), lds(s), lane(threadIdx.x & 63), wave(threadIdx.x >> 6), g(lane >> 4), n16(lane & 15) {}

  // Rows of the pools of a tile's slots, one slot a lane (lane % kKeys), and which of them are seen, as bits.  The table's entry is
  // loaded a tile before it is looked at (slots behind the sequence: the first one's).
  struct Rows { uint32_t row, seen; };
  __device__ __forceinline__ int page_of(const int32_t *table, uint32_t len, uint32_t tile) const {
    const uint32_t slot = tile * kKeys + (lane & (kKeys - 1));
    return table[args.by_page(slot < len ? slot : 0)];
  }
  __device__ __forceinline__ Rows rows_of(int id, uint32_t len, int h, uint32_t tile) const {
    const uint32_t slot = tile * kKeys + (lane & (kKeys - 1)), pg = args.by_page(slot < len ? slot : 0);
    const bool seen = slot < len && id >= 0 && id < args.pages;
    Rows r;
    r.row = seen ? ((uint32_t)id * args.Zkv + h) * args.by_page.d + (slot - pg * args.by_page.d) : 0u;
    r.seen = (uint32_t)__ballot(seen) & (kKeys == 32 ? ~0u : 0xffffu);
    return r;
  }
  __device__ __forceinline__ void load_k(const Rows &r) {
    uint32_t row[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) row[t] = __shfl(r.row, 16 * t + n16);
    __builtin_amdgcn_sched_barrier(0);  // (one wait for all of them)
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const u32x4 *p = reinterpret_cast<const u32x4 *>(static_cast<const T *>(args.Kc) + (uint64_t)row[t] * A) + g;
#pragma unroll
      for (int i = 0; i < KF; ++i) kr[t][i] = __builtin_nontemporal_load(p + 4 * i);
    }
  }
  __device__ __forceinline__ int key_of(int j) const { return 16 * (j >> 2) + 4 * g + (j & 3); }
  __device__ __forceinline__ void load_v(const Rows &r) {
    uint32_t row[VR];
#pragma unroll
    for (int j = 0; j < VR; ++j) row[j] = __shfl(r.row, key_of(j));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < VR; ++j) {
      const VReg *p = reinterpret_cast<const VReg *>(static_cast<const T *>(args.Vc) + (uint64_t)row[j] * A) + n16;
#pragma unroll
      for (int b = 0; b < NB; ++b) vr[j][b] = __builtin_nontemporal_load(p + 16 * b);
    }
  }
  __device__ __forceinline__ void load_q(int b, int h, int tile) {
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      const int in = (tile * NQ + x) * 16 + n16;
      const u32x4 *p = reinterpret_cast<const u32x4 *>(static_cast<const T *>(args.Q) + (int64_t)b * args.qs[0] +
                                                       (int64_t)(h * args.group + in) * args.qs[1]) + g;
#pragma unroll
      for (int i = 0; i < KF; ++i) q[x][i] = in < args.group ? p[4 * i] : u32x4{0, 0, 0, 0};
    }
  }

  // Scores of the tile in kr: s[x][j] is key key_of(j)'s
  __device__ __forceinline__ void scores(f32x4 (&s)[NQ][KT]) {
#pragma unroll
    for (int x = 0; x < NQ; ++x)
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KF; ++i) {
          if constexpr (kHalf) {
            a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[t][i]), __builtin_bit_cast(bf16x8, q[x][i]), a, 0, 0, 0);
          } else {
            const f32x4 kf = __builtin_bit_cast(f32x4, kr[t][i]), qf = __builtin_bit_cast(f32x4, q[x][i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[e], a, 0, 0, 0);
          }
        }
        s[x][t] = a;
      }
  }
  // The running maximum, and s to probabilities relative to it
  __device__ __forceinline__ void softmax(f32x4 (&s)[NQ][KT], uint32_t seen) {
    const bool all = seen == (kKeys == 32 ? ~0u : 0xffffu);
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      if (!all) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[x][t][r] = (seen >> (16 * t + 4 * g + r)) & 1 ? s[x][t][r] : -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < KT; ++t) top = fmaxf(top, fmaxf(fmaxf(s[x][t][0], s[x][t][1]), fmaxf(s[x][t][2], s[x][t][3])));
      top = xhalf_max(xrow_max(top));
      const float mn = fmaxf(m[x], top * args.c);
      if (__any(mn > m[x])) {
        const float keep = __builtin_amdgcn_exp2f(m[x] - (mn == -INFINITY ? 0.f : mn));
        m[x] = mn;
        l[x] *= keep;
#pragma unroll
        for (int k = 0; k < NB * VW; ++k) acc[x][k] *= keep;
      }
      const float ref = m[x] == -INFINITY ? 0.f : m[x];
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[x][t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][t][r], args.c, -ref));
          l[x] += s[x][t][r];
        }
    }
  }
  __device__ __forceinline__ void add_values(const f32x4 (&p)[NQ][KT], uint32_t seen) {
    // (0 times what lies in a slot that is not seen could be NaN)
    if (seen != (kKeys == 32 ? ~0u : 0xffffu)) {
#pragma unroll
      for (int j = 0; j < VR; ++j)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < kDw; ++e) vr[j][b][e] = (seen >> key_of(j)) & 1 ? vr[j][b][e] : 0u;
    }
    if constexpr (kHalf) {
      // The matrix core takes bf16: a probability goes to it as three, its first eight bits, the next eight and the rest, all 24 of
      // it (as two, 2^-16 of it is lost, which shows where values cancel.  Long walks from HBM take the same, whose matrix cores wait for
      // memory; one of 200 slots 5.2 and 5.3 us, 16 of 8192 from the infinity cache with 32 queries a key head 21.3 and 22.3).  No part is
      // 0 where the probability is not (exp2 gives none below 2^-126): times an infinite value that were NaN.  The later ones are at
      // least the smallest number that bf16 has, 2^-133, which the matrix cores take as it is: less than 2^-24 of a probability of 2^-108.
      bf16x8 pb[NQ][3];
#pragma unroll
      for (int x = 0; x < NQ; ++x) {
        u32x4 w[3];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float part[3][2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float y = p[x][k >> 1 ? KT - 1 : 0][2 * (k & 1) + e], r = y - first_bits(y);
            part[0][e] = y;
            part[1][e] = __builtin_amdgcn_fmed3f(r, 0x1p-133f, y);
            part[2][e] = __builtin_amdgcn_fmed3f(r - first_bits(r), 0x1p-133f, y);
          }
#pragma unroll
          for (int i = 0; i < 3; ++i)
            w[i][k] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, part[i][1]), __builtin_bit_cast(uint32_t, part[i][0]), 0x07060302u);
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) pb[x][i] = __builtin_bit_cast(bf16x8, w[i]);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          u32x4 w;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            w[k] = __builtin_amdgcn_perm(vr[(2 * k + 1) % VR][b][(i >> 1) % kDw], vr[(2 * k) % VR][b][(i >> 1) % kDw],
                                         i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int x = 0; x < NQ; ++x)
#pragma unroll
            for (int n = 2; n >= 0; --n)
              acc[x][b * VW + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), pb[x][n], acc[x][b * VW + i], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < VW; ++i)
#pragma unroll
          for (int x = 0; x < NQ; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const f32x4 v = __builtin_bit_cast(f32x4, vr[r][b]);  // (as a whole: the cast of an element takes the first)
              acc[x][b * VW + i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i % 4], p[x][0][r], acc[x][b * VW + i], 0, 0, 0);
            }
    }
  }

  // Tiles [t, end) of key head h, query tile `tile`, of sequence b: this wave's are every fourth.
  // The keys of the next tile are on their way while this one's probabilities are formed, its values while the next scores are,
  // the table's entries for the tile behind that one before its values.
  __device__ __forceinline__ void walk(int b, int h, int tile, uint32_t len, uint32_t t, uint32_t end) {
    const int32_t *table = args.table + (int64_t)b * args.width;
    t += wave;
    load_q(b, h, tile);
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      m[x] = -INFINITY;
      l[x] = 0.f;
#pragma unroll
      for (int k = 0; k < NB * VW; ++k) acc[x][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (t >= end) return;
    Rows now = rows_of(page_of(table, len, t), len, h, t);
    load_k(now);
    __builtin_amdgcn_sched_barrier(0);  // (issued in the loop's order, which its waits count by)
    int id = page_of(table, len, t + kWaves);
    __builtin_amdgcn_sched_barrier(0);
    load_v(now);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s[NQ][KT];
    for (; t + kWaves < end; t += kWaves) {  // (the last tile behind the loop: in it, no wait counts loads that may be missing)
      scores(s);
      const Rows next = rows_of(id, len, h, t + kWaves);
      load_k(next);
      id = page_of(table, len, t + 2 * kWaves);
      softmax(s, now.seen);
      add_values(s, now.seen);
      load_v(next);
      now = next;
    }
    scores(s);
    softmax(s, now.seen);
    add_values(s, now.seen);
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      l[x] += __shfl_xor(l[x], 16);
      l[x] += __shfl_xor(l[x], 32);
    }
  }

  // The waves' results together: the segment's row, or (part) one share's
  __device__ __forceinline__ void finish(int b, int h, int tile, float *part) {
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      const int rows = args.group - (tile * NQ + x) * 16;  // of this tile
      __syncthreads();                                     // (LDS is read to the end)
      if (rows <= 0) break;
      if (n16 < rows) {
        if (g == 0) { lds.m[wave][n16] = m[x]; lds.l[wave][n16] = l[x]; }
        // accumulator (b, i), register r: column b * 16 VW + VW * (4 g + r) + i
#pragma unroll
        for (int bl = 0; bl < NB; ++bl)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < VW; i += 4) {
              const f32x4 v = {acc[x][bl * VW + i][r], acc[x][bl * VW + i + 1][r], acc[x][bl * VW + i + 2][r], acc[x][bl * VW + i + 3][r]};
              *reinterpret_cast<f32x4 *>(&lds.o[wave][n16][bl * 16 * VW + VW * (4 * g + r) + i]) = v;
            }
      }
      __syncthreads();
      const int most = rows < 16 ? rows : 16;
      for (int e = threadIdx.x; e < most * (A / 4); e += 64 * kWaves) {
        const int row = e / (A / 4), col = (e - row * (A / 4)) * 4;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds.m[w][row]);
        const float ref = top == -INFINITY ? 0.f : top;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(lds.m[w][row] - ref);
          sum += f * lds.l[w][row];
          o += f * *reinterpret_cast<const f32x4 *>(&lds.o[w][row][col]);
        }
        if (part) {
          float *p = part + (size_t)(x * 16 + row) * (A + 4);
          *reinterpret_cast<f32x4 *>(p + col) = o;
          if (col == 0) *reinterpret_cast<float2 *>(p + A) = make_float2(top, sum);
        } else {
          store_row(args, b, h * args.group + (tile * NQ + x) * 16 + row, col, o, top, sum);
        }
      }
    }
  }

  // Four columns of a row's result from sums relative to 2^top, and its LSE.
  static __device__ __forceinline__ void store_row(const AttendArgs &args, int b, int z, int col, f32x4 o, float top, float sum) {
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    T *y = static_cast<T *>(args.O) + (int64_t)b * args.os[0] + (int64_t)z * args.os[1] + col;
    if constexpr (kHalf) {
      *reinterpret_cast<u32x2 *>(y) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
    } else {
      *reinterpret_cast<f32x4 *>(y) = o * inv;
    }
    if (col == 0) args.LSE[(int64_t)b * args.Z + z] = sum != 0.f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
  }
};

__device__ __forceinline__ uint32_t length_of(const AttendArgs &args, int b) {
  const int n = args.lengths[b], most = args.width * (int)args.by_page.d;
  return (uint32_t)(n < 0 ? 0 : n < most ? n : most);
}

// A sequence with no key.
template <typename T, int A, int NQ> __device__ __forceinline__ void store_empty(const AttendArgs &args, int b) {
  for (int e = threadIdx.x; e < args.Z * (A / 4); e += 64 * Attend<T, A, NQ>::kWaves)
    Attend<T, A, NQ>::store_row(args, b, e / (A / 4), e % (A / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f}, -INFINITY, 0.f);
}

// One work-group a segment: a sequence's key head and query tile.
template <typename T, int A, int NQ>
__global__ __launch_bounds__((64 * Attend<T, A, NQ>::kWaves), (Attend<T, A, NQ>::kSimd)) void attend_whole_kernel(AttendArgs args) {
  typedef Attend<T, A, NQ> At;
  __shared__ typename At::Lds lds;
  At at(args, lds);
  const uint32_t head = args.by_tiles(blockIdx.x), tile = blockIdx.x - head * args.by_tiles.d, b = head / (uint32_t)args.Zkv, h = head - b * args.Zkv;
  const uint32_t len = length_of(args, b);
  at.walk(b, h, tile, len, 0, (len + At::kKeys - 1) / At::kKeys);
  at.finish(b, h, tile, nullptr);
}

// The work of all segments, in units of kUnit slots, in equal shares: sequences in their order, their key heads and query tiles,
// their units.  A share may begin and end inside a segment; such parts go to the work-group's two places in the workspace, and the
// work-group that has a divided segment's beginning writes down for the join where its parts lie: in the place of the segment or, if
// there are more segments than shares, in its own (a share begins one divided segment at most).  Every place gets a note, if only that
// there is nothing to do.
template <typename T, int A, int NQ>
__global__ __launch_bounds__((64 * Attend<T, A, NQ>::kWaves), (Attend<T, A, NQ>::kSimd)) void attend_shares_kernel(AttendArgs args) {
  typedef Attend<T, A, NQ> At;
  __shared__ typename At::Lds lds;
  At at(args, lds);
  const uint32_t heads = args.Zkv * args.by_tiles.d, w = blockIdx.x;
  const int4 nothing = make_int4(-1, 0, 0, 0);
  bool empty = false;
  const auto units_of = [&](int b) {
    const uint32_t len = length_of(args, b);
    empty |= len == 0;
    return (len + At::kUnit - 1) / At::kUnit;
  };
  const Count count(args.B, args.per, units_of);
  const uint32_t units = count.all() * heads;
  if (__any(empty))
    for (int b = w; b < args.B; b += gridDim.x)
      if (length_of(args, b) == 0) {
        store_empty<T, A, NQ>(args, b);
        if (args.by_segment)
          for (uint32_t k = threadIdx.x; k < heads; k += 64 * At::kWaves) args.joins[b * heads + k] = nothing;
      }
  // one share a CU, a second (third) where each then still has four units
  uint32_t groups = kCUs * (1 + units / (4 * kCUs));
  groups = groups < gridDim.x ? groups : gridDim.x;
  groups = groups < units ? groups : units;
  if (w >= groups) {
    if (threadIdx.x == 0 && !args.by_segment) args.joins[w] = nothing;
    return;
  }
  const Shares sh(units, groups);
  uint32_t unit = sh.begin(w);
  const uint32_t end = sh.begin(w + 1);
  // where the first unit is
  uint32_t before;
  int b = count.find(unit / heads, args.B, args.per, units_of, before);
  uint32_t len = __builtin_amdgcn_readfirstlane(length_of(args, b)), n = (len + At::kUnit - 1) / At::kUnit;
  uint32_t rest = unit - before * heads, head = rest / n, in = rest - head * n;
  int4 join = nothing;
  const size_t place = (size_t)(args.group < 16 * NQ ? args.group : 16 * NQ) * (A + 4);
  for (bool begun = false; unit < end; begun = true) {
    const uint32_t left = end - unit, take = n - in < left ? n - in : left;
    const uint32_t h = args.by_tiles(head), tile = head - h * args.by_tiles.d;
    at.walk(b, h, tile, len, in * At::kTiles, take == n - in ? (len + At::kKeys - 1) / At::kKeys : (in + take) * At::kTiles);
    at.finish(b, h, tile, take == n ? nullptr : args.part + (size_t)(2 * w + begun) * place);
    if (in == 0) {
      const int4 note = take == n ? nothing : make_int4(b, (int)head, 2 * (int)w + begun, (int)sh.of(unit + n - 1));
      if (take < n) join = note;
      if (args.by_segment && threadIdx.x == 0) args.joins[b * heads + head] = note;
    }
    unit += take;
    in = 0;
    if (unit < end && ++head == heads) {
      head = 0;
      // the next sequence that is not empty, of 64 at a time (one by one, 2000 empty ones took 150 us)
      for (++b; b < args.B; b += 64) {
        const uint32_t x = b + at.lane < args.B ? length_of(args, b + at.lane) : 0u;
        const uint64_t some = __ballot(x > 0);
        if (some == 0) continue;
        b += __builtin_ctzll(some);
        len = __builtin_amdgcn_readlane(x, __builtin_ctzll(some));
        break;
      }
      n = (len + At::kUnit - 1) / At::kUnit;
    }
  }
  if (threadIdx.x == 0 && !args.by_segment) args.joins[w] = join;
}

// A divided segment's parts: the first at place note.z, then place 2 v of the shares v behind it up to note.w.  A work-group a
// row and CB columns: teams of CB / 4 threads take the parts in turn, eight in flight (another XCD has written them: a load is a trip to
// memory).  Segments of 128 parts and more: 32 columns, so that 256 parts are in flight (one key head of 256, 16 queries, 32768
// slots, 23.6 us as a whole with all columns, 18.6 with 32; one of 128, 32 queries, 131072 slots, 32.1 and 28.2; but eight of 128
// with 8192 slots, 32 parts each, 13.8 and 14.5).
template <typename T, int A, int NQ, int CB>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs args) {
  constexpr int cols = CB / 4, teams = 256 / cols;
  __shared__ f32x4 sums[teams * cols];
  __shared__ float2 ends[teams];
  const int most = args.group < 16 * NQ ? args.group : 16 * NQ, team = threadIdx.x / cols;
  const int col = (int)blockIdx.z * CB + (threadIdx.x - team * cols) * 4;
  const size_t place = (size_t)most * (A + 4);
  const float *base = args.part + (size_t)blockIdx.y * (A + 4);
  struct Part {
    f32x4 o;
    float2 ml;
    __device__ __forceinline__ void load(const float *p, int col) {
      ml = *reinterpret_cast<const float2 *>(p + A);
      o = *reinterpret_cast<const f32x4 *>(p + col);
    }
    __device__ __forceinline__ void none() {
      ml = make_float2(-INFINITY, 0.f);
      o = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  const int4 j = args.joins[blockIdx.x];
  if (j.x < 0) return;
  const uint32_t head = (uint32_t)j.y, h = args.by_tiles(head), tile = head - h * args.by_tiles.d;
  const int in = (int)tile * 16 * NQ + blockIdx.y, w = j.z >> 1, parts = j.w - w + 1;
  if (in >= args.group) return;
  float top = -INFINITY, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (team < teams) {
    constexpr int ahead = 8;
    for (int k0 = team; k0 < parts; k0 += ahead * teams) {
      Part x[ahead];
#pragma unroll
      for (int k = 0; k < ahead; ++k) {
        const int i = k0 + k * teams;
        if (i < parts) x[k].load(base + (size_t)(i == 0 ? j.z : 2 * (w + i)) * place, col);
        else x[k].none();
      }
      float mn = top;
#pragma unroll
      for (int k = 0; k < ahead; ++k) mn = fmaxf(mn, x[k].ml.x);
      const float ref = mn == -INFINITY ? 0.f : mn, keep = __builtin_amdgcn_exp2f(top - ref);
      top = mn;
      sum *= keep;
      o *= keep;
#pragma unroll
      for (int k = 0; k < ahead; ++k) {
        const float f = __builtin_amdgcn_exp2f(x[k].ml.x - ref);
        sum += f * x[k].ml.y;
        o += f * x[k].o;
      }
    }
    sums[threadIdx.x] = o;
    if (threadIdx.x == team * cols) ends[team] = make_float2(top, sum);
  }
  __syncthreads();
  if (team != 0) return;
  const int used = parts < teams ? parts : teams;
#pragma unroll 8
  for (int k = 1; k < used; ++k) top = fmaxf(top, ends[k].x);
  const float ref = top == -INFINITY ? 0.f : top;
  sum = 0.f;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int k = 0; k < used; ++k) {
    const float f = __builtin_amdgcn_exp2f(ends[k].x - ref);
    sum += f * ends[k].y;
    o += f * sums[k * cols + threadIdx.x];
  }
  Attend<T, A, NQ>::store_row(args, j.x, (int)h * args.group + in, col, o, top, sum);
}

// ------------------------------------------------------------------ join ----
// O = sum_n exp(LSE_n - LSE) O_n.  Every share is read once: HBM, or for few rows the trips to it, bound this.  A thread takes 16 bytes of a
// row, A elements, four shares in flight at a time, against the running maximum (eight: 30 us for 16 shares that take 24).
// The maximum is taken off before the factor log2(e): the product of an LSE itself would be off by 2^-24 of its size.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const T *Op, const float *LSEp, T *O, float *LSE, uint32_t units, uint32_t rows, int N,
                                                   int A, FastDiv by_units, OutLayout lay) {
  constexpr int W = 16 / sizeof(T), ahead = 4;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= units) return;
  const uint32_t row = by_units(i);
  const int col = (int)(i - row * by_units.d) * W;
  const T *x = Op + (int64_t)row * A + col;
  float top = -INFINITY, sum = 0.f, o[W];
#pragma unroll
  for (int k = 0; k < W; ++k) o[k] = 0.f;
  for (int n0 = 0; n0 < N; n0 += ahead) {
    float l[ahead];
    Chunk<T, W> c[ahead];
#pragma unroll
    for (int n = 0; n < ahead; ++n) {
      l[n] = -INFINITY;
      if (n0 + n < N) {
        l[n] = LSEp[(int64_t)(n0 + n) * rows + row];
        c[n].load_once(x + (int64_t)(n0 + n) * rows * A);
        // (waits for the LSE, so that not all shares' loads go out at once: 16 shares of 16384 rows of 128 in fp32 take 24.2 us, 27.3
        // without; few rows, 16 of 512 rows of 64, 8.0 and 5.0)
        asm volatile("" : "+v"(l[n]));
      }
    }
    float mn = top;
#pragma unroll
    for (int n = 0; n < ahead; ++n) mn = fmaxf(mn, l[n]);
    const float ref = mn == -INFINITY ? 0.f : mn, keep = __builtin_amdgcn_exp2f((top - ref) * kLog2e);
    top = mn;
    sum *= keep;
#pragma unroll
    for (int k = 0; k < W; ++k) o[k] *= keep;
#pragma unroll
    for (int n = 0; n < ahead; ++n) {
      if (l[n] == -INFINITY) continue;  // (what such a share's row holds counts nothing)
      const float w = __builtin_amdgcn_exp2f((l[n] - ref) * kLog2e);
      sum += w;
#pragma unroll
      for (int k = 0; k < W; ++k) o[k] += w * c[n].get(k);
    }
  }
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
  Chunk<T, W> y;
#pragma unroll
  for (int k = 0; k < W; k += 2) y.set2(k, o[k] * inv, o[k + 1] * inv);
  y.store(O + lay.row_off(row) + col);
  if (col == 0) LSE[row] = sum != 0.f ? __builtin_fmaf(__builtin_amdgcn_logf(sum), kLn2, top) : -INFINITY;
}

}  // namespace

hipError_t cache_append(const CacheDims &d, int T, int R, int adjacent, const float *inv_freq, const void *Q, const void *K,
                        const void *V, const int32_t *table, const int32_t *lengths, const int32_t *counts, const int32_t *first,
                        void *Qr, void *Kc, void *Vc, hipStream_t st) {
  AppendArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.Qr = Qr; a.Kc = Kc; a.Vc = Vc;
  a.table = table; a.lengths = lengths; a.counts = counts; a.first = first;
  for (int k = 0; k < 3; ++k) { a.qs[k] = d.qs[k]; a.ks[k] = d.ks[k]; }
  const int W = chunk_width(d.dtype, R);
  a.ro = {R, adjacent, inv_freq, 1.f};
  a.shape = make_append_shape(d.A, R, W);
  a.by_T = make_fast_div(T); a.by_page = make_fast_div(d.page);
  a.B = d.B; a.Zq = Q ? d.Z : 0; a.Zkv = d.Zkv; a.A = d.A; a.pages = d.pages; a.width = d.width;
  a.tokens = (uint32_t)((int64_t)d.B * T);
  // uneven sequences, each of several tiles: counted (4096 of them at most, 64 a lane)
  const uint32_t rows = a.shape.rows;
  a.per = counts && T > (int)rows && d.B <= 4096 ? (d.B + 63) / 64 : 0;
  const uint32_t tiles = a.per ? d.B * ((T + rows - 1) / rows) : (a.tokens + rows - 1) / rows;
  // few tokens: their heads go to several work-groups, up to two on a CU
  const uint32_t heads = 256 / a.shape.lanes, passes = (a.Zq + 2 * a.Zkv + heads - 1) / heads, few = (2 * kCUs + tiles - 1) / tiles;
  a.by_split = make_fast_div(few < passes ? few : passes);
  const uint64_t items = (uint64_t)tiles * a.by_split.d, most = a.per ? 4 * kCUs : 1u << 20;  // (four fit a CU)
  const uint32_t grid = (uint32_t)(items < most ? items : most);
  if (d.dtype == RSA_BF16) launch_append<bf16_t>(a, W, grid, st);
  else launch_append<float>(a, W, grid, st);
  return hipGetLastError();
}

namespace {

// How a call's work is laid over the chip, from what the host knows: the table's width, not the lengths.
struct AttendPlan {
  int nq, tiles, rows, groups;  // 16-query tiles of a wave; query tiles of a key head and their rows; shares (0: whole segments)
  bool by_segment, many_parts;  // notes for the join; whether segments may be in so many parts that each goes to several work-groups
};
// Whole segments where a table has room for 96 KB of a key head's keys at most.  One work-group then takes 2 us and as many again for
// every 256 slots of 64 elements; shares and their join take 2.5 us more at the least, but no longer for longer sequences.  us,
// shares and whole segments: 16 key heads of 64 with 768 slots 7.8 and 7.0, with 1024 7.8 and 9.1; 8 of 128, four queries each, 384
// slots 8.1 and 6.4, 768 8.8 and 9.8; four of 256, 192 slots 10.3 and 8.0, 384 10.8 and 12.1; fp32, 48 of 64, 384 slots 8.3 and 8.9.
// Shares: up to three a CU for heads of 64, two, or with heads of 256 one, as registers leave room.  More than 4096 sequences (a lane
// counts 64) or 2^31 units go by whole segments whatever their length: one sequence of 131072 slots among 4095 of 64 takes 122 us, among
// 4096 of them 1730.
AttendPlan attend_plan(const CacheDims &d) {
  AttendPlan p;
  const int group = d.Z / d.Zkv, unit = 64;  // (of at least that many slots)
  p.nq = group > 16 && d.A <= 128 ? 2 : 1;   // (two tiles of longer heads do not fit the registers)
  p.tiles = (group + 16 * p.nq - 1) / (16 * p.nq);
  p.rows = group < 16 * p.nq ? group : 16 * p.nq;
  const int64_t slots = (int64_t)d.width * d.page, heads = (int64_t)d.Zkv * p.tiles, units = d.B * (slots / unit + 1) * heads;
  const bool whole = slots * d.A * (d.dtype == RSA_BF16 ? 2 : 4) <= 96 * 1024 || d.B > 4096 || units >= (1LL << 31);
  p.groups = whole ? 0 : (d.A == 64 ? 3 : d.A == 256 ? 1 : 2) * kCUs;
  const int64_t segments = d.B * heads;
  p.by_segment = segments <= p.groups;
  // 128 parts a segment and more, where the table is full
  const int64_t most = units < p.groups ? units : p.groups;
  p.many_parts = most >= 128 * segments;
  return p;
}
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <typename T, int A, int NQ>
void launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if (p.groups == 0) {
    attend_whole_kernel<T, A, NQ><<<a.B * a.Zkv * p.tiles, 64 * Attend<T, A, NQ>::kWaves, 0, st>>>(a);
    return;
  }
  attend_shares_kernel<T, A, NQ><<<p.groups, 64 * Attend<T, A, NQ>::kWaves, 0, st>>>(a);
  const uint32_t notes = a.by_segment ? a.B * a.Zkv * p.tiles : p.groups;
  if (p.many_parts) attend_join_kernel<T, A, NQ, 32><<<dim3(notes, p.rows, A / 32), 256, 0, st>>>(a);
  else attend_join_kernel<T, A, NQ, A><<<dim3(notes, p.rows), 256, 0, st>>>(a);
}
template <typename T, int A>
void launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if constexpr (A <= 128) {
    if (p.nq == 2) return launch_attend<T, A, 2>(a, p, st);
  }
  launch_attend<T, A, 1>(a, p, st);
}
template <typename T>
void launch_attend(const AttendArgs &a, const AttendPlan &p, int A, hipStream_t st) {
  switch (A) {
    case 64: return launch_attend<T, 64>(a, p, st);
    case 128: return launch_attend<T, 128>(a, p, st);
    case 192: return launch_attend<T, 192>(a, p, st);
    default: return launch_attend<T, 256>(a, p, st);
  }
}

}  // namespace

// The join's notes, 16 bytes a share, then two parts of a segment a share: rows of A sums, the maximum, the sum, two unused.
size_t cache_workspace_bytes(const CacheDims &d) {
  const AttendPlan p = attend_plan(d);
  return p.groups == 0 ? 0 : align256(p.groups * sizeof(int4)) + align256((size_t)2 * p.groups * p.rows * (d.A + 4) * 4);
}

hipError_t cache_attend(const CacheDims &d, const void *Q, const void *Kc, const void *Vc, const int32_t *table,
                        const int32_t *lengths, void *O, float *LSE, void *ws, hipStream_t st) {
  const AttendPlan p = attend_plan(d);
  AttendArgs a{};
  a.Q = Q; a.Kc = Kc; a.Vc = Vc; a.table = table; a.lengths = lengths; a.O = O; a.LSE = LSE;
  for (int k = 0; k < 3; ++k) { a.qs[k] = d.qs[k]; a.os[k] = d.os[k]; }
  a.by_page = make_fast_div(d.page); a.by_tiles = make_fast_div(p.tiles);
  a.B = d.B; a.Z = d.Z; a.Zkv = d.Zkv; a.group = d.Z / d.Zkv; a.pages = d.pages; a.width = d.width;
  a.per = (d.B + 63) / 64;
  a.c = d.scale * kLog2e;
  a.joins = static_cast<int4 *>(ws);
  a.by_segment = p.by_segment;
  a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + align256(p.groups * sizeof(int4)));
  if (d.dtype == RSA_BF16) launch_attend<bf16_t>(a, p, d.A, st);
  else launch_attend<float>(a, p, d.A, st);
  return hipGetLastError();
}

hipError_t cache_join(const CacheDims &d, int N, const void *Op, const float *LSEp, void *O, float *LSE, hipStream_t st) {
  const int unit = d.dtype == RSA_BF16 ? 8 : 4;
  const uint32_t rows = (uint32_t)(d.B * d.Z), units = rows * (uint32_t)(d.A / unit);
  const OutLayout lay = make_out_layout(d.os, 1, d.Z);
  const FastDiv by_units = make_fast_div(d.A / unit);
  const dim3 grid((units + 255) / 256);
  if (d.dtype == RSA_BF16) join_kernel<<<grid, 256, 0, st>>>((const bf16_t *)Op, LSEp, (bf16_t *)O, LSE, units, rows, N, d.A, by_units, lay);
  else join_kernel<<<grid, 256, 0, st>>>((const float *)Op, LSEp, (float *)O, LSE, units, rows, N, d.A, by_units, lay);
  return hipGetLastError();
}

}  // namespace rsa
