// A paged cache in 8 bits: keys and values of new tokens stored in e4m3, a power of two per row of a head (rsa_cache_append8), and the
// tokens of a cache, in 8 bits or in the calls' own type, read back as dense tensors (rsa_cache_read).
#include "rsa_cache_tokens.h"
#include "rsa_kernels.h"
#include "rsa_rotary.h"

namespace rsa {
namespace {

// ---------------------------------------------------------------- append ----
// What is stored of a row x: e4m3(x 2^-e), e the least integer with max |x| <= 448 2^e (448 the largest number of e4m3), within
// [-64, 120]; infinite elements, which have no e4m3, and NaN are stored as NaN and do not count for e.  The numbers are those of the
// definition, also next to the middle of two of them: keys are turned in fp64, from cosines and sines in fp64 of the exact angles
// (elements turned in fp32 land on the other side once in 10^6), and rounded once.  e >= -64: a row of less than 2^-55 has nothing to
// say, and times a probability no part of it falls out of the range of fp32.  e <= 120: a turned pair of bf16 numbers has at
// most 1.42 2^128.
//
// A work-group has eight tokens, whose angles its threads work out together (fp64: a table of 256 cosines and sines and a short series; the
// functions themselves in the loop took 74 us for 8 prompts of up to 2048 tokens that take 45); a lane has eight elements of a row, 16 bytes of
// bf16.  Those prompts (32 query, 8 key heads of 128, 162 MB): 45 us, 3.6 TB/s, two thirds of it memory, the rest the fp64 products and the search of each
// row's largest element; a token of each of 64 sequences 6.4: lengths, table, angles, a row's maximum, one after the other.  Heads of a tile over 2, 3, 4
// work-groups: 63, 67, 70 for 61 (with the read behind it); four heads ahead 48 for 45 (registers spill).
struct Append8Args {
  TokenArgs tok;
  const uint16_t *Q, *K, *V;
  uint16_t *Qr;
  uint8_t *Kc, *Vc, *Ks, *Vs;
  const int32_t *first;
  int64_t qs[3], ks[3];
  Rotary ro;
  FastDiv by_half;  // R / 2 angles of a token
  int Zq, Zkv;      // Zq: 0 without queries
};
constexpr int kTokens = 8;

struct CosSin { double c, s; };
// Cosine and sine in fp64 of x half turns, |x| <= 1, from those of the nearest 128th of one (kept by the work-group, so that the
// function itself and its constants are outside the loop) and the series of what is left, t <= pi / 256: t^8 / 8! and t^9 / 9! are
// below 2^-65.
constexpr int kTurn = 256;
__device__ __forceinline__ CosSin turned_by(const CosSin *turn, double x) {
  const double k = __builtin_rint(x * (kTurn / 2)), t = (x - k * (2.0 / kTurn)) * 3.14159265358979323846, u = t * t;
  const double c = 1.0 + u * (-1.0 / 2 + u * (1.0 / 24 - u * (1.0 / 720))), s = t + t * u * (-1.0 / 6 + u * (1.0 / 120 - u * (1.0 / 5040)));
  const CosSin a = turn[(int)k & (kTurn - 1)];
  return {a.c * c - a.s * s, a.s * c + a.c * s};
}

__device__ __forceinline__ float element(const u32x4 &w, int k) {
  return __builtin_bit_cast(float, k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
}
// Numbers by their bits, which full-rate integer instructions take apart: conversions and comparisons of fp64 run at a fraction of that.
struct Bits {
  uint32_t lo, hi;
  __device__ __forceinline__ explicit Bits(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    lo = (uint32_t)u; hi = (uint32_t)(u >> 32);
  }
  __device__ __forceinline__ uint32_t size() const { return hi & 0x7fffffffu; }
  __device__ __forceinline__ bool finite() const { return size() < 0x7ff00000u; }
  // In the order of the numbers' sizes, 21 bits of each, any bit behind them counted upwards; 0 for what is infinite or NaN
  __device__ __forceinline__ uint32_t rank() const { return finite() ? size() + (lo != 0) : 0u; }
  // x 2^-e as the fp32 number that rounds to e4m3 as x 2^-e does: cut off, and odd where anything was
  __device__ __forceinline__ float to_odd(int e) const {
    const int t = (int)size() - ((896 + e) << 20);  // (below fp32's normal numbers: no e4m3 number but 0)
    const uint32_t u = t < 0 ? 0u : ((uint32_t)t << 3 | lo >> 29) | ((lo & 0x1fffffffu) != 0);
    return __builtin_bit_cast(float, finite() ? u | (hi & 0x80000000u) : 0x7fc00000u);
  }
};
// The exponent that a row needs for its largest element's rank: 448 = 1.75 2^8
__device__ __forceinline__ int exponent_for(uint32_t rank) { return (int)(rank >> 20) - 1023 - 8 + ((rank & 0xfffffu) > 0xc0000u ? 1 : 0); }
__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
// The exponent of a row of which the lane knows the largest rank of its part, and one after the other's
template <int LANES> __device__ __forceinline__ int exponent_of_row(uint32_t rank) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)rank, o);
    rank = rank > y ? rank : y;
  }
  const int e = exponent_for(rank);
  return e < -64 ? -64 : e > 120 ? 120 : e;
}

// How a row's pairs lie over the lanes' pieces of eight elements: no turn; neighbours; whole pieces that change places; anything else.
enum Pairs { kNone, kNeighbours, kPieces, kAny };
// A: head size; LANES: lanes of a row (A / 8, or more)
template <int A, int PAIRS>
__global__ __launch_bounds__(256, 4) void append8_kernel(Append8Args a) {
  constexpr int LANES = A <= 64 ? 8 : A <= 128 ? 16 : 32, kRows = 256 / LANES, kHeads = kRows / kTokens;
  __shared__ CosSin turn[kTurn], angles[kTokens * A / 2 + 1];  // the last one: no turn
  const int lane = threadIdx.x % LANES, r = threadIdx.x / LANES % kTokens, head0 = threadIdx.x / LANES / kTokens;
  const int R = a.ro.R, half = R / 2, at = lane * 8;
  const bool in = at < A;  // (heads of 192: 24 of 32 lanes)
  TokenTiles<kTokens> tiles(a.tok);
  if constexpr (PAIRS != kNone) sincospi((double)threadIdx.x * (2.0 / kTurn), &turn[threadIdx.x].s, &turn[threadIdx.x].c);
  if (threadIdx.x == 0) angles[kTokens * A / 2] = {1.0, -0.0};  // (-0 stays -0)
  const bool adjacent = PAIRS == kNeighbours || (PAIRS == kAny && a.ro.adjacent);
  // Where a token's pairs are kept: such that the lanes of a row, each with its k-th, read one place after the other (in their own order, 16
  // lanes met in eight banks)
  const auto kept = [&](int p) __attribute__((always_inline)) {
    if constexpr (PAIRS == kPieces) return (p & 7) * (half / 8) + (p >> 3);
    if constexpr (PAIRS == kNeighbours) return (p & 3) * (half / 4) + (p >> 2);
    return p;
  };
  int pair[8];  // of element k
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int e = at + k;
    pair[k] = e >= R ? kTokens * A / 2 : r * half + kept(adjacent ? e >> 1 : e < half ? e : e - half);
  }
  const int from = (int)(threadIdx.x & 63) + (at >= R ? 0 : at < half ? half / 8 : -(half / 8));
  const uint32_t sign = adjacent ? 0x8000u : at < half ? 0x80008000u : 0u;  // of the partner of a pair's first element
  // own: the lane's elements of row x.  An element becomes itself times the cosine and this times the sine.
  const auto partners = [&](const u32x4 &own, const uint16_t *x) __attribute__((always_inline)) {
    u32x4 w{0, 0, 0, 0};
    if constexpr (PAIRS == kAny) {
#pragma unroll 1
      for (int k = 0; k < 8; ++k) {
        const int e = at + k;
        if (e < R) {
          const bool first = adjacent ? !(k & 1) : e < half;
          const uint32_t y = x[adjacent ? e ^ 1 : first ? e + half : e - half] ^ (first ? 0x8000u : 0u), z = k & 1 ? y << 16 : y;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] |= k >> 1 == i ? z : 0u;
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = (adjacent ? own[k] << 16 | own[k] >> 16 : (uint32_t)__shfl(own[k], from)) ^ sign;
    }
    return w;
  };
  // (the next heads' rows are on their way while some are turned, the first ones while the angles are worked out)
  const auto row_at = [&](const uint16_t *x, bool any) __attribute__((always_inline)) {
    return any ? *reinterpret_cast<const u32x4 *>(x) : u32x4{0, 0, 0, 0};
  };
  for (uint32_t item = blockIdx.x; item < tiles.items; item += gridDim.x) {
    const uint32_t tile = a.tok.by_split(item);
    tiles.begin(tile);
    const TokenPlace p = tiles.place(r);
    if (!__syncthreads_or(p.there)) continue;  // (the angles of the tile before are read)
    const int step = kHeads * (int)a.tok.by_split.d;
    // heads of Q, then of K, then of V, are dealt to the work-groups and rows in turn: this one's first of those from `base` on
    const int z0 = (int)(item - tile * a.tok.by_split.d) * kHeads + head0;
    const auto first_from = [&](int base) { return z0 >= base ? z0 - base : (base - z0 + step - 1) / step * step + z0 - base; };
    // (heads from here on, one after the other: additions instead of products of 64 bits)
    const int64_t q = (int64_t)p.b * a.qs[0] + (int64_t)p.t * a.qs[2] + z0 * a.qs[1] + at, q_step = step * a.qs[1];
    const int64_t kv = (int64_t)p.b * a.ks[0] + (int64_t)p.t * a.ks[2] + at, kv_step = step * a.ks[1];
    constexpr int kAhead = 2;
    const bool mine = p.there && in;
    u32x4 x[kAhead], first_kv[2];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) x[n] = row_at(a.Q + q + n * q_step, mine && z0 + n * step < a.Zq);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const int z = first_from(a.Zq + side * a.Zkv);
      first_kv[side] = row_at((side ? a.V : a.K) + kv + z * a.ks[1], mine && z < a.Zkv);
    }
    for (int i = threadIdx.x; PAIRS != kNone && i < kTokens * half; i += 256) {
      const uint32_t w = a.by_half(i);
      const TokenPlace q = tiles.place(w);
      if (q.there) angles[w * half + kept(i - w * half)] = turned_by(turn, half_turns_of(q.slot + (a.first ? a.first[q.b] : 0), a.ro.inv_freq[i - w * half]));
    }
    const int64_t row = p.row(a.tok, a.Zkv);
    __syncthreads();
    if (!p.there) continue;
    if (z0 < a.Zq) {
      float c[8], sn[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) { c[k] = (float)angles[pair[k]].c; sn[k] = (float)angles[pair[k]].s; }
      const uint16_t *from_q = a.Q + q;
      uint16_t *to_q = a.Qr + q;
      for (int z = z0; z < a.Zq; z += kAhead * step) {
        u32x4 next[kAhead];
        const uint16_t *behind = from_q + kAhead * q_step;
#pragma unroll
        for (int n = 0; n < kAhead; ++n) next[n] = row_at(behind + n * q_step, in && z + (kAhead + n) * step < a.Zq);
#pragma unroll
        for (int n = 0; n < kAhead; ++n) {
          if (z + n * step < a.Zq) {
            if constexpr (PAIRS != kNone) {
              const u32x4 w = partners(x[n], from_q - at);
              u32x4 y;
#pragma unroll
              for (int k = 0; k < 4; ++k)
                y[k] = pack_bf16(element(x[n], 2 * k) * c[2 * k] + element(w, 2 * k) * sn[2 * k],
                                 element(x[n], 2 * k + 1) * c[2 * k + 1] + element(w, 2 * k + 1) * sn[2 * k + 1]);
              x[n] = at < R ? y : x[n];
            }
            if (in) *reinterpret_cast<u32x4 *>(to_q) = x[n];
          }
          from_q += q_step;
          to_q += q_step;
          x[n] = next[n];
        }
      }
    }
    if (row < 0) continue;
#pragma unroll
    for (int side = 0; side < 2; ++side) {  // keys, values
      uint8_t *pool = side ? a.Vc : a.Kc, *scales = side ? a.Vs : a.Ks;
      int z = first_from(a.Zq + side * a.Zkv);
      const uint16_t *src = (side ? a.V : a.K) + kv + z * a.ks[1];
      int64_t to = row + (int64_t)z * a.tok.by_page.d;
      const int64_t to_step = (int64_t)step * a.tok.by_page.d;
      u32x4 x = first_kv[side];
      for (; z < a.Zkv; z += step, src += kv_step, to += to_step) {
        const u32x4 next = row_at(src + kv_step, in && z + step < a.Zkv);
        float f[8];
        uint32_t top = 0;
        int e;
        if (side == 0 && PAIRS != kNone) {
          double v[8];
          const u32x4 w = partners(x, src - at);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const CosSin t = angles[pair[k]];
            v[k] = (double)element(x, k);
            v[k] = at + k < R ? v[k] * t.c + (double)element(w, k) * t.s : v[k];
            const uint32_t n = Bits(v[k]).rank();
            top = top > n ? top : n;
            if (k & 1) __builtin_amdgcn_sched_barrier(0);  // (all eight at once take 40 registers more)
          }
          e = exponent_of_row<LANES>(top);
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] = Bits(v[k]).to_odd(e);
        } else {  // (bf16 numbers as they are: fp32 holds them times any power of two here)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t u = __builtin_bit_cast(uint32_t, element(x, k)) & 0x7fffffffu;
            top = u < 0x7f800000u && u > top ? u : top;
          }
          e = exponent_of_row<LANES>((top >> 3) + (896u << 20));
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float y = element(x, k);
            f[k] = __builtin_fabsf(y) < INFINITY ? y * __builtin_bit_cast(float, (uint32_t)(127 - e) << 23) : __builtin_nanf("");
          }
        }
        if (in) *reinterpret_cast<u32x2 *>(pool + to * A + at) = u32x2{four_e4m3(f[0], f[1], f[2], f[3]), four_e4m3(f[4], f[5], f[6], f[7])};
        if (lane == 0) scales[to] = (uint8_t)(e + 127);
        x = next;
      }
    }
  }
}

// ------------------------------------------------------------------ read ----
// Rows of the call's tokens out of their pages: copies, or e4m3 times its power of two, which bf16 holds exactly.  Bytes bound it: 4
// sequences of up to 32768 tokens of 8 heads of 128 move 700 MB in 143 us, 4.9 TB/s, what a copy of 4 GB reaches.
// A lane has 16 bytes of a result's row, kAhead heads' in flight (32 bytes 151 us, tiles of 16 tokens 150, nontemporal stores the same).
struct ReadArgs {
  TokenArgs tok;
  const void *Kc, *Vc;
  const uint8_t *Ks, *Vs;
  void *K, *V;
  int64_t ks[3];
  int Zkv, pad;
};
// P: type of the pools (uint8_t: e4m3), T of the results
template <typename P, typename T, int A>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
  constexpr int W = 16 / sizeof(T), kUnits = A / W, LANES = kUnits <= 8 ? 8 : kUnits <= 16 ? 16 : kUnits <= 32 ? 32 : 64;
  constexpr int kRows = 256 / LANES, kTok = kRows < kTokens ? kRows : kTokens, kHeads = kRows / kTok, kAhead = 4;
  const int lane = threadIdx.x % LANES, r = threadIdx.x / LANES % kTok, head0 = threadIdx.x / LANES / kTok, at = lane * W;
  TokenTiles<kTok> tiles(a.tok);
  for (uint32_t item = blockIdx.x; item < tiles.items; item += gridDim.x) {
    const uint32_t tile = a.tok.by_split(item);
    tiles.begin(tile);
    const TokenPlace p = tiles.place(r);
    const int64_t row = p.row(a.tok, a.Zkv);
    const int write = p.there ? 3 : p.any ? a.pad : 0;  // keys, values
    if (!write || at >= A) continue;
    const int step = kHeads * (int)a.tok.by_split.d;
    const int64_t to = (int64_t)p.b * a.ks[0] + (int64_t)p.t * a.ks[2] + at;
    // heads of K, then of V
    for (int z = (int)(item - tile * a.tok.by_split.d) * kHeads + head0; z < 2 * a.Zkv; z += kAhead * step) {
      u32x4 x[kAhead];
      uint32_t e[kAhead];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int h = z + n * step;
        x[n] = u32x4{0, 0, 0, 0};  // (what is not held, or not there)
        e[n] = 127;
        if (h < 2 * a.Zkv && row >= 0) {
          const int64_t from = row + (int64_t)(h < a.Zkv ? h : h - a.Zkv) * a.tok.by_page.d;
          const P *pool = static_cast<const P *>(h < a.Zkv ? a.Kc : a.Vc) + from * A + at;
          if constexpr (sizeof(P) == 1) {
            const u32x2 y = *reinterpret_cast<const u32x2 *>(pool);
            x[n][0] = y[0];
            x[n][1] = y[1];
            e[n] = (h < a.Zkv ? a.Ks : a.Vs)[from];
          } else {
            x[n] = *reinterpret_cast<const u32x4 *>(pool);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int h = z + n * step;
        if (h >= 2 * a.Zkv) break;
        if (!(write & (h < a.Zkv ? 1 : 2))) continue;
        if constexpr (sizeof(P) == 1) x[n] = widened8(x[n][0], x[n][1], __builtin_bit_cast(float, e[n] << 23));
        T *y = h < a.Zkv ? static_cast<T *>(a.K) + h * a.ks[1] : static_cast<T *>(a.V) + (h - a.Zkv) * a.ks[1];
        *reinterpret_cast<u32x4 *>(y + to) = x[n];
      }
    }
  }
}
template <typename P, typename T, int A> constexpr int read_rows() {
  constexpr int units = A * (int)sizeof(T) / 16;
  return 256 / (units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64);
}

TokenArgs token_args(const CacheDims &d, const int32_t *table, const int32_t *lengths, const int32_t *counts) {
  TokenArgs t{};
  t.table = table; t.lengths = lengths; t.counts = counts;
  t.by_page = make_fast_div(d.page); t.pages = d.pages; t.width = d.width;
  return t;
}

template <int A>
void launch_append8(const CacheDims &d, Append8Args a, int T, hipStream_t st) {
  constexpr int heads = 256 / (A <= 64 ? 8 : A <= 128 ? 16 : 32) / kTokens;
  const uint32_t grid = token_grid(a.tok, d.B, T, a.tok.counts, kTokens, (a.Zq + 2 * a.Zkv + heads - 1) / heads);
  const int R = a.ro.R;
  if (R == 0) append8_kernel<A, kNone><<<grid, 256, 0, st>>>(a);
  else if (a.ro.adjacent && R % 8 == 0) append8_kernel<A, kNeighbours><<<grid, 256, 0, st>>>(a);
  else if (!a.ro.adjacent && R % 16 == 0) append8_kernel<A, kPieces><<<grid, 256, 0, st>>>(a);
  else append8_kernel<A, kAny><<<grid, 256, 0, st>>>(a);
}
template <typename P, typename T, int A>
void launch_read(const CacheDims &d, ReadArgs a, int tokens, hipStream_t st) {
  constexpr int rows = read_rows<P, T, A>(), tok = rows < kTokens ? rows : kTokens, heads = rows / tok;
  const uint32_t grid = token_grid(a.tok, d.B, tokens, a.pad ? nullptr : a.tok.counts, tok, (2 * a.Zkv + heads - 1) / heads);
  read_kernel<P, T, A><<<grid, 256, 0, st>>>(a);
}
template <typename P, typename T>
void launch_read(const CacheDims &d, const ReadArgs &a, int tokens, hipStream_t st) {
  switch (d.A) {
    case 64: return launch_read<P, T, 64>(d, a, tokens, st);
    case 128: return launch_read<P, T, 128>(d, a, tokens, st);
    case 192: return launch_read<P, T, 192>(d, a, tokens, st);
    default: return launch_read<P, T, 256>(d, a, tokens, st);
  }
}

}  // namespace

hipError_t cache_append8(const CacheDims &d, const CachePools &c, int T, int R, int adjacent, const float *inv_freq, const void *Q,
                         const void *K, const void *V, const int32_t *table, const int32_t *lengths, const int32_t *counts,
                         const int32_t *first, void *Qr, hipStream_t st) {
  Append8Args a{};
  a.tok = token_args(d, table, lengths, counts);
  a.Q = static_cast<const uint16_t *>(Q); a.K = static_cast<const uint16_t *>(K); a.V = static_cast<const uint16_t *>(V);
  a.Qr = static_cast<uint16_t *>(Qr);
  a.Kc = static_cast<uint8_t *>(c.Kc); a.Vc = static_cast<uint8_t *>(c.Vc); a.Ks = c.Ks; a.Vs = c.Vs;
  a.first = first;
  for (int k = 0; k < 3; ++k) { a.qs[k] = d.qs[k]; a.ks[k] = d.ks[k]; }
  a.ro = {R, adjacent, inv_freq, 1.f};
  a.by_half = make_fast_div(R > 1 ? R / 2 : 1);
  a.Zq = Q ? d.Z : 0; a.Zkv = d.Zkv;
  switch (d.A) {
    case 64: launch_append8<64>(d, a, T, st); break;
    case 128: launch_append8<128>(d, a, T, st); break;
    case 192: launch_append8<192>(d, a, T, st); break;
    default: launch_append8<256>(d, a, T, st);
  }
  return hipGetLastError();
}

hipError_t cache_read(const CacheDims &d, const CachePools &c, int T, int pad, const int32_t *table, const int32_t *lengths, const int32_t *counts,
                      void *K, void *V, hipStream_t st) {
  ReadArgs a{};
  a.tok = token_args(d, table, lengths, counts);
  a.Kc = c.Kc; a.Vc = c.Vc; a.Ks = c.Ks; a.Vs = c.Vs; a.K = K; a.V = V;
  for (int k = 0; k < 3; ++k) a.ks[k] = d.ks[k];
  a.Zkv = d.Zkv; a.pad = pad;
  if (c.Ks) launch_read<uint8_t, bf16_t>(d, a, T, st);
  else if (d.dtype == RSA_BF16) launch_read<bf16_t, bf16_t>(d, a, T, st);
  else launch_read<float, float>(d, a, T, st);
  return hipGetLastError();
}

}  // namespace rsa
