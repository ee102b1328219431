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
// Bytes bound it, for few tokens the chain of loads.  A work-group has eight tokens, whose angles its threads work out together; a
// lane has eight elements of a row, 16 bytes of bf16.
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
// The exponent that a row needs for its largest finite element `top`: 448 = 1.75 2^8
__device__ __forceinline__ int exponent_for(double top) {
  const uint64_t u = __builtin_bit_cast(uint64_t, top);
  const int k = (int)(u >> 52) - 1023;  // (top >= 0)
  return k - 8 + ((u & 0xfffffffffffffULL) > 0xc000000000000ULL ? 1 : 0);
}
// x as the fp32 number that rounds to e4m3 as x does: one that is not exact becomes the odd one of its two neighbours.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  const double back = (double)f;
  uint32_t u = __builtin_bit_cast(uint32_t, f);
  if (back != x) u = (u - (__builtin_fabs(back) > __builtin_fabs(x) ? 1u : 0u)) | 1u;
  return __builtin_bit_cast(float, u);
}
__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ double power_of_two(int e) { return __builtin_bit_cast(double, (uint64_t)(e + 1023) << 52); }

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
  int pair[8];  // of element k
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int e = at + k;
    pair[k] = e >= R ? kTokens * A / 2 : r * half + (adjacent ? e >> 1 : e < half ? e : e - half);
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
  // (the next head's row is on its way while one is turned)
  const auto row_at = [&](const uint16_t *x, int z, int heads) __attribute__((always_inline)) {
    return in && z < heads ? *reinterpret_cast<const u32x4 *>(x + at) : u32x4{0, 0, 0, 0};
  };
  for (uint32_t item = blockIdx.x; item < tiles.items; item += gridDim.x) {
    const uint32_t tile = a.tok.by_split(item);
    tiles.begin(tile);
    const TokenPlace p = tiles.place(r);
    if (!__syncthreads_or(p.there)) continue;  // (the angles of the tile before are read)
    for (int i = threadIdx.x; PAIRS != kNone && i < kTokens * half; i += 256) {
      const uint32_t w = a.by_half(i);
      const TokenPlace q = tiles.place(w);
      if (q.there) angles[i] = turned_by(turn, half_turns_of(q.slot + (a.first ? a.first[q.b] : 0), a.ro.inv_freq[i - w * half]));
    }
    const int64_t row = p.row(a.tok, a.Zkv);
    __syncthreads();
    if (!p.there) continue;
    const int step = kHeads * (int)a.tok.by_split.d;
    // heads of Q, then of K, then of V, are dealt to the work-groups and rows in turn: this one's first of those from `base` on
    const int z0 = (int)(item - tile * a.tok.by_split.d) * kHeads + head0;
    const auto first_from = [&](int base) { return z0 >= base ? z0 - base : (base - z0 + step - 1) / step * step + z0 - base; };
    const int64_t q = (int64_t)p.b * a.qs[0] + (int64_t)p.t * a.qs[2], kv = (int64_t)p.b * a.ks[0] + (int64_t)p.t * a.ks[2];

    if (z0 < a.Zq) {
      float c[8], sn[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) { c[k] = (float)angles[pair[k]].c; sn[k] = (float)angles[pair[k]].s; }
      u32x4 x = row_at(a.Q + q + z0 * a.qs[1], z0, a.Zq);
      for (int z = z0; z < a.Zq; z += step) {
        const int64_t off = q + z * a.qs[1];
        const u32x4 next = row_at(a.Q + off + step * a.qs[1], z + step, a.Zq);
        if constexpr (PAIRS != kNone) {
          const u32x4 w = partners(x, a.Q + off);
          u32x4 y;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            y[k] = pack_bf16(element(x, 2 * k) * c[2 * k] + element(w, 2 * k) * sn[2 * k],
                             element(x, 2 * k + 1) * c[2 * k + 1] + element(w, 2 * k + 1) * sn[2 * k + 1]);
          x = at < R ? y : x;
        }
        if (in) *reinterpret_cast<u32x4 *>(a.Qr + off + at) = x;
        x = next;
      }
    }
    if (row < 0) continue;
#pragma unroll
    for (int side = 0; side < 2; ++side) {  // keys, values
      const uint16_t *src = (side ? a.V : a.K) + kv;
      uint8_t *pool = side ? a.Vc : a.Kc, *scales = side ? a.Vs : a.Ks;
      int z = first_from(a.Zq + side * a.Zkv);
      u32x4 x = row_at(src + z * a.ks[1], z, a.Zkv);
      for (; z < a.Zkv; z += step) {
        const u32x4 next = row_at(src + (z + step) * a.ks[1], z + step, a.Zkv);
        double v[8], top = 0.0;
        u32x4 w{};
        if (side == 0 && PAIRS != kNone) w = partners(x, src + z * a.ks[1]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v[k] = (double)element(x, k);
          if (side == 0 && PAIRS != kNone) {
            const CosSin t = angles[pair[k]];
            v[k] = at + k < R ? v[k] * t.c + (double)element(w, k) * t.s : v[k];
            if (k & 1) __builtin_amdgcn_sched_barrier(0);  // (all eight at once take 40 registers more)
          }
          const double size = __builtin_fabs(v[k]);
          top = size < __builtin_inf() ? __builtin_fmax(top, size) : top;
        }
        int e = exponent_for(top);
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) {
          const int y = __shfl_xor(e, o);
          e = e > y ? e : y;
        }
        e = e < -64 ? -64 : e > 120 ? 120 : e;
        const double power = power_of_two(-e);
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          f[k] = __builtin_fabs(v[k]) < __builtin_inf() ? to_odd(v[k] * power) : __builtin_nanf("");
          __builtin_amdgcn_sched_barrier(0);
        }
        const int64_t to = row + (int64_t)z * a.tok.by_page.d;
        if (in) *reinterpret_cast<u32x2 *>(pool + to * A + at) = u32x2{four_e4m3(f[0], f[1], f[2], f[3]), four_e4m3(f[4], f[5], f[6], f[7])};
        if (lane == 0) scales[to] = (uint8_t)(e + 127);
        x = next;
      }
    }
  }
}

// ------------------------------------------------------------------ read ----
// Rows of the call's tokens out of their pages: copies, or e4m3 times its power of two, which bf16 holds exactly.  Bytes bound it.
// A lane has 16 bytes of a result's row, kAhead heads' in flight.
struct ReadArgs {
  TokenArgs tok;
  const void *Kc, *Vc;
  const uint8_t *Ks, *Vs;
  void *K, *V;
  int64_t ks[3];
  int Zkv, pad, past;
};
// P: type of the pools (uint8_t: e4m3), T of the results
// past: results of 16 MB and more are stored past the caches
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
        u32x4 *place = reinterpret_cast<u32x4 *>(y + to);
        if (a.past) __builtin_nontemporal_store(x[n], place);
        else *place = x[n];
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
  a.past = (int64_t)d.B * d.Zkv * T * d.A * (d.dtype == RSA_BF16 ? 2 : 4) >= 16 << 20;
  if (c.Ks) launch_read<uint8_t, bf16_t>(d, a, T, st);
  else if (d.dtype == RSA_BF16) launch_read<bf16_t, bf16_t>(d, a, T, st);
  else launch_read<float, float>(d, a, T, st);
  return hipGetLastError();
}

}  // namespace rsa
