// Rotation by position, shared by the ring's rows (rsa_rotate.hip) and the cache's new tokens (rsa_cache.hip).
#pragma once
#include "rsa_common.h"

namespace rsa {

// How the first R elements of a head are paired, and the angles per position.
struct Rotary {
  int R, adjacent;        // R = 0: nothing is turned
  const float *inv_freq;  // R / 2
  float sign;             // -1: the transposed rotation
};

// cos and sin of pos * freq, the angle taken as the exact product: of the turns pos * freq / (2 pi) only the fraction
// counts, which 24 bits lose from position 10^4 on.  So the product and 1 / (2 pi) are two 53-bit words each:
// the fraction errs by less than 2^-50 of a turn at any position before it is rounded to fp32, once, as a number of at
// most one half; with the sine's own rounding the results err by less than 2^-22.
__device__ __forceinline__ float2 angle_of(int64_t pos, float freq) {
#pragma clang fp contract(off)  // (t is to be the rounded product, whose error te is)
  constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;  // 1 / (2 pi)
  const double n = (double)pos, f = (double)freq, p = n * f, pe = __builtin_fma(n, f, -p);
  const double t = p * hi, te = __builtin_fma(p, hi, -t) + __builtin_fma(p, lo, pe * hi);
  const float x = 2.f * (float)((t - __builtin_rint(t)) + te);
  return make_float2(cospif(x), sinpif(x));
}

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
struct TurnShape {
  int lanes, rows;
  FastDiv by_lanes, by_units, by_half;  // threads of a group; of a row; R / 2 angles of a row
};
// The widest chunks that the pairs allow: 16 bytes, a half or a quarter of it, an element.
inline int chunk_width(int dtype, int R) {
  if (dtype != RSA_BF16) return R % 8 == 0 ? 4 : 1;
  return R % 16 == 0 ? 8 : R % 8 == 0 ? 4 : R % 4 == 0 ? 2 : 1;
}
// heads of a thread whose loads are in flight
template <typename T, int W> constexpr int kAhead = W * (int)sizeof(T) >= 8 ? 2 : 4;
inline int heads_in_flight(int dtype, int W) { return W * (dtype == RSA_BF16 ? 2 : 4) >= 8 ? 2 : 4; }
// groups of `least` threads, rounded to a power of two from 32 to 128, where they are enough for a row
inline TurnShape make_turn_shape(int A, int R, int W, int least) {
  const int units = A / (2 * W);
  TurnShape s;
  s.lanes = 32;
  while (s.lanes < 128 && (s.lanes < least || s.lanes < units)) s.lanes *= 2;
  s.rows = s.lanes / units;
  s.by_lanes = make_fast_div(s.lanes); s.by_units = make_fast_div(units); s.by_half = make_fast_div(R > 1 ? R / 2 : 1);
  return s;
}

}  // namespace rsa
