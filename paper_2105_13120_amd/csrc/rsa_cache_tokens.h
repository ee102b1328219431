// What the calls on the paged cache share: uneven sequences counted by every wave, the tokens of a call and where they lie, elements
// in e4m3.
#pragma once
#include "rsa_common.h"

namespace rsa {

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

// The new tokens of a call: up to T of every sequence, at its last slots.  Work-groups take them in tiles of a few; where sequences
// have uneven numbers of them, only the tiles that there are.
struct TokenArgs {
  const int32_t *table, *lengths, *counts;
  FastDiv by_T, by_page, by_split;  // by_split: work-groups that share a tile's heads
  int B, pages, width;
  uint32_t tokens;                  // B T
  int per;                          // sequences a lane counts; 0: no count, all of the B T tokens in turn
  __device__ __forceinline__ int count_of(uint32_t b) const {
    const int T = (int)by_T.d, c = counts ? counts[b] : T;
    return c < T ? c : T;
  }
};
// Token t of sequence b: whether there is such a row, whether the token is there, its slot, and the row of a pool's first head that it lies in (-1: on no page that is
// held, page * Zkv * tokens of a page + place otherwise).
struct TokenPlace {
  uint32_t b, t;
  int64_t slot;
  bool any, there;
  __device__ __forceinline__ int64_t row(const TokenArgs &a, int Zkv) const {
    const uint32_t page = a.by_page.d;
    if (!there || slot < 0 || slot >= (int64_t)a.width * page) return -1;
    const uint32_t pg = a.by_page((uint32_t)slot);
    const int id = a.table[(int64_t)b * a.width + pg];
    return id >= 0 && id < a.pages ? (int64_t)id * Zkv * page + ((uint32_t)slot - pg * page) : -1;
  }
};
template <int ROWS>
struct TokenTiles {
  const TokenArgs &a;
  Count count;
  uint32_t items;
  __device__ __forceinline__ static uint32_t tiles_of(const TokenArgs &a, int b) {
    const int c = a.count_of(b);
    return c > 0 ? (uint32_t)(c + ROWS - 1) / ROWS : 0u;
  }
  __device__ __forceinline__ explicit TokenTiles(const TokenArgs &args)
      : a(args), count(args.per ? args.B : 0, args.per, [&](int b) { return tiles_of(args, b); }) {
    items = (a.per ? count.all() : (a.tokens + ROWS - 1) / ROWS) * a.by_split.d;
  }
  uint32_t b0, t0;
  __device__ __forceinline__ void begin(uint32_t tile) {
    b0 = 0; t0 = tile * ROWS;
    if (a.per) {
      uint32_t before;
      b0 = count.find(tile, a.B, a.per, [&](int b) { return tiles_of(a, b); }, before);
      t0 = (tile - before) * ROWS;
    }
  }
  __device__ __forceinline__ TokenPlace place(uint32_t r) const {
    TokenPlace p{b0, t0 + r, 0, false, false};
    if (a.per ? p.t >= a.by_T.d : p.t >= a.tokens) return p;
    if (!a.per) { p.b = a.by_T(p.t); p.t -= p.b * a.by_T.d; }
    p.any = true;
    const int c = a.count_of(p.b);
    p.there = (int)p.t < c;
    p.slot = (int64_t)a.lengths[p.b] - c + p.t;
    return p;
  }
};
// ... and their grid: up to four work-groups a CU where tokens are counted; few tokens' heads go to several, up to two on a CU.
inline uint32_t token_grid(TokenArgs &a, int B, int T, const int32_t *counts, int rows, int passes) {
  a.B = B; a.by_T = make_fast_div(T); a.tokens = (uint32_t)((int64_t)B * T);
  a.per = counts && T > rows && B <= 4096 ? (B + 63) / 64 : 0;  // (64 a lane)
  const uint32_t tiles = a.per ? B * ((T + rows - 1) / rows) : (a.tokens + rows - 1) / rows, few = (2 * kCUs + tiles - 1) / tiles;
  a.by_split = make_fast_div(few < (uint32_t)passes ? few : passes);
  const uint64_t items = (uint64_t)tiles * a.by_split.d, most = a.per ? 4 * kCUs : 1u << 20;
  return (uint32_t)(items < most ? items : most);
}

// The eight bits of x that a bf16 number has, cut off behind.
__device__ __forceinline__ float first_bits(float x) {
  return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u);
}
// The matrix core takes bf16: a probability goes to it as three, its first eight bits, the next eight and the rest, all 24 of it; here
// of two probabilities.  No part is 0 where the probability is not (exp2 gives none below 2^-126): times an infinite value that were
// NaN.  The later ones are at least the smallest number that bf16 has, 2^-133, which the matrix cores take as it is: less than 2^-24 of a
// probability of 2^-108.
__device__ __forceinline__ void three_parts(float a, float b, uint32_t (&w)[3]) {
  const float y[2] = {a, b};
  float part[3][2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float r = y[e] - first_bits(y[e]);
    part[0][e] = y[e];
    part[1][e] = __builtin_amdgcn_fmed3f(r, 0x1p-133f, y[e]);
    part[2][e] = __builtin_amdgcn_fmed3f(r - first_bits(r), 0x1p-133f, y[e]);
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) w[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, part[i][1]), __builtin_bit_cast(uint32_t, part[i][0]), 0x07060302u);
}

// Elements in e4m3 times a power of two (a float, of which only the exponent counts), as bf16, exactly: two of a dword's, eight.
__device__ __forceinline__ uint32_t widened2(uint32_t x, float power, bool hi) {
  return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, power, true))
            : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, power, false));
}
__device__ __forceinline__ u32x4 widened8(uint32_t lo, uint32_t hi, float power) {
  return u32x4{widened2(lo, power, false), widened2(lo, power, true), widened2(hi, power, false), widened2(hi, power, true)};
}

}  // namespace rsa
