// Attention of several new tokens per sequence to the paged cache (rsa_cache_attend_chunk), bf16, pools in bf16 or e4m3.
//
// The rows of a key head are (token, query head) pairs, token by token with the group's heads side by side, so that all of them share
// the tiles of keys and values: a work-group owns 32 QB RW rows (RW waves) and walks the slots in tiles of 64, one pass with the
// running maximum and sum:
//   S^T = K Q^T      A operand: rows of the K tile from LDS, B operand: Q^T in registers
//   softmax on S^T   lane l owns row l % 32, so maximum and sum are in-lane but for one exchange of the halves
//   O^T += V^T P^T   A operand: V^T by transpose reads, B operand: P^T straight from the accumulators, rounded to bf16
// P is rounded once, to 2^-9 of itself, which for many keys errs as much as the stored O's own rounding does (three parts of P, as the kernels for few rows
// have them, would triple half of the matrix work, which is what bounds this kernel).
// Tiles come into LDS by direct loads from wherever their slots' pages are, a slot per lane looked up one tile further ahead; pools in
// e4m3 come through registers, where what they stand for is formed exactly in bf16, once for all rows of the work-group.
// Slots that are not seen: a score is -inf, and a value is cleared in LDS, since 0 times what lies there could be NaN.  Where rows of a
// work-group see different slots of a tile, infinite and NaN values are taken out likewise and given to the rows that see them.
#include "rsa_cache_tokens.h"
#include "rsa_fused_tile.h"
#include "rsa_kernels.h"

namespace rsa {
namespace {

struct ChunkArgs {
  const uint16_t *Q;
  const void *Kc, *Vc;
  const uint8_t *Ks, *Vs;
  const int32_t *table, *lengths, *counts;
  uint16_t *O;
  float *LSE;
  int64_t qs[3], os[3];
  FastDiv by_page, by_group, by_heads, by_Zkv, by_row;  // by_heads: B Zkv; by_row: 16-byte pieces of a row in e4m3
  int Z, Zkv, T, pages, width, causal, tiles;           // tiles: row tiles of a key head
  float cl2;                                            // scale log2(e)
  // divided walks (gridDim.y > 1): per part, key head and row the unnormalised O and the pair (maximum cl2, sum) that it is relative to
  float *part_o, *part_ml;
};

__device__ __forceinline__ int tokens_of(const ChunkArgs &a, int b) {
  const int n = a.counts ? a.counts[b] : a.T;
  return n < 0 ? 0 : n < a.T ? n : a.T;
}
__device__ __forceinline__ uint32_t length_of(const ChunkArgs &a, int b) {
  const int n = a.lengths[b], most = a.width * (int)a.by_page.d;
  return (uint32_t)(n < 0 ? 0 : n < most ? n : most);
}

template <int AH, int QB, int RW, bool EIGHT>
__global__ void __launch_bounds__(64 * RW, AH <= 2 ? 2 : 1) chunk_kernel(ChunkArgs a) {
  constexpr int A = 64 * AH, R = 32 * QB, BM = R * RW, THREADS = 64 * RW;
  // (two buffers, each an object of its own, so that the compiler sees that loads into one miss the reads of the other)
  __shared__ __attribute__((aligned(16))) unsigned char K0[AH][kTileBytes], K1[AH][kTileBytes], V0[AH][kTileBytes], V1[AH][kTileBytes];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  uint32_t head_, rank;
  longest_first(blockIdx.x, a.by_heads, head_, rank);
  const uint32_t head = settled(head_), b = settled(a.by_Zkv(head)), h = head - b * (uint32_t)a.Zkv;
  const int group = (int)a.by_group.d, tokens = tokens_of(a, (int)b), rows = tokens * group;
  const int row0 = (a.tiles - 1 - (int)rank) * BM;
  if (row0 >= rows) return;
  const uint32_t len = length_of(a, (int)b);
  const int64_t slot0 = (int64_t)a.lengths[b] - tokens;
  // the first slot that a row does not see
  const auto limit_of = [&](int row) -> uint32_t {
    const int64_t n = slot0 + (int)a.by_group((uint32_t)row) + 1;
    return !a.causal ? len : n < 0 ? 0u : n < (int64_t)len ? (uint32_t)n : len;
  };
  const int last = (row0 + BM < rows ? row0 + BM : rows) - 1;
  const uint32_t least = limit_of(row0), most = limit_of(last);
  // this work-group's tiles of the walk
  const uint32_t all = (most + kTileKeys - 1) / kTileKeys, per = (all + gridDim.y - 1) / gridDim.y;
  uint32_t t = blockIdx.y * per;
  const uint32_t end = t + per < all ? t + per : all;

  // Q^T operand: lane (col, half) holds elements dk 16 + half 8 .. + 8 of its row
  bf16x8 qreg[QB][4 * AH];
  uint32_t lim[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    int row = row0 + wave * R + qb * 32 + col;
    row = row < rows ? row : rows - 1;
    lim[qb] = limit_of(row);
    const int token = (int)a.by_group((uint32_t)row), z = (int)h * group + row - token * group;
    const uint16_t *q = a.Q + (int64_t)b * a.qs[0] + (int64_t)z * a.qs[1] + (int64_t)token * a.qs[2] + half * 8;
#pragma unroll
    for (int dk = 0; dk < 4 * AH; ++dk) qreg[qb][dk] = *reinterpret_cast<const bf16x8 *>(q + dk * 16);
  }

  // ---- the tiles' slots, one a lane
  const int32_t *table = a.table + (int64_t)b * a.width;
  const auto page_of = [&](uint32_t tile) {
    const uint32_t slot = tile * kTileKeys + lane;
    return table[a.by_page(slot < most ? slot : 0)];
  };
  struct Rows { uint32_t row; uint64_t seen; };
  const auto rows_of = [&](int id, uint32_t tile) __attribute__((always_inline)) {
    const uint32_t slot = tile * kTileKeys + lane, pg = a.by_page(slot < most ? slot : 0);
    const bool seen = slot < most && id >= 0 && id < a.pages;
    Rows r;
    r.row = seen ? ((uint32_t)id * a.Zkv + h) * a.by_page.d + (slot - pg * a.by_page.d) : 0u;
    r.seen = __ballot(seen);
    return r;
  };

  // ---- tiles into LDS.  bf16: wave w moves pieces (w PER + j) 64 + lane of 16 bytes (see TileDMAT).  e4m3: thread i has pieces
  // i, i + THREADS, ..., of 16 elements each.
  constexpr int PER = 8 / RW, P8 = 64 * (A / 16) / THREADS;
  u32x4 kraw[EIGHT ? P8 : 1], vraw[EIGHT ? P8 : 1];
  uint32_t kexp[EIGHT ? P8 : 1], vexp[EIGHT ? P8 : 1];
  const auto place8 = [&](int i, int &row, int &pc) {
    const uint32_t p = i * THREADS + tid;
    row = (int)a.by_row(p);
    pc = (int)p - row * (A / 16);
  };
  const auto load = [&](const Rows &r, auto &Kn, auto &Vn) __attribute__((always_inline)) {
    if constexpr (EIGHT) {
#pragma unroll
      for (int i = 0; i < P8; ++i) {
        int row, pc;
        place8(i, row, pc);
        const uint64_t from = __shfl(r.row, row);
        kraw[i] = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(a.Kc) + from * A + pc * 16);
        vraw[i] = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(a.Vc) + from * A + pc * 16);
        kexp[i] = a.Ks[from];
        vexp[i] = a.Vs[from];
        if (!((r.seen >> row) & 1)) kexp[i] = vexp[i] = 127;  // (not what lies there)
      }
    } else {
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int row = (wave * PER + j) * 8 + (lane >> 3), cc = (lane & 7) ^ swz_rot(row);
        const uint64_t off = (uint64_t)__shfl(r.row, row) * A + cc * 8;
#pragma unroll
        for (int ah = 0; ah < AH; ++ah) {
          lds_dma16(static_cast<const uint16_t *>(a.Kc) + off + ah * 64, Kn[ah] + (wave * PER + j) * 1024);
          lds_dma16(static_cast<const uint16_t *>(a.Vc) + off + ah * 64, Vn[ah] + (wave * PER + j) * 1024);
        }
      }
    }
  };
  // what has come through registers
  const auto store = [&](auto &Kn, auto &Vn) __attribute__((always_inline)) {
    if constexpr (EIGHT) {
#pragma unroll
      for (int i = 0; i < P8; ++i) {
        int row, pc;
        place8(i, row, pc);
        const int at0 = tile_off(row, 2 * (pc & 3)), at1 = tile_off(row, 2 * (pc & 3) + 1);
        const float kp = __builtin_bit_cast(float, kexp[i] << 23), vp = __builtin_bit_cast(float, vexp[i] << 23);
        unsigned char *k = Kn[pc >> 2], *v = Vn[pc >> 2];
        *reinterpret_cast<u32x4 *>(k + at0) = widened8(kraw[i][0], kraw[i][1], kp);
        *reinterpret_cast<u32x4 *>(k + at1) = widened8(kraw[i][2], kraw[i][3], kp);
        *reinterpret_cast<u32x4 *>(v + at0) = widened8(vraw[i][0], vraw[i][1], vp);
        *reinterpret_cast<u32x4 *>(v + at1) = widened8(vraw[i][2], vraw[i][3], vp);
      }
    }
  };

  f32x16 o[2 * AH][QB];
  float m[QB], mc[QB], l[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = -INFINITY; mc[qb] = 0.f; l[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < 2 * AH; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[db][qb][v] = 0.f;
  }
  const TileLanes tl(lane);

  Rows now{0, 0}, next{0, 0};
  int id = 0;
  if (t < end) {
    next = rows_of(page_of(t), t);
    load(next, K0, V0);
    id = page_of(t + 1);
    store(K0, V0);
  }
  wait_vmem();
  __syncthreads();

  // one tile: start the loads of the next one into (Kn, Vn), compute on (Kt, Vt)
  const auto stage = [&](auto &Kt, auto &Vt, auto &Kn, auto &Vn) __attribute__((always_inline)) {
    now = next;
    const bool more = t + 1 < end;
    if (more) {
      next = rows_of(id, t + 1);
      load(next, Kn, Vn);
      id = page_of(t + 2);
    }
    const uint32_t k0 = t * kTileKeys;
    const bool edge = now.seen != ~0ull || k0 + kTileKeys > least;  // some row does not see some slot
    if (edge) {
      // values that no row sees to 0; whether others are infinite or NaN
      bool special = false;
#pragma unroll
      for (int i = 0; i < 8 * AH / RW; ++i) {
        const int p = i * THREADS + tid, row = (p >> 3) & 63, ah = p >> 9;
        u32x4 *x = reinterpret_cast<u32x4 *>(Vt[ah] + row * 128 + (p & 7) * 16);
        if ((now.seen >> row) & 1) {
          const u32x4 w = *x;
#pragma unroll
          for (int k = 0; k < 4; ++k) special |= (w[k] & 0x7f800000u) == 0x7f800000u || (w[k] & 0x7f80u) == 0x7f80u;
        } else {
          *x = u32x4{0, 0, 0, 0};
        }
      }
      if (__syncthreads_or(special)) {
        // What kinds a row's element gets of those that it sees is counted by a product of ones (the row sees the slot) and 1, 2^10,
        // 2^20 (infinite, -infinite, NaN).
        const auto kind = [](uint32_t x) __attribute__((always_inline)) {
          return (x & 0x7f80u) != 0x7f80u ? 0u : x & 0x7fu ? 0x4980u : x & 0x8000u ? 0x4480u : 0x3f80u;
        };
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const uint64_t sees = lim[qb] > k0 ? now.seen & (lim[qb] - k0 < 64 ? (1ull << (lim[qb] - k0)) - 1 : ~0ull) : 0ull;
#pragma unroll
          for (int db = 0; db < 2 * AH; ++db) {
            f32x16 n;
#pragma unroll
            for (int v = 0; v < 16; ++v) n[v] = 0.f;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              __builtin_amdgcn_sched_barrier(0);
              const u32x4 va = __builtin_bit_cast(u32x4, tl.read_cols(Vt[db >> 1], kk * 16, db & 1));
              const uint32_t bits = (uint32_t)(sees >> (kk * 16 + half * 4));
              u32x4 w, ones;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int e = 2 * k, s0 = (e >> 2) * 8 + (e & 3);
                w[k] = kind(va[k] & 0xffffu) | kind(va[k] >> 16) << 16;
                ones[k] = ((bits >> s0) & 1 ? 0x3f80u : 0u) | ((bits >> (s0 + 1)) & 1 ? 0x3f800000u : 0u);
              }
              n = mfma_32x32x16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, ones), n);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const uint32_t c = (uint32_t)n[v];
              if (c) o[db][qb][v] += c >= (1u << 20) || ((c & 1023u) && c >= 1024u) ? __builtin_nanf("") : c >= 1024u ? -INFINITY : INFINITY;
            }
          }
        }
        __syncthreads();
        // ... and they are 0 from here on
#pragma unroll
        for (int i = 0; i < 8 * AH / RW; ++i) {
          const int p = i * THREADS + tid, row = (p >> 3) & 63, ah = p >> 9;
          u32x4 *x = reinterpret_cast<u32x4 *>(Vt[ah] + row * 128 + (p & 7) * 16);
          u32x4 w = *x;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            w[k] &= ((w[k] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u) | ((w[k] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu);
          *x = w;
        }
        __syncthreads();
      }
    }

    // ---- S^T = K Q^T
    f32x16 s[2][QB];
    float tm[QB];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      bf16x8 ka[4 * AH];
#pragma unroll
      for (int dk = 0; dk < 4 * AH; ++dk) ka[dk] = tl.read_rows(Kt[dk >> 2], kb * 32, dk & 3);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[kb][qb][v] = 0.f;
#pragma unroll
        for (int dk = 0; dk < 4 * AH; ++dk) s[kb][qb] = mfma_32x32x16(ka[dk], qreg[qb][dk], s[kb][qb]);
      }
    }
    if (edge) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int n = (int)lim[qb] - (int)k0;  // (slots are below 2^31)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const uint32_t seen = ((uint32_t)(now.seen >> (kb * 32)) & low_bits(n - kb * 32)) >> (half * 4);
#pragma unroll
          for (int v = 0; v < 16; ++v) s[kb][qb][v] = keep_bit(s[kb][qb][v], seen, (v >> 2) * 8 + (v & 3));
        }
      }
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float x = s[0][qb][0];
#pragma unroll
      for (int v = 1; v < 16; ++v) x = fmaxf(x, s[0][qb][v]);
#pragma unroll
      for (int v = 0; v < 16; ++v) x = fmaxf(x, s[1][qb][v]);
      tm[qb] = xhalf_max(x);
    }
    // ---- the accumulators are rescaled only when some row's maximum grew by more than 2^8 (exact: l and O share the stale one)
    bool need = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) need |= (tm[qb] - m[qb]) * a.cl2 > 8.0f;
    if (__builtin_amdgcn_ballot_w64(need) != 0) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        // (a row that has seen no key yet keeps mc = 0)
        const float mn = fmaxf(m[qb], tm[qb]);
        const bool any = mn > -INFINITY;
        const float alpha = any ? __builtin_amdgcn_exp2f((m[qb] - mn) * a.cl2) : 1.0f;
        m[qb] = mn;
        mc[qb] = any ? mn * a.cl2 : 0.f;
        l[qb] *= alpha;
#pragma unroll
        for (int db = 0; db < 2 * AH; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][qb][v] *= alpha;
      }
    }
    // ---- P^T = exp2(S^T cl2 - m cl2), packed to bf16 as the B operand
    bf16x8 pf[QB][4];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        float p[16];
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          p[v] = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][v], a.cl2, -mc[qb]));
          l[qb] += p[v];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const u32x4 w = {pack_bf16(p[u * 8 + 0], p[u * 8 + 1]), pack_bf16(p[u * 8 + 2], p[u * 8 + 3]),
                           pack_bf16(p[u * 8 + 4], p[u * 8 + 5]), pack_bf16(p[u * 8 + 6], p[u * 8 + 7])};
          pf[qb][kb * 2 + u] = __builtin_bit_cast(bf16x8, w);
        }
      }
    // ---- O^T += V^T P^T
#pragma unroll
    for (int db = 0; db < 2 * AH; ++db)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const bf16x8 va = tl.read_cols(Vt[db >> 1], kk * 16, db & 1);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) o[db][qb] = mfma_32x32x16(va, pf[qb][kk], o[db][qb]);
      }
    if (more) store(Kn, Vn);
    wait_vmem();
    __syncthreads();
    ++t;
  };
  while (t < end) {
    stage(K0, V0, K1, V1);
    if (t >= end) break;
    stage(K1, V1, K0, V0);
  }

  if (gridDim.y > 1) {  // this part's result
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float lt = xhalf_sum(l[qb]);
      const int row = row0 + wave * R + qb * 32 + col;
      if (row >= rows) continue;
      const int64_t pr = ((int64_t)blockIdx.y * a.by_heads.d + head) * ((int64_t)a.T * group) + row;
      float *po = a.part_o + pr * A + half * 4;
#pragma unroll
      for (int db = 0; db < 2 * AH; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4 *>(po + db * 32 + g * 8) =
              f32x4{o[db][qb][g * 4 + 0], o[db][qb][g * 4 + 1], o[db][qb][g * 4 + 2], o[db][qb][g * 4 + 3]};
      if (half == 0) *reinterpret_cast<float2 *>(a.part_ml + pr * 2) = make_float2(lt != 0.f ? mc[qb] : -INFINITY, lt);
    }
    return;
  }

  // ---- O = O^T / l, LSE = s m + ln l.  The wave's rows go through its own part of the buffers (no load is in flight) and leave
  // as whole pieces of 128 bytes.
  float inv[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float lt = xhalf_sum(l[qb]);
    inv[qb] = lt != 0.f ? 1.0f / lt : 0.f;
    const int row = row0 + wave * R + qb * 32 + col;
    if (row < rows && half == 0) {
      const int token = (int)a.by_group((uint32_t)row), z = (int)h * group + row - token * group;
      a.LSE[((int64_t)b * a.Z + z) * a.T + token] = lt != 0.f ? (mc[qb] + __builtin_amdgcn_logf(lt)) * kLn2 : -INFINITY;
    }
  }
  unsigned char *ot = wave == 0 ? K0[0] : wave == 1 ? K1[0] : wave == 2 ? V0[0] : V1[0];
#pragma unroll
  for (int ah = 0; ah < AH; ++ah) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) stage_block_T(ot, qb * 32, o[2 * ah][qb], o[2 * ah + 1][qb], inv[qb], lane);
#pragma unroll
    for (int it = 0; it < R / 8; ++it) {
      const int r = it * 8 + (lane >> 3), cc = lane & 7, row = row0 + wave * R + r;
      if (row < rows) {
        const int token = (int)a.by_group((uint32_t)row), z = (int)h * group + row - token * group;
        *reinterpret_cast<u32x4 *>(a.O + (int64_t)b * a.os[0] + (int64_t)z * a.os[1] + (int64_t)token * a.os[2] + ah * 64 + cc * 8) =
            *reinterpret_cast<const u32x4 *>(ot + tile_off(r, cc));
      }
    }
  }
}

// The parts of divided walks: with M the largest of a row's maxima, O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s.  A part that
// saw no key of the row has m = -inf and is left out.  A / 4 lanes a row, 4 columns each; eight parts in flight.
__global__ void __launch_bounds__(256) chunk_join_kernel(ChunkArgs a, FastDiv by_units, FastDiv by_rows, int A, int parts, uint32_t units) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= units) return;
  const uint32_t flat = by_units(i), col = (i - flat * by_units.d) * 4, head = by_rows(flat), row = flat - head * by_rows.d;
  const uint32_t b = a.by_Zkv(head), h = head - b * (uint32_t)a.Zkv;
  const int group = (int)a.by_group.d;
  if ((int)row >= tokens_of(a, (int)b) * group) return;
  const int64_t rows = (int64_t)a.by_heads.d * by_rows.d;
  float M = -INFINITY, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < parts; s0 += 8) {
    float2 ml[8];
    f32x4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t pr = (int64_t)(s0 + k < parts ? s0 + k : s0) * rows + flat;
      ml[k] = *reinterpret_cast<const float2 *>(a.part_ml + pr * 2);
      x[k] = *reinterpret_cast<const f32x4 *>(a.part_o + pr * A + col);
      if (s0 + k >= parts) ml[k].x = -INFINITY;
    }
    float top = M;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = fmaxf(top, ml[k].x);
    const float ref = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(M - ref);
    M = top;
    sum *= keep;
    o *= keep;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (ml[k].x == -INFINITY) continue;
      const float w = __builtin_amdgcn_exp2f(ml[k].x - ref);
      sum = fmaf(w, ml[k].y, sum);
      o += x[k] * w;
    }
  }
  const int token = (int)a.by_group(row), z = (int)h * group + (int)row - token * group;
  const float inv = sum != 0.f ? 1.0f / sum : 0.f;
  *reinterpret_cast<u32x2 *>(a.O + (int64_t)b * a.os[0] + (int64_t)z * a.os[1] + (int64_t)token * a.os[2] + col) =
      u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  if (col == 0) a.LSE[((int64_t)b * a.Z + z) * a.T + token] = sum != 0.f ? (M + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

// How a call is laid over the chip, from what the host knows: the tokens and the table's width, not counts and lengths.
struct ChunkPlan {
  bool few;         // by 16 or 32 rows at a time, from memory to the operands (rsa_cache.hip)
  int qb, rw;       // 32-row blocks of a wave, waves
  int tiles, parts;
};
ChunkPlan plan_of(const CacheDims &d, int T) {
  ChunkPlan p{};
  const int64_t rows = (int64_t)T * (d.Z / d.Zkv), heads = (int64_t)d.B * d.Zkv;
  p.few = d.dtype != RSA_BF16 || rows <= 32;
  if (p.few) return p;
  p.qb = 1; p.rw = rows <= 64 ? 2 : 4;
  if (d.A == 64 && heads * ((rows + 255) / 256) >= 512) p.qb = 2;
  p.tiles = (int)((rows + 32 * p.qb * p.rw - 1) / (32 * p.qb * p.rw));
  // too few work-groups for two on every CU: their walks are divided, sixteen tiles and more a part
  const int64_t wgs = heads * p.tiles, walk = ((int64_t)d.width * d.page + kTileKeys - 1) / kTileKeys;
  const int64_t want = (2 * kCUs + wgs - 1) / wgs, most = walk / 16 < 32 ? walk / 16 : 32;
  p.parts = (int)(want < most ? want : most > 1 ? most : 1);
  return p;
}

template <int AH, int QB, int RW>
void launch_chunk(const ChunkArgs &a, const ChunkPlan &p, hipStream_t st) {
  const dim3 grid((unsigned)(a.by_heads.d * p.tiles), (unsigned)p.parts);
  if (a.Ks) chunk_kernel<AH, QB, RW, true><<<grid, 64 * RW, 0, st>>>(a);
  else chunk_kernel<AH, QB, RW, false><<<grid, 64 * RW, 0, st>>>(a);
}
template <int AH>
void launch_chunk(const ChunkArgs &a, const ChunkPlan &p, hipStream_t st) {
  if constexpr (AH == 1) {
    if (p.qb == 2) return launch_chunk<AH, 2, 4>(a, p, st);
  }
  if (p.rw == 2) launch_chunk<AH, 1, 2>(a, p, st);
  else launch_chunk<AH, 1, 4>(a, p, st);
}

}  // namespace

size_t chunk_workspace_bytes(const CacheDims &d, int T) {
  const ChunkPlan p = plan_of(d, T);
  if (p.few) return chunk_few_workspace_bytes(d, T);
  return p.parts == 1 ? 0 : ((size_t)p.parts * d.B * d.Z * T * (d.A + 2) * 4 + 255) & ~(size_t)255;
}

hipError_t cache_attend_chunk(const CacheDims &d, const CachePools &c, int T, int causal, const void *Q, const int32_t *table,
                              const int32_t *lengths, const int32_t *counts, void *O, float *LSE, void *ws, hipStream_t st) {
  const ChunkPlan p = plan_of(d, T);
  if (p.few) return chunk_few(d, c, T, causal, Q, table, lengths, counts, O, LSE, ws, st);
  ChunkArgs a{};
  a.Q = static_cast<const uint16_t *>(Q); a.Kc = c.Kc; a.Vc = c.Vc; a.Ks = c.Ks; a.Vs = c.Vs;
  a.table = table; a.lengths = lengths; a.counts = counts; a.O = static_cast<uint16_t *>(O); a.LSE = LSE;
  for (int k = 0; k < 3; ++k) { a.qs[k] = d.qs[k]; a.os[k] = d.os[k]; }
  a.by_page = make_fast_div(d.page); a.by_group = make_fast_div(d.Z / d.Zkv);
  a.by_heads = make_fast_div((int64_t)d.B * d.Zkv); a.by_Zkv = make_fast_div(d.Zkv); a.by_row = make_fast_div(d.A / 16);
  a.Z = d.Z; a.Zkv = d.Zkv; a.T = T; a.pages = d.pages; a.width = d.width; a.causal = causal; a.tiles = p.tiles;
  a.cl2 = d.scale * kLog2e;
  const int64_t rows = (int64_t)d.B * d.Z * T;
  a.part_o = static_cast<float *>(ws);
  a.part_ml = a.part_o + (p.parts > 1 ? p.parts * rows * d.A : 0);
  switch (d.A) {
    case 64: launch_chunk<1>(a, p, st); break;
    case 128: launch_chunk<2>(a, p, st); break;
    case 192: launch_chunk<3>(a, p, st); break;
    default: launch_chunk<4>(a, p, st);
  }
  if (p.parts > 1) {
    const uint32_t units = (uint32_t)(rows * (d.A / 4));
    chunk_join_kernel<<<(units + 255) / 256, 256, 0, st>>>(a, make_fast_div(d.A / 4), make_fast_div((int64_t)T * (d.Z / d.Zkv)), d.A, p.parts, units);
  }
  return hipGetLastError();
}

}  // namespace rsa
