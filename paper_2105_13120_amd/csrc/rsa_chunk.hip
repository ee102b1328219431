// Attention of several new tokens per sequence to the paged cache (rsa_cache_attend_chunk), bf16, pools in bf16 or e4m3.
//
// The rows of a key head are (token, query head) pairs, token by token with the group's heads side by side, so that all of them share
// the tiles of keys and values: a work-group owns 32 QB rows for each of its RW waves, or KS of them, and walks the slots in tiles of 64, one pass
// with the running maximum and sum:
//   S^T = K Q^T      A operand: rows of the K tile from LDS, B operand: Q^T in registers
//   softmax on S^T   lane l owns row l % 32, so maximum and sum are in-lane but for one exchange of the halves
//   O^T += V^T P^T   A operand: V^T by transpose reads, B operand: P^T straight from the accumulators, rounded to bf16
// Up to 32 rows of a key head P goes to the matrix cores whole, as three bf16 numbers.  Beyond, it is rounded once, by 2^-8 of itself at most, as in
// rsa_forward: results err by 2.0 to 2.4e-3 of their RMS, where the rounding of the stored O alone errs by 1.6 to 1.7e-3 (three parts would triple half of the
// matrix work, which bounds these calls: up to 64 rows, where it bounds them least, 3 to 30 % more time).
// Tiles come into LDS by direct loads from wherever their slots' pages are, a slot per lane looked up one tile further ahead; pools in
// e4m3 come through registers, where what they stand for is formed exactly in bf16, once for all rows of the work-group.
// Bound by the matrix cores, busy in 54 % of the cycles, and the vector ALU, busy with softmax in 43 %: 2048 tokens of 65536 slots, 32 query, 8 key heads of 128, run at 1.07 to 1.13 PFLOP/s from one GPU to another, where
// a product of two 8192 x 8192 matrices by the library does 1.23; prompts of up to 2048 tokens at 0.58, of which a work-group's start and end, when
// the matrix cores wait, take a third.
// Tried: work-groups that stay and ask for the next item's first tile ahead (1954 -> 2172 us, prompts 126 -> 142); loads a tile and a half ahead with two
// barriers (3 to 9 % slower but for short walks).
// Slots that are not seen: a score is -inf, and a value is cleared in LDS, since 0 times what lies there could be NaN.  Where rows of a
// work-group see different slots of a tile, infinite and NaN values are taken out likewise and given to the rows that see them.  What such a
// row has is infinite from then on, whatever its sums so far weigh beside later ones (Weight).
#include "rsa_cache_tokens.h"
#include "rsa_fused_tile.h"
#include "rsa_kernels.h"

#include <algorithm>

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
  int B, Z, Zkv, T, pages, width, causal, pad, tiles;   // tiles: row tiles of a key head
  float cl2;                                            // scale log2(e)
  // Divided walks, where there may be parts > 1 of them: how many parts each sequence's are in, and per part, key head and row tile the
  // unnormalised O, as the accumulators hold it (16 bytes a lane), and per row the pair (maximum cl2, sum) that it is relative to
  int parts;
  uint32_t *divided;
  float *part_o, *part_ml;
};

__device__ __forceinline__ int tokens_of(const ChunkArgs &a, int b) {
  const int n = a.counts ? a.counts[b] : a.T;
  return n < 0 ? 0 : n < a.T ? n : a.T;
}
__device__ __forceinline__ uint32_t slots_of(const ChunkArgs &a, int length) {
  const int most = a.width * (int)a.by_page.d;
  return (uint32_t)(length < 0 ? 0 : length < most ? length : most);
}

// 2^x, x <= 0, as two factors that are not 0: an infinity times 0 were NaN, where a row had seen no key yet (x = -inf) or none near the largest score.
// From -126 on, below which exp2 gives 0, the second is 1; finite numbers times both become less than 2^-124 at x <= -252.
struct Weight {
  float a, b;
  __device__ __forceinline__ explicit Weight(float x)
      : a(__builtin_amdgcn_exp2f(fmaxf(x, -126.f))), b(__builtin_amdgcn_exp2f(fminf(fmaxf(x + 126.f, -126.f), 0.f))) {}
};

// What a call's work-groups take: a row tile of a key head of a sequence and, where its walk is divided, one of its parts.
struct Item {
  uint32_t b, h;
  int tile, part, parts;
  int tokens, length;  // of the sequence: new tokens that are there, its entry of `lengths`
};

// Sequences of different lengths with different numbers of new tokens leave tiles without rows and walks of all lengths.  Up to
// kSorted sequences are laid out by what they have: all items by the length of their walks, the longest first, without gaps (8 prompts of 128 to
// 2048 tokens by the tiles of the longest, empty ones among them: 154 us; in this order 126).  A walk that is long beside a place's share of all the
// work is divided.
//
// A tile's walk is w = ceil(n / P) long, n the tiles of 64 slots that its last row sees and P the parts of its sequence's walks.  The
// last row's limit grows with the tile, so that the tiles of a sequence with walks of w and more are those from a first one on, and
// F(w), how many items there are of w and more, is a sum over the sequences.  The item `id` in descending order is in level w with
// F(w + 1) <= id < F(w), found by halves; a lane has a sequence.
constexpr int kSorted = 64;

// Sums of a lane and those before it
__device__ __forceinline__ uint32_t scan_lanes(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true);  // row_shr 1, 2, 4, 8: within 16 lanes
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);  // lane 15 of a row to the next, lane 31 to the upper half
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
  return x;
}
__device__ __forceinline__ uint32_t sum_lanes(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)scan_lanes(x), 63); }
template <int BM, int PLACES>
struct Layout {
  const ChunkArgs &a;
  int lane, tokens, length, tiles, most, slot0, parts;  // of the lane's sequence, row tiles that have any, tiles of its longest walk, its first token's slot
  __device__ __forceinline__ static uint32_t walk_of(const ChunkArgs &a, int64_t slot0, uint32_t len, int token) {
    const int64_t n = slot0 + token + 1;
    const uint32_t see = !a.causal ? len : n < 0 ? 0u : n < (int64_t)len ? (uint32_t)n : len;
    return (see + kTileKeys - 1) / kTileKeys;
  }
  __device__ __forceinline__ static int of(int x, int b) { return __builtin_amdgcn_readlane(x, b); }
  // Tiles of a sequence whose walks are longer than n.  (n < most: 64 n lies in front of the last token's slot, and nothing passes 32 bits;
  // for others the product may, and is not used.)
  __device__ __forceinline__ static int longer(const ChunkArgs &a, int n, int tiles, int most, int slot0) {
    const int x = (int)((uint32_t)n * kTileKeys - (uint32_t)slot0);  // their last rows are of this token at least
    const int first = a.causal && x > 0 ? (int)((uint32_t)x * a.by_group.d / BM) : 0;
    return n < most ? tiles - first : 0;
  }
  __device__ __forceinline__ explicit Layout(const ChunkArgs &args) : a(args), lane(threadIdx.x & 63) {
    const bool in = lane < a.B;
    tokens = in ? tokens_of(a, lane) : 0;
    length = in ? a.lengths[lane] : 0;
    const uint32_t len = slots_of(a, length);
    slot0 = len > 0 ? length - tokens : 0;  // (of a sequence with slots)
    const int rows = tokens * (int)a.by_group.d;
    tiles = (rows + BM - 1) / BM;
    most = tokens > 0 ? (int)walk_of(a, slot0, len, tokens - 1) : 0;
    parts = 1;
    if (a.parts > 1) divide(len, rows);
  }
  // How many parts: lane q - 1 estimates what the call takes, in tiles of a place, with parts of at most a q-th of the longest walk.  Walks
  // of about one length go by the rounds that they need, others are dealt to the places as these become free; a walk needs three
  // tiles' time besides, as a part another three for its result, their join five.
  __device__ __forceinline__ void divide(uint32_t len, int rows) {
    int longest = 0;
    for (int b = 0; b < a.B; ++b) longest = longest > of(most, b) ? longest : of(most, b);
    const int q = lane + 1, per = (longest + q - 1) / q;
    const float share = 1.f / (float)(per > 0 ? per : 1);
    const int mean2 = most + (rows > 0 ? (int)walk_of(a, slot0, len, ((BM < rows ? BM : rows) - 1) / (int)a.by_group.d) : 0);
    float all = 0.f, items = 0.f;
    for (int b = 0; b < a.B; ++b) {
      const float t = (float)(of(tiles, b) * a.Zkv);
      all += t * 0.5f * (float)of(mean2, b);
      items += t * __builtin_ceilf((float)of(most, b) * share);
    }
    constexpr float places = PLACES;
    const float rounds = __builtin_ceilf(items / places), longest_one = PLACES > kCUs && items <= kCUs ? 0.6f * (float)per : (float)per;
    const float walks = all > 0.85f * items * (float)per ? rounds * longest_one : fmaxf(longest_one, all / places + 0.2f * (float)per);
    float cost = walks + items / places * (q > 1 ? 6.f : 3.f) + (q > 1 ? 5.f : 0.f);
    if (q > a.parts) cost = INFINITY;
    float best = cost;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) best = fminf(best, __shfl_xor(best, o));
    const int chosen = __builtin_ctzll(__ballot(cost == best)) + 1, most_of_part = (longest + chosen - 1) / chosen;
    parts = most > most_of_part ? (most + most_of_part - 1) / most_of_part : 1;
  }
  // Items of levels w and more
  __device__ __forceinline__ uint32_t upto(int w) const {
    const int have = longer(a, w > 0 ? (w - 1) * parts : 0, tiles, most, slot0);
    return sum_lanes(lane >= a.B ? 0u : (uint32_t)(w > 0 ? have * parts : have * (parts - 1) + a.tiles)) * (uint32_t)a.Zkv;
  }
  __device__ __forceinline__ bool find(uint32_t id, Item &it) const {
    if (id >= upto(0)) return false;
    int lo = 0, hi = (int)(((uint32_t)a.width * a.by_page.d + kTileKeys - 1) / kTileKeys) + 1;  // F(lo) > id >= F(hi)
    while (hi - lo > 1) {
      const int w = (lo + hi) >> 1;
      if (upto(w) > id) lo = w;
      else hi = w;
    }
    const int above = longer(a, lo * parts, tiles, most, slot0), mine = longer(a, lo > 0 ? (lo - 1) * parts : 0, tiles, most, slot0);
    const uint32_t n = (lane < a.B ? (uint32_t)(lo > 0 ? (mine - above) * parts : a.tiles - mine) : 0u) * (uint32_t)a.Zkv, s = scan_lanes(n);
    const uint32_t r = id - upto(lo + 1);
    const int b = __builtin_ctzll(__ballot(r < s));
    const uint32_t j = r - (uint32_t)of((int)(s - n), b), k = a.by_Zkv(j);
    it.b = (uint32_t)b; it.h = j - k * (uint32_t)a.Zkv;
    it.tokens = of(tokens, b); it.length = of(length, b);
    it.parts = lo > 0 ? of(parts, b) : 1;
    const uint32_t t = it.parts > 1 ? k / (uint32_t)it.parts : k;
    it.part = (int)(k - t * (uint32_t)it.parts);
    const int first = of(tiles - mine, b);  // the first tile of this level; level 0: those in front of the others, those without rows
    it.tile = lo > 0 ? first + (int)t : (int)t < first ? (int)t : of(tiles, b) + (int)t - first;
    return true;
  }
};

// KS: the waves that share a row block's rows, two each with half of a tile's keys; four of them for half of the result's columns, too, since
// probabilities go to the matrix cores with all their bits there, in three parts
template <int AH, int QB, int RW, int KS, bool EIGHT>
__global__ void __launch_bounds__(64 * RW, AH <= 2 || RW == 8 ? 2 : 1) chunk_kernel(ChunkArgs a) {
  constexpr int A = 64 * AH, R = 32 * QB, ROWS = RW / KS, BM = R * ROWS, THREADS = 64 * RW;
  constexpr int PARTS = KS == 4 ? 3 : 1, COLS = KS == 4 ? 2 : 1, DB = 2 * AH / COLS;  // DB: a wave's blocks of 32 columns
  constexpr bool SHARED = KS > 1;                                                    // keys
  constexpr int KB = SHARED || (RW == 8 && (AH == 4 || (AH == 3 && EIGHT))) ? 1 : 2;
  // Long heads' pools in e4m3 wait in LDS (K1, V1) as they are, since registers have no room for them, and are widened into K0 and V0 when their turn
  // comes (2048 tokens of 16384 slots, us: heads of 192 963 -> 764, of 256 1872 -> 1197)
  constexpr bool RAW = EIGHT && RW == 8 && AH > 2;
  // (two buffers, each an object of its own, so that the compiler sees that loads into one miss the reads of the other)
  __shared__ __attribute__((aligned(16))) unsigned char K0[AH][kTileBytes], K1[AH][kTileBytes], V0[AH][kTileBytes], V1[AH][kTileBytes];
  __shared__ float2 shared_ends[SHARED ? BM : 1];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5, block = wave & (ROWS - 1), share = wave / ROWS & 1;
  const int side = COLS == 2 ? wave >> 1 : 0;  // its blocks of columns: one of each 64
  // The lane as a number of its own, from which a tile's addresses are worked out anew where registers are scarce (kept over the walk they
  // would be spilled, and a reload waits for the next tile's loads: heads of 256, 2048 tokens of 16384 slots 1117 -> 1083 us, 1024 of 1024 99 -> 85)
  const auto anew = [&]() __attribute__((always_inline)) {
    int l = lane;
    if constexpr (RW == 8 && KB == 1) asm volatile("" : "+v"(l));
    return l;
  };
  Item it{};
  if (a.B <= kSorted) {
    const Layout<BM, (RW == 8 || AH > 2 ? kCUs : 2 * kCUs)> layout(a);
    if (!layout.find(blockIdx.x, it)) return;
    if (a.parts > 1 && blockIdx.x == 0 && tid < a.B) a.divided[tid] = (uint32_t)layout.parts;
  } else {
    uint32_t head, rank;
    longest_first(blockIdx.x, a.by_heads, head, rank);
    it.b = a.by_Zkv(head); it.h = head - it.b * (uint32_t)a.Zkv; it.tile = a.tiles - 1 - (int)rank; it.parts = 1;
    it.tokens = tokens_of(a, (int)it.b); it.length = a.lengths[it.b];
  }
  const uint32_t b = settled(it.b), h = settled(it.h), head = b * (uint32_t)a.Zkv + h;
  const int parts = (int)settled((uint32_t)it.parts), part = (int)settled((uint32_t)it.part);
  const int group = (int)a.by_group.d, tokens = (int)settled((uint32_t)it.tokens), rows = tokens * group, rows_all = a.T * group;
  const int length = (int)settled((uint32_t)it.length);
  const int row0 = (int)settled((uint32_t)it.tile) * BM;
  const uint32_t len = slots_of(a, length);
  const int64_t slot0 = (int64_t)length - tokens;
  // the first slot that a row does not see
  const auto limit_of = [&](int row) -> uint32_t {
    const int64_t n = slot0 + (int)a.by_group((uint32_t)row) + 1;
    return !a.causal ? len : n < 0 ? 0u : n < (int64_t)len ? (uint32_t)n : len;
  };
  const int last = (row0 + BM < rows ? row0 + BM : rows) - 1;
  const bool some = row0 < rows;
  if (!some && !a.pad) return;
  const uint32_t least = some ? limit_of(row0) : 0u, most = some ? limit_of(last) : 0u;
  // this work-group's tiles of the walk
  const uint32_t all = (most + kTileKeys - 1) / kTileKeys, per = (all + (uint32_t)parts - 1) / (uint32_t)parts;
  uint32_t t = (uint32_t)part * per;
  const uint32_t end = t + per < all ? t + per : all;

  // Q^T operand: lane (col, half) holds elements dk 16 + half 8 .. + 8 of its row
  bf16x8 qreg[QB][4 * AH];
  uint32_t lim[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    int row = row0 + block * R + qb * 32 + col;
    row = row < rows_all ? row : rows_all - 1;
    lim[qb] = row < rows ? limit_of(row) : 0u;
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
  constexpr int PER = 8 / RW, P8 = (64 * (A / 16) + THREADS - 1) / THREADS;
  constexpr bool kUneven = 64 * (A / 16) % THREADS != 0;  // (the last of some threads' pieces is not there: its row is beyond the tile's)
  u32x4 raw[2][EIGHT ? P8 : 1];  // keys, values
  uint32_t exps[2][EIGHT ? P8 : 1];
  const auto place8 = [&](int i, int &row, int &pc) {
    const uint32_t p = i * THREADS + wave * 64 + anew();
    row = (int)a.by_row(p);
    pc = (int)p - row * (A / 16);
  };
  const auto load8 = [&](const Rows &r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < P8; ++i) {
      int row, pc;
      place8(i, row, pc);
      const uint64_t from = __shfl(r.row, row);
      raw[0][i] = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(a.Kc) + from * A + pc * 16);
      raw[1][i] = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(a.Vc) + from * A + pc * 16);
      exps[0][i] = a.Ks[from];
      exps[1][i] = a.Vs[from];
    }
  };
  const auto piece8 = [&](int i, int side) { return (side ? &V1[0][0] : &K1[0][0]) + (i * THREADS + wave * 64) * 16; };  // of the wave's first lane
  const auto load_raw = [&](const Rows &r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < P8; ++i) {
      int row, pc;
      place8(i, row, pc);
      const uint64_t from = __shfl(r.row, row);
      if (kUneven && i * THREADS + wave * 64 >= 64 * (A / 16)) break;  // (whole waves)
      lds_dma16(static_cast<const uint8_t *>(a.Kc) + from * A + pc * 16, piece8(i, 0));
      lds_dma16(static_cast<const uint8_t *>(a.Vc) + from * A + pc * 16, piece8(i, 1));
      exps[0][i] = a.Ks[from];
      exps[1][i] = a.Vs[from];
    }
  };
  const auto store8 = [&](const Rows &r, auto &Kn, auto &Vn) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < P8; ++i) {
      int row, pc;
      place8(i, row, pc);
      if (kUneven && i == P8 - 1 && row >= kTileKeys) continue;
      const bool seen = (r.seen >> row) & 1;
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const float power = __builtin_bit_cast(float, (seen ? exps[side][i] : 127u) << 23);  // (not what lies there)
        const u32x4 x = RAW ? reinterpret_cast<const u32x4 *>(piece8(i, side))[lane] : raw[side][i];
        unsigned char *y = side ? Vn[pc >> 2] : Kn[pc >> 2];
        *reinterpret_cast<u32x4 *>(y + tile_off(row, 2 * (pc & 3))) = widened8(x[0], x[1], power);
        *reinterpret_cast<u32x4 *>(y + tile_off(row, 2 * (pc & 3) + 1)) = widened8(x[2], x[3], power);
      }
    }
  };
  const auto load = [&](const Rows &r, auto &Kn, auto &Vn) __attribute__((always_inline)) {
    const int lane = anew();
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
  };

  f32x16 o[DB][QB];
  float m[QB], mc[QB], l[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = -INFINITY; mc[qb] = 0.f; l[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[db][qb][v] = 0.f;
  }
  Rows now{0, 0}, next{0, 0};
  int id = 0;
  if (t < end) {
    next = rows_of(page_of(t), t);
    if constexpr (RAW) {
      load_raw(next);
      id = page_of(t + 1);
    } else if constexpr (EIGHT) {
      load8(next);
      id = page_of(t + 1);
      store8(next, K0, V0);
    } else {
      load(next, K0, V0);
      id = page_of(t + 1);
    }
  }
  wait_vmem();
  __syncthreads();

  // one tile: start the loads of the next one into (Kn, Vn), compute on (Kt, Vt)
  const auto stage = [&](auto &Kt, auto &Vt, auto &Kn, auto &Vn) __attribute__((always_inline)) {
    TileLanes tl(anew());
    if constexpr (COLS == 2) {
#pragma unroll
      for (int e = 0; e < 2; ++e) tl.cols_off[0][e] = side ? tl.cols_off[1][e] : tl.cols_off[0][e];
    }
    const auto columns = [&](int db, int row) __attribute__((always_inline)) {
      return COLS == 2 ? tl.read_cols(Vt[db], row, 0) : tl.read_cols(Vt[db >> 1], row, db & 1);
    };
    now = next;
    const bool more = t + 1 < end;
    if constexpr (RAW) {  // (a lane reads what it has asked for itself)
      store8(now, Kt, Vt);
      __syncthreads();
    }
    if (more) {
      next = rows_of(id, t + 1);
      if constexpr (RAW) {
        load_raw(next);
      } else if constexpr (EIGHT) {
        load8(next);
      } else {
        load(next, Kn, Vn);
      }
      id = page_of(t + 2);
    }
    const uint32_t k0 = t * kTileKeys;
    const bool edge = now.seen != ~0ull || k0 + kTileKeys > least;  // some row does not see some slot
    if (edge) {
      // values that no row sees to 0; whether others are infinite or NaN
      bool special = false;
#pragma unroll
      for (int i = 0; i < 8 * AH / RW; ++i) {
        const int p = i * THREADS + wave * 64 + anew(), row = (p >> 3) & 63, ah = p >> 9;
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
          for (int db = 0; db < DB; ++db) {
            f32x16 n;
#pragma unroll
            for (int v = 0; v < 16; ++v) n[v] = 0.f;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              __builtin_amdgcn_sched_barrier(0);
              const u32x4 va = __builtin_bit_cast(u32x4, columns(db, kk * 16));
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
          const int p = i * THREADS + wave * 64 + anew(), row = (p >> 3) & 63, ah = p >> 9;
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

    // ---- by blocks of 32 keys: both at once or, where the accumulators leave no room for both's scores, one after the other
#pragma unroll
    for (int k0th = 0; k0th < (SHARED ? 1 : 2); k0th += KB) {
      const int k1 = SHARED ? share : k0th;
      // ---- S^T = K Q^T
      f32x16 s[KB][QB];
      float tm[QB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        bf16x8 ka[4 * AH];
#pragma unroll
        for (int dk = 0; dk < 4 * AH; ++dk) ka[dk] = tl.read_rows(Kt[dk >> 2], (k1 + kb) * 32, dk & 3);
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
          for (int kb = 0; kb < KB; ++kb) {
            const uint32_t seen = ((uint32_t)(now.seen >> ((k1 + kb) * 32)) & low_bits(n - (k1 + kb) * 32)) >> (half * 4);
#pragma unroll
            for (int v = 0; v < 16; ++v) s[kb][qb][v] = keep_bit(s[kb][qb][v], seen, (v >> 2) * 8 + (v & 3));
          }
        }
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float x = s[0][qb][0];
#pragma unroll
        for (int i = 1; i < 16 * KB; ++i) x = fmaxf(x, s[i >> 4][qb][i & 15]);
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
          const Weight w(any ? (m[qb] - mn) * a.cl2 : 0.f);
          m[qb] = mn;
          mc[qb] = any ? mn * a.cl2 : 0.f;
          l[qb] = l[qb] * w.a * w.b;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[db][qb][v] = o[db][qb][v] * w.a * w.b;
        }
      }
      // ---- P^T = exp2(S^T cl2 - m cl2), packed to bf16 as the B operand
      bf16x8 pf[QB][2 * KB][PARTS];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          float p[16];
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            p[v] = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][v], a.cl2, -mc[qb]));
            l[qb] += p[v];
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            u32x4 w[PARTS];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float x = p[u * 8 + 2 * k], y = p[u * 8 + 2 * k + 1];
              if constexpr (PARTS == 3) {
                uint32_t parts[3];
                three_parts(x, y, parts);
#pragma unroll
                for (int i = 0; i < 3; ++i) w[i][k] = parts[i];
              } else {
                w[0][k] = pack_bf16(x, y);
              }
            }
#pragma unroll
            for (int i = 0; i < PARTS; ++i) pf[qb][kb * 2 + u][i] = __builtin_bit_cast(bf16x8, w[i]);
          }
        }
      // ---- O^T += V^T P^T
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int kk = 0; kk < 2 * KB; ++kk) {
          const bf16x8 va = columns(db, (k1 * 2 + kk) * 16);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int i = PARTS - 1; i >= 0; --i) o[db][qb] = mfma_32x32x16(va, pf[qb][kk][i], o[db][qb]);
        }
    }
    if (EIGHT && !RAW && more) store8(next, Kn, Vn);
    wait_vmem();
    __syncthreads();
    ++t;
  };
  while (t < end) {
    stage(K0, V0, K1, V1);
    if constexpr (!RAW) {
      if (t >= end) break;
      stage(K1, V1, K0, V0);
    }
  }

  const int own = COLS == 2 ? side : block & 3;  // the wave's buffer
  if constexpr (SHARED) {  // the shares of a block's rows together, as parts are
    float *other = reinterpret_cast<float *>(own == 0 ? K0[0] : own == 1 ? K1[0] : own == 2 ? V0[0] : V1[0]);
    float2 *ends = shared_ends + block * R + col;
    float lt = xhalf_sum(l[0]), top = lt != 0.f ? mc[0] : -INFINITY;
    if (share == 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          reinterpret_cast<f32x4 *>(other)[(db * 4 + g) * 64 + lane] = f32x4{o[db][0][g * 4 + 0], o[db][0][g * 4 + 1], o[db][0][g * 4 + 2], o[db][0][g * 4 + 3]};
      if (half == 0 && side == 0) *ends = make_float2(top, lt);
    }
    __syncthreads();
    if (share == 1) return;
    const float2 x = *ends;
    const bool one = top > -INFINITY, two = x.x > -INFINITY;
    const float M = fmaxf(top, x.x);
    const Weight w0(top - M), w1(x.x - M);  // (of a share that has seen keys)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 y = reinterpret_cast<const f32x4 *>(other)[(db * 4 + g) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = one ? o[db][0][g * 4 + e] * w0.a * w0.b : 0.f;
          o[db][0][g * 4 + e] = two ? fmaf(w1.a, y[e] * w1.b, z) : z;
        }
      }
    l[0] = half == 0 ? (one ? lt * w0.a * w0.b : 0.f) + (two ? x.y * w1.a * w1.b : 0.f) : 0.f;
    mc[0] = one || two ? M : 0.f;
  }

  if (parts > 1) {  // this part's result
    const int64_t place = ((int64_t)part * a.by_heads.d + head) * a.tiles + it.tile;
    f32x4 *po = reinterpret_cast<f32x4 *>(a.part_o + (place * BM + block * R) * A) + lane;
    float2 *ml = reinterpret_cast<float2 *>(a.part_ml) + place * BM + block * R + col;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float lt = xhalf_sum(l[qb]);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          po[((qb * 2 * AH + (COLS == 2 ? 2 * db + side : db)) * 4 + g) * 64] = f32x4{o[db][qb][g * 4 + 0], o[db][qb][g * 4 + 1], o[db][qb][g * 4 + 2], o[db][qb][g * 4 + 3]};
      if (half == 0 && side == 0) ml[qb * 32] = make_float2(lt != 0.f ? mc[qb] : -INFINITY, lt);
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
    const int row = row0 + block * R + qb * 32 + col;
    if (half == 0 && side == 0 && (row < rows || ((a.pad & 2) && row < rows_all))) {
      const int token = (int)a.by_group((uint32_t)row), z = (int)h * group + row - token * group;
      a.LSE[((int64_t)b * a.Z + z) * a.T + token] = lt != 0.f && row < rows ? (mc[qb] + __builtin_amdgcn_logf(lt)) * kLn2 : -INFINITY;
    }
  }
  unsigned char *ot = (own == 0 ? K0[0] : own == 1 ? K1[0] : own == 2 ? V0[0] : V1[0]) + (block >> 2) * 32 * 128;
#pragma unroll
  for (int ah = 0; ah < AH; ++ah) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) stage_block_T(ot, qb * 32, o[COLS == 2 ? ah : 2 * ah][qb], o[COLS == 2 ? ah : 2 * ah + 1][qb], inv[qb], lane);
#pragma unroll
    for (int it = 0; it < R / 8; ++it) {
      const int r = it * 8 + (lane >> 3), cc = lane & 7, row = row0 + block * R + r;
      if ((COLS == 1 || cc >> 2 == side) && (row < rows || ((a.pad & 1) && row < rows_all))) {
        const int token = (int)a.by_group((uint32_t)row), z = (int)h * group + row - token * group;
        *reinterpret_cast<u32x4 *>(a.O + (int64_t)b * a.os[0] + (int64_t)z * a.os[1] + (int64_t)token * a.os[2] + ah * 64 + cc * 8) =
            row < rows ? *reinterpret_cast<const u32x4 *>(ot + tile_off(r, cc)) : u32x4{0, 0, 0, 0};
      }
    }
  }
}

// The parts of divided walks: with M the largest of a row's maxima, O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s.  A part that
// saw no key of the row has m = -inf and is left out.  Memory bounds it (8 x 512 tokens of up to 16384 slots: 15 us of 505).
// A work-group has 32 rows, a thread 16 bytes of every 32 columns as a lane of the
// accumulators had them; the rows leave through LDS.
template <int AH>
__global__ void __launch_bounds__(256) chunk_join_kernel(ChunkArgs a, int BM) {
  constexpr int A = 64 * AH;
  __shared__ __attribute__((aligned(16))) uint16_t out[32][A + 8];
  const uint32_t blocks = (uint32_t)(a.tiles * (BM / 32)), head = blockIdx.x / blocks, block = blockIdx.x - head * blocks;
  const uint32_t b = a.by_Zkv(head), h = head - b * (uint32_t)a.Zkv;
  const int parts = (int)a.divided[b], group = (int)a.by_group.d, tokens = tokens_of(a, (int)b), have = tokens * group;
  const int row0 = (int)block * 32, first = row0 / BM * BM;
  if (parts <= 1 || first >= have) return;
  // (a tile that sees nothing is not divided)
  const int last = (first + BM < have ? first + BM : have) - 1;
  if (a.causal && (int64_t)a.lengths[b] - tokens + (int)a.by_group((uint32_t)last) < 0) return;
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6, col = lane & 31, half = lane >> 5, row = row0 + col;
  const int64_t step = (int64_t)a.by_heads.d * a.tiles * BM, rows = (int64_t)head * a.tiles * BM + row0;
  const f32x4 *po = reinterpret_cast<const f32x4 *>(a.part_o + rows * A) + g * 64 + lane;
  const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + rows + col;
  float M = -INFINITY, sum = 0.f;
  f32x4 o[2 * AH];
#pragma unroll
  for (int db = 0; db < 2 * AH; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < parts; ++s) M = fmaxf(M, ml[s * step].x);
#pragma unroll 2
  for (int s = 0; s < parts; ++s) {
    const float2 x = ml[s * step];
    f32x4 y[2 * AH];
#pragma unroll
    for (int db = 0; db < 2 * AH; ++db) y[db] = po[s * step * (A / 4) + db * 256];
    const Weight w(x.x - M);
    sum = x.x > -INFINITY ? fmaf(w.a, x.y * w.b, sum) : sum;
#pragma unroll
    for (int db = 0; db < 2 * AH; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[db][e] = x.x > -INFINITY ? fmaf(w.a, y[db][e] * w.b, o[db][e]) : o[db][e];
  }
  const bool there = row < have;
  const float inv = sum != 0.f ? 1.0f / sum : 0.f;
#pragma unroll
  for (int db = 0; db < 2 * AH; ++db)
    *reinterpret_cast<u32x2 *>(&out[col][db * 32 + g * 8 + half * 4]) =
        there ? u32x2{pack_bf16(o[db][0] * inv, o[db][1] * inv), pack_bf16(o[db][2] * inv, o[db][3] * inv)} : u32x2{0, 0};
  const auto place = [&](int r, int &token, int &z) { token = (int)a.by_group((uint32_t)r); z = (int)h * group + r - token * group; };
  const int all = a.T * group;
  if (g == 0 && half == 0 && (there || ((a.pad & 2) && row < all))) {
    int token, z;
    place(row, token, z);
    a.LSE[((int64_t)b * a.Z + z) * a.T + token] = there && sum != 0.f ? (M + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * (A / 8); i += 256) {
    const int r = i / (A / 8), c = i - r * (A / 8), y = row0 + r;
    if (y < have || ((a.pad & 1) && y < all)) {
      int token, z;
      place(y, token, z);
      *reinterpret_cast<u32x4 *>(a.O + (int64_t)b * a.os[0] + (int64_t)z * a.os[1] + (int64_t)token * a.os[2] + c * 8) =
          *reinterpret_cast<const u32x4 *>(&out[r][c * 8]);
    }
  }
}

// How a call is laid over the chip, from what the host knows: the tokens and the table's width, not counts and lengths.
// Work-groups.  256 rows by eight waves read a tile from memory for twice the rows, but leave a CU to one work-group: heads of 192 and 256, whose four
// waves would be alone on it too (2048 tokens of 16384 slots, 8 key heads, us: 1073 -> 747, 1504 -> 1083, in e4m3 1657 -> 764, 1872 -> 1197; 1024 of 1024,
// 4 x 16 key heads of 256, 82 -> 85 and 112 -> 97), and of 128 where these work-groups fill the chip twice, or
// once with walks of about one length (the same 512 -> 501, 64k slots 2145 -> 1973, 8 x 512 of 8192 572 -> 541, in e4m3 578 -> 527; but 2048 of
// 2048 57 -> 65, 512 of 8192 84 -> 97, 4 x 1024 of 1024, 16 key heads, 36 -> 43).  Heads of 64 take 64 rows a wave where these fill the chip (eight
// waves of 32: 307 -> 341).  Up to 128 rows of a key head half of such a work-group would have none of its own (32 and 64 sequences of 4096, 8 key heads, 4 query heads
// each, us, with and without, bf16 and e4m3: 16 tokens, heads of 128, 164 -> 114 and 157 -> 88; 24 tokens, heads of 128, 324 -> 249 and 308 -> 213, of 64
// 196 -> 133 and 214 -> 150).
// Fewer rows leave waves without any, or CUs with few waves.  Two waves then share 32 rows, each with half of a tile's keys, and are joined at the end: up to
// 64 rows on four waves (16 tokens of each of 16 sequences of 4096, 4 query heads a key head, us, before and with it, bf16 and e4m3: heads of 64
// 37 -> 34, 39 -> 32, of 128 68 -> 65, 58 -> 46, of 192 114 -> 101, 115 -> 86, of 256 146 -> 127, 198 -> 127), up to 128 of long heads on eight (32 tokens:
// heads of 192 118 -> 107, 115 -> 98, of 256 in e4m3 195 -> 165; in bf16 these spill, 148 -> 181, and take four waves, one a row block).
// Up to 32 rows four waves share them, two by two each half of the columns besides (P's three parts on all columns by two waves: heads of 64 36 -> 40 us, in e4m3
// 36 -> 40, of 192 95 -> 108, 83 -> 106, of 256 121 -> 136).
// Up to 16 rows go straight from memory to the operands; up to 32 in heads of 128 and, in e4m3, of 256 (8 tokens of each of 16 sequences of 4096, of 64 of 1024, 4
// query heads a key head, 30 of one of 65536, 16 heads, us, so and by tiles in LDS, in bf16 heads of 64 47 and 36, 60 and 30, 68 and 69, of 128 66 and 64, 68 and 58,
// 111 and 123, of 192 140 and 95, 136 and 92, 230 and 156, of 256 173 and 121, 199 and 120, 289 and 198; in e4m3 of 64 42 and 36, 54 and 29, 58 and 68, of 128 48 and 49, 48
// and 46, 75 and 96, of 192 86 and 83, 84 and 80, 142 and 142, of 256 99 and 107, 119 and 106, 167 and 188; the smallest calls, one tile of one sequence, 6 to 11 and 7 to 14).
struct ChunkPlan {
  bool few;         // by 16 or 32 rows at a time, from memory to the operands (rsa_cache.hip)
  int qb, rw;       // 32-row blocks of a wave, waves of different rows
  int rows;         // of a work-group, 32 qb rw: the row tiles, the parts' places and their join go by it
  int tiles, parts; // row tiles of a key head; parts of a walk at most
};
ChunkPlan plan_of(const CacheDims &d, int T, bool eight) {
  ChunkPlan p{};
  const int64_t rows = (int64_t)T * (d.Z / d.Zkv), heads = (int64_t)d.B * d.Zkv;
  p.few = d.dtype != RSA_BF16 || rows <= (d.A == 128 || (d.A == 256 && eight) ? 32 : 16);
  if (p.few) return p;
  p.qb = 1; const int64_t large = rows > 128 ? heads * ((rows + 255) / 256) : 0, slots = (int64_t)d.width * d.page;
  p.rw = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  if (d.A >= 192 ? rows > 128 : d.A == 128 && (large >= 512 || (large >= 256 && slots >= 4 * (int64_t)T))) p.rw = 8;
  if (d.A == 64 && large >= 512) p.qb = 2;
  p.rows = 32 * p.qb * p.rw;
  p.tiles = (int)((rows + p.rows - 1) / p.rows);
  // Parts.  None where the walks are short for a full chip, where one sequence alone fills two rounds of places (one or two work-groups on a
  // CU), where the only one fills its rounds; else up to eight rounds of them, eight tiles and more a part, results within 512 MB.
  const int64_t wgs = heads * p.tiles, walk = (slots + kTileKeys - 1) / kTileKeys;
  const int64_t places = p.rw == 8 || d.A > 128 ? kCUs : 2 * kCUs;
  const int64_t room = (512LL << 20) / (wgs * p.rows * (d.A + 2) * 4), want = (8 * places + wgs - 1) / wgs;
  const int64_t most = std::min<int64_t>(std::min<int64_t>(walk / 8, room), 32), rounds = (wgs + places - 1) / places;
  const bool whole = d.B > kSorted || (wgs >= places && walk < 64) || wgs / d.B >= 2 * places || (d.B == 1 && wgs * 20 >= rounds * places * 17);
  p.parts = whole ? 1 : (int)(want < most ? want : most > 1 ? most : 1);
  return p;
}

template <int AH, int QB, int RW, int KS>
hipError_t launch_chunk(const ChunkArgs &a, const ChunkPlan &p, hipStream_t st) {
  if (p.rows != 32 * QB * RW / KS) return hipErrorInvalidConfiguration;  // (not the plan's form)
  // (128 rows of heads of 256 in bf16: see plan_of)
  constexpr bool apart = AH == 4 && RW == 8 && KS == 2;
  // (up to 32 rows of heads of 256 in e4m3: by the kernels for few)
  constexpr bool eight = !(AH == 4 && KS == 4);
  const unsigned grid = (unsigned)(a.by_heads.d * p.tiles * p.parts);
  if (a.Ks) {
    if constexpr (eight) chunk_kernel<AH, QB, RW, KS, true><<<grid, 64 * RW, 0, st>>>(a);
    else return hipErrorInvalidConfiguration;
  } else if constexpr (apart) {
    chunk_kernel<AH, QB, 4, 1, false><<<grid, 256, 0, st>>>(a);
  } else {
    chunk_kernel<AH, QB, RW, KS, false><<<grid, 64 * RW, 0, st>>>(a);
  }
  return hipSuccess;
}
template <int AH>
hipError_t launch_chunk(const ChunkArgs &a, const ChunkPlan &p, hipStream_t st) {
  if constexpr (AH > 2) {
    if (p.rw == 4) return launch_chunk<AH, 1, 8, 2>(a, p, st);
  }
  if constexpr (AH == 1) {
    if (p.qb == 2) return launch_chunk<AH, 2, 4, 1>(a, p, st);
  }
  if constexpr (AH != 2) {  // (of heads of 128 the kernels for few take up to 32 rows)
    if (p.rw == 1) return launch_chunk<AH, 1, 4, 4>(a, p, st);
  }
  if (p.rw == 2) return launch_chunk<AH, 1, 4, 2>(a, p, st);
  if constexpr (AH >= 2) {
    if (p.rw == 8) return launch_chunk<AH, 1, 8, 1>(a, p, st);
  }
  if constexpr (AH <= 2) return launch_chunk<AH, 1, 4, 1>(a, p, st);
  return hipErrorInvalidConfiguration;
}
template <int AH>
hipError_t launch_all(const ChunkArgs &a, const ChunkPlan &p, hipStream_t st) {
  const hipError_t e = launch_chunk<AH>(a, p, st);
  if (e != hipSuccess) return e;
  if (p.parts > 1) chunk_join_kernel<AH><<<(unsigned)(a.by_heads.d * a.tiles * (p.rows / 32)), 256, 0, st>>>(a, p.rows);
  return hipGetLastError();
}

}  // namespace

namespace {
size_t part_rows(const CacheDims &d, const ChunkPlan &p) { return (size_t)p.parts * d.B * d.Zkv * p.tiles * p.rows; }
}  // namespace

size_t chunk_workspace_bytes(const CacheDims &d, int T) {
  size_t most = 0;  // (of pools in the queries' type and in e4m3)
  for (const bool eight : {false, true}) {
    const ChunkPlan p = plan_of(d, T, eight);
    const size_t n = p.few ? chunk_few_workspace_bytes(d, T) : p.parts == 1 ? 0 : kSorted * sizeof(uint32_t) + part_rows(d, p) * (d.A + 2) * 4;
    most = n > most ? n : most;
  }
  return most;
}

hipError_t cache_attend_chunk(const CacheDims &d, const CachePools &c, int T, int causal, int pad, const void *Q, const int32_t *table,
                              const int32_t *lengths, const int32_t *counts, void *O, float *LSE, void *ws, hipStream_t st) {
  const ChunkPlan p = plan_of(d, T, c.Ks != nullptr);
  if (p.few) return chunk_few(d, c, T, causal, pad, Q, table, lengths, counts, O, LSE, ws, st);
  ChunkArgs a{};
  a.Q = static_cast<const uint16_t *>(Q); a.Kc = c.Kc; a.Vc = c.Vc; a.Ks = c.Ks; a.Vs = c.Vs;
  a.table = table; a.lengths = lengths; a.counts = counts; a.O = static_cast<uint16_t *>(O); a.LSE = LSE;
  for (int k = 0; k < 3; ++k) { a.qs[k] = d.qs[k]; a.os[k] = d.os[k]; }
  a.by_page = make_fast_div(d.page); a.by_group = make_fast_div(d.Z / d.Zkv);
  a.by_heads = make_fast_div((int64_t)d.B * d.Zkv); a.by_Zkv = make_fast_div(d.Zkv); a.by_row = make_fast_div(d.A / 16);
  a.B = d.B; a.Z = d.Z; a.Zkv = d.Zkv; a.T = T; a.pages = d.pages; a.width = d.width; a.causal = causal; a.pad = pad; a.tiles = p.tiles;
  a.cl2 = d.scale * kLog2e;
  a.parts = p.parts;
  if (p.parts > 1) {
    a.divided = static_cast<uint32_t *>(ws);
    a.part_o = static_cast<float *>(ws) + kSorted;
    a.part_ml = a.part_o + part_rows(d, p) * d.A;
  }
  switch (d.A) {
    case 64: return launch_all<1>(a, p, st);
    case 128: return launch_all<2>(a, p, st);
    case 192: return launch_all<3>(a, p, st);
    default: return launch_all<4>(a, p, st);
  }
}

}  // namespace rsa
