// The paged cache of keys and values: appending to it, attention of one new token per sequence to it, and the join of
// results over shares of it (rsa_cache_append, rsa_cache_attend, rsa_cache_join).
#include "rsa_kernels.h"
#include "rsa_rotary.h"

namespace rsa {
namespace {

// ---------------------------------------------------------------- append ----
struct AppendArgs {
  const void *Q, *K, *V;
  void *Qr, *Kc, *Vc;
  const int32_t *table, *lengths, *counts, *first;
  int64_t qs[3], ks[3];
  Rotary ro;
  TurnShape shape;
  FastDiv by_T, by_page;
  int B, Zq, Zkv, A, pages, width;  // Zq: 0 without queries
  uint32_t tokens, tiles;           // B T
};

// Token t of sequence b: whether it is there, its slot.
struct Token {
  uint32_t b, t;
  int64_t slot;
  bool there;
};
__device__ __forceinline__ Token token_of(const AppendArgs &a, uint32_t n) {
  Token k;
  k.b = a.by_T(n); k.t = n - k.b * a.by_T.d;
  const int T = (int)a.by_T.d, c = a.counts ? a.counts[k.b] : T, count = c < T ? c : T;
  k.there = (int)k.t < count;
  k.slot = (int64_t)a.lengths[k.b] - count + k.t;
  return k;
}

// A work-group takes a few tokens, works out their angles (one a thread), turns their heads of Q and K and moves those of V.
template <typename T, int W>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs args) {
  __shared__ float2 angles[256];
  const TurnShape &sh = args.shape;
  const uint32_t tid = threadIdx.x, head0 = sh.by_lanes(tid), lane = tid - head0 * sh.lanes, rr = sh.by_units(lane);
  const int u = (int)(lane - rr * sh.by_units.d), heads = 256 / sh.lanes, half = args.ro.R / 2;
  const uint32_t ar = sh.by_half(tid), ai = tid - ar * sh.by_half.d;  // this thread's angle
  const int2 at = Pair<T, W>::place(args.ro, u);
  const bool turns = u < args.ro.R / (2 * W);
  for (uint32_t tile = blockIdx.x; tile < args.tiles; tile += gridDim.x) {
    const uint32_t n0 = tile * sh.rows;
    if (tile != blockIdx.x) __syncthreads();  // (the angles of the tile before are read)
    if (half && ar < (uint32_t)sh.rows && n0 + ar < args.tokens) {
      const Token k = token_of(args, n0 + ar);
      angles[tid] = angle_of(k.slot + (args.first ? args.first[k.b] : 0), args.ro.inv_freq[ai]);
    }
    __syncthreads();
    const uint32_t n = n0 + rr;
    if (rr >= (uint32_t)sh.rows || n >= args.tokens) continue;
    const Token k = token_of(args, n);
    if (!k.there) continue;
    float2 cs[W];
    if (turns) {
#pragma unroll
      for (int i = 0; i < W; ++i) cs[i] = angles[rr * half + u * W + i];
    }
    // where its keys and values go; -1: nowhere
    int64_t dst = -1;
    const uint32_t page = args.by_page.d;
    if (k.slot >= 0 && k.slot < (int64_t)args.width * page) {
      const uint32_t pg = args.by_page((uint32_t)k.slot);
      const int id = args.table[(int64_t)k.b * args.width + pg];
      if (id >= 0 && id < args.pages) dst = ((int64_t)id * args.Zkv * page + ((uint32_t)k.slot - pg * page)) * args.A;
    }
    const int64_t q = (int64_t)k.b * args.qs[0] + (int64_t)k.t * args.qs[2], kv = (int64_t)k.b * args.ks[0] + (int64_t)k.t * args.ks[2];
    for (int h = (int)(blockIdx.y * heads + head0); h < args.Zq + 2 * args.Zkv; h += heads * gridDim.y) {
      const bool query = h < args.Zq, value = h >= args.Zq + args.Zkv;
      if (!query && dst < 0) break;
      const int z = query ? h : h - args.Zq - (value ? args.Zkv : 0);
      const T *src = query ? static_cast<const T *>(args.Q) + q + z * args.qs[1]
                           : static_cast<const T *>(value ? args.V : args.K) + kv + z * args.ks[1];
      T *to = query ? static_cast<T *>(args.Qr) + q + z * args.qs[1]
                    : static_cast<T *>(value ? args.Vc : args.Kc) + dst + (int64_t)z * page * args.A;
      Pair<T, W> p;
      p.load(src, at);
      if (turns && !value) p.turn(cs, args.ro.adjacent);
      p.store(to, at);
    }
  }
}

template <typename T>
void launch_append(const AppendArgs &a, int W, dim3 grid, hipStream_t st) {
  constexpr int wide = sizeof(T) == 2 ? 8 : 4;
  if (W == wide) append_kernel<T, wide><<<grid, 256, 0, st>>>(a);
  else if constexpr (sizeof(T) == 2) {
    if (W == 2) append_kernel<T, 2><<<grid, 256, 0, st>>>(a);
    else append_kernel<T, 1><<<grid, 256, 0, st>>>(a);
  } else append_kernel<T, 1><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- attend ----
struct AttendArgs {
  const void *Q, *Kc, *Vc;
  const int32_t *table, *lengths;
  void *O;
  float *LSE;
  int64_t qs[3], os[3];
  FastDiv by_page;
  int Z, Zkv, group, A, pages, width;
  float scale;
};

// One work-group a row: scores of 256 keys at a time, their softmax against the running maximum, their values summed.
template <typename T>
__global__ __launch_bounds__(256) void attend_kernel(AttendArgs args) {
  __shared__ float q[256], p[256], red[8];
  __shared__ int64_t row[256];
  const int tid = threadIdx.x, b = blockIdx.x / args.Z, z = blockIdx.x - b * args.Z, h = z / args.group, A = args.A;
  if (tid < A) q[tid] = (float)static_cast<const T *>(args.Q)[b * args.qs[0] + z * args.qs[1] + tid];
  const int64_t page = args.by_page.d, most = args.width * page;
  int64_t len = args.lengths[b];
  len = len < 0 ? 0 : len < most ? len : most;
  float m = -INFINITY, sum = 0.f, o = 0.f;
  for (int64_t j0 = 0; j0 < len; j0 += 256) {
    __syncthreads();
    const int64_t j = j0 + tid;
    float s = -INFINITY;
    int64_t at = -1;
    if (j < len) {
      const uint32_t pg = args.by_page((uint32_t)j);
      const int id = args.table[(int64_t)b * args.width + pg];
      if (id >= 0 && id < args.pages) {
        at = (((int64_t)id * args.Zkv + h) * page + (j - pg * page)) * A;
        s = 0.f;
        for (int a = 0; a < A; ++a) s += q[a] * (float)static_cast<const T *>(args.Kc)[at + a];
        s *= args.scale;
      }
    }
    row[tid] = at;
    const float w = wave_max(s);
    if ((tid & 63) == 0) red[tid >> 6] = w;
    __syncthreads();
    const float mn = fmaxf(fmaxf(m, fmaxf(red[0], red[1])), fmaxf(red[2], red[3])), ref = mn == -INFINITY ? 0.f : mn;
    const float e = at >= 0 ? expf(s - ref) : 0.f, keep = expf(m - ref), ws = wave_sum(e);
    p[tid] = e;
    if ((tid & 63) == 0) red[4 + (tid >> 6)] = ws;
    __syncthreads();
    sum = sum * keep + ((red[4] + red[5]) + (red[6] + red[7]));
    o *= keep;
    m = mn;
    if (tid < A)
      for (int k = 0; k < 256; ++k)
        if (row[k] >= 0) o += p[k] * (float)static_cast<const T *>(args.Vc)[row[k] + tid];
  }
  if (tid < A) static_cast<T *>(args.O)[b * args.os[0] + z * args.os[1] + tid] = (T)(sum != 0.f ? o / sum : 0.f);
  if (tid == 0) args.LSE[blockIdx.x] = sum != 0.f ? m + logf(sum) : -INFINITY;
}

// ------------------------------------------------------------------ join ----
// O = sum_n exp(LSE_n - LSE) O_n: a thread takes four elements of a row.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const T *Op, const float *LSEp, T *O, float *LSE, uint32_t n4, uint32_t rows, int N,
                                                   int A, OutLayout lay) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n4) return;
  const uint32_t row = (uint32_t)(((uint64_t)i * 4) / A);
  const int a = (int)((uint64_t)i * 4 - (uint64_t)row * A);
  float m = -INFINITY;
  for (int n = 0; n < N; ++n) m = fmaxf(m, LSEp[(int64_t)n * rows + row]);
  const float ref = m == -INFINITY ? 0.f : m;
  float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int n = 0; n < N; ++n) {
    const float l = LSEp[(int64_t)n * rows + row];
    if (l == -INFINITY) continue;
    const float w = expf(l - ref);
    sum += w;
    const T *x = Op + ((int64_t)n * rows + row) * A + a;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] += w * (float)x[k];
  }
  T *y = O + lay.row_off(row) + a;
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = (T)(sum != 0.f ? o[k] / sum : 0.f);
  if (a == 0) LSE[row] = sum != 0.f ? m + logf(sum) : -INFINITY;
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
  a.shape = make_turn_shape(d.A, R, W);
  a.by_T = make_fast_div(T); a.by_page = make_fast_div(d.page);
  a.B = d.B; a.Zq = Q ? d.Z : 0; a.Zkv = d.Zkv; a.A = d.A; a.pages = d.pages; a.width = d.width;
  a.tokens = (uint32_t)((int64_t)d.B * T);
  a.tiles = (a.tokens + a.shape.rows - 1) / a.shape.rows;
  const dim3 grid(a.tiles < (1u << 20) ? a.tiles : (1u << 20));
  if (d.dtype == RSA_BF16) launch_append<bf16_t>(a, W, grid, st);
  else launch_append<float>(a, W, grid, st);
  return hipGetLastError();
}

size_t cache_workspace_bytes(const CacheDims &) { return 0; }

hipError_t cache_attend(const CacheDims &d, const void *Q, const void *Kc, const void *Vc, const int32_t *table,
                        const int32_t *lengths, void *O, float *LSE, void *, hipStream_t st) {
  AttendArgs a{};
  a.Q = Q; a.Kc = Kc; a.Vc = Vc; a.table = table; a.lengths = lengths; a.O = O; a.LSE = LSE;
  for (int k = 0; k < 3; ++k) { a.qs[k] = d.qs[k]; a.os[k] = d.os[k]; }
  a.by_page = make_fast_div(d.page);
  a.Z = d.Z; a.Zkv = d.Zkv; a.group = d.Z / d.Zkv; a.A = d.A; a.pages = d.pages; a.width = d.width; a.scale = d.scale;
  if (d.dtype == RSA_BF16) attend_kernel<bf16_t><<<d.B * d.Z, 256, 0, st>>>(a);
  else attend_kernel<float><<<d.B * d.Z, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t cache_join(const CacheDims &d, int N, const void *Op, const float *LSEp, void *O, float *LSE, hipStream_t st) {
  const uint32_t rows = (uint32_t)(d.B * d.Z), n4 = rows * (uint32_t)(d.A / 4);
  const OutLayout lay = make_out_layout(d.os, 1, d.Z);
  const dim3 grid((n4 + 255) / 256);
  if (d.dtype == RSA_BF16) join_kernel<<<grid, 256, 0, st>>>((const bf16_t *)Op, LSEp, (bf16_t *)O, LSE, n4, rows, N, d.A, lay);
  else join_kernel<<<grid, 256, 0, st>>>((const float *)Op, LSEp, (float *)O, LSE, n4, rows, N, d.A, lay);
  return hipGetLastError();
}

}  // namespace rsa
