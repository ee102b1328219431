// Rotation of queries and keys by position (rsa_rotate, rsa_rotate_bwd).
//
// y = x turned by its token's angles: every element is read and written once, so HBM bounds it.  A work-group takes a few rows
// of one sequence, works out their angles (one a thread) and turns all heads of these rows with them.
#include "rsa_kernels.h"
#include "rsa_rotary.h"

namespace rsa {
namespace {

struct Side {  // Q or K
  const void *x;
  void *y;
  int64_t st[3];
  FastDiv by_rows;  // rows of a sequence
  uint32_t rows;    // of all sequences
  uint32_t tiles;
};
struct RotateArgs {
  Side side[2];
  Rotary ro;
  TurnShape shape;
  RowMap map;  // rows of Q
  int Z;
};

template <typename T, int W>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs args) {
  __shared__ float2 angles[256];
  const TurnShape &sh = args.shape;
  const uint32_t tid = threadIdx.x, head0 = sh.by_lanes(tid), lane = tid - head0 * sh.lanes, rr = sh.by_units(lane);
  const int u = (int)(lane - rr * sh.by_units.d), heads = 256 / sh.lanes;
  const uint32_t ar = sh.by_half(tid), ai = tid - ar * sh.by_half.d;  // this thread's angle
  const int2 at = Pair<T, W>::place(args.ro, u);
  const bool turns = u < args.ro.R / (2 * W);
  const uint32_t tiles = args.side[0].tiles + args.side[1].tiles;
  for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const bool keys = tile >= args.side[0].tiles;
    const Side &s = args.side[keys ? 1 : 0];
    const uint32_t n0 = (tile - (keys ? args.side[0].tiles : 0u)) * sh.rows;
    if (tile != blockIdx.x) __syncthreads();  // (the angles of the tile before are read)
    if (ar < (uint32_t)sh.rows && n0 + ar < s.rows) {
      const uint32_t n = n0 + ar, r = n - s.by_rows(n) * s.by_rows.d;
      const float2 cs = angle_of(keys ? (int64_t)r : args.map((int64_t)r), args.ro.inv_freq[ai]);
      angles[tid] = make_float2(cs.x, args.ro.sign * cs.y);
    }
    __syncthreads();
    const uint32_t n = n0 + rr;
    if (rr >= (uint32_t)sh.rows || n >= s.rows) continue;
    float2 cs[W];
    if (turns) {
#pragma unroll
      for (int k = 0; k < W; ++k) cs[k] = angles[rr * sh.by_half.d + u * W + k];
    }
    const uint32_t b = s.by_rows(n);
    const int64_t off = (int64_t)b * s.st[0] + (int64_t)(n - b * s.by_rows.d) * s.st[2];
    for (int h = (int)head0; h < args.Z; h += heads) {
      Pair<T, W> p;
      p.load(static_cast<const T *>(s.x) + off + h * s.st[1], at);
      if (turns) p.turn(cs, args.ro.adjacent);
      p.store(static_cast<T *>(s.y) + off + h * s.st[1], at);
    }
  }
}

template <typename T>
void launch(const RotateArgs &a, int W, unsigned grid, hipStream_t st) {
  constexpr int wide = sizeof(T) == 2 ? 8 : 4;
  if (W == wide) rotate_kernel<T, wide><<<grid, 256, 0, st>>>(a);
  else if constexpr (sizeof(T) == 2) {
    if (W == 2) rotate_kernel<T, 2><<<grid, 256, 0, st>>>(a);
    else rotate_kernel<T, 1><<<grid, 256, 0, st>>>(a);
  } else rotate_kernel<T, 1><<<grid, 256, 0, st>>>(a);
}

}  // namespace

hipError_t rotate_rows(const Dims &d, int dtype, int R, int adjacent, const float *inv_freq, bool back, const void *Q,
                       const void *K, void *Qr, void *Kr, hipStream_t st) {
  const int W = chunk_width(dtype, R);
  RotateArgs a{};
  a.ro = {R, adjacent, inv_freq, back ? -1.f : 1.f};
  a.shape = make_turn_shape(d.A, R, W);
  a.map = make_row_map(d);
  a.Z = d.Z;
  for (int i = 0; i < 2; ++i) {
    Side &s = a.side[i];
    const int64_t rows = i ? d.L : d.Lq;
    s.x = i ? K : Q; s.y = i ? Kr : Qr;
    for (int k = 0; k < 3; ++k) s.st[k] = i ? d.ks[k] : d.qs[k];
    s.by_rows = make_fast_div(rows);
    s.rows = s.x ? (uint32_t)(d.B * rows) : 0;
    s.tiles = (s.rows + a.shape.rows - 1) / a.shape.rows;
  }
  const uint64_t tiles = (uint64_t)a.side[0].tiles + a.side[1].tiles;
  const unsigned grid = (unsigned)(tiles < (1u << 20) ? tiles : (1u << 20));
  if (grid == 0) return hipSuccess;
  if (dtype == RSA_BF16) launch<bf16_t>(a, W, grid, st);
  else launch<float>(a, W, grid, st);
  return hipGetLastError();
}

}  // namespace rsa
