// Rotation of queries and keys by position (rsa_rotate, rsa_rotate_bwd).
//
// y = x turned by its token's angles: every element is read and written once, so HBM bounds it.  The angles are the same for all
// heads, and 75 instructions each: a work-group takes a few rows, works out their angles and turns these rows of several
// heads, all of whose loads are in flight meanwhile.  Eight rows of a head are 1 or 2 KB in one piece; with four of 128 elements
// (B4 Z8 L8192, bf16) the two tensors took 54 us, with eight 50, with sixteen 51; with eight of 64 (B8 Z16 L2048) 26, with sixteen 28.
// All sequences' heads by one work-group, their angles worked out once, 55 and 29.5: too many pieces far apart at a time.
// Nontemporal loads or stores: 4 to 30 us slower.
#include "rsa_kernels.h"
#include "rsa_rotary.h"

namespace rsa {
namespace {

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

template <typename T, int W>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs args) {
  constexpr int ahead = kAhead<T, W>;
  __shared__ float2 angles[1024];  // rows of a tile times R / 2: below lanes * W
  const TurnShape &sh = args.shape;
  const uint32_t tid = threadIdx.x, head0 = sh.by_lanes(tid), lane = tid - head0 * sh.lanes, rr = sh.by_units(lane);
  const int u = (int)(lane - rr * sh.by_units.d), heads = 256 / sh.lanes, step = heads;
  const uint32_t tile = blockIdx.z * gridDim.x + blockIdx.x;
  if (tile >= args.side[0].tiles + args.side[1].tiles) return;
  const bool keys = tile >= args.side[0].tiles;
  const Side &s = args.side[keys ? 1 : 0];
  const uint32_t n0 = (tile - (keys ? args.side[0].tiles : 0u)) * sh.rows, n = n0 + rr;
  const bool have = rr < (uint32_t)sh.rows && n < s.rows;
  const int2 at = Pair<T, W>::place(args.ro, u);
  const int64_t row = (int64_t)n * s.st[2];
  const auto offset = [&](int h) { return head_offset((uint32_t)h, args.by_Z, s.st) + row; };
  const int h = have ? (int)(blockIdx.y * ahead * heads + head0) : args.heads;
  Pair<T, W> p[ahead];
#pragma unroll
  for (int k = 0; k < ahead; ++k)
    if (h + k * step < args.heads) p[k].load(static_cast<const T *>(s.x) + offset(h + k * step), at);
  for (uint32_t e = tid; e < sh.rows * sh.by_half.d; e += 256) {
    const uint32_t ar = sh.by_half(e);
    if (n0 + ar >= s.rows) break;
    const int64_t pos = keys ? (int64_t)(n0 + ar) : args.map((int64_t)(n0 + ar));
    const float2 cs = angle_of(pos, args.ro.inv_freq[e - ar * sh.by_half.d]);
    angles[e] = make_float2(cs.x, args.ro.sign * cs.y);
  }
  barrier_lds();
  const bool turns = u < args.ro.R / (2 * W);
  float2 cs[W];
#pragma unroll
  for (int k = 0; k < W; ++k) cs[k] = turns ? angles[(have ? rr * sh.by_half.d : 0u) + u * W + k] : make_float2(1.f, 0.f);
#pragma unroll
  for (int k = 0; k < ahead; ++k)
    if (h + k * step < args.heads) {
      if (turns) p[k].turn(cs, args.ro.adjacent);
      p[k].store(static_cast<T *>(s.y) + offset(h + k * step), at);
    }
}

template <typename T>
void launch(const RotateArgs &a, int W, dim3 grid, hipStream_t st) {
  constexpr int wide = sizeof(T) == 2 ? 8 : 4;
  if (W == wide) rotate_kernel<T, wide><<<grid, 256, 0, st>>>(a);
  else if constexpr (sizeof(T) == 2) {
    if (W == 4) rotate_kernel<T, 4><<<grid, 256, 0, st>>>(a);
    else if (W == 2) rotate_kernel<T, 2><<<grid, 256, 0, st>>>(a);
    else rotate_kernel<T, 1><<<grid, 256, 0, st>>>(a);
  } else rotate_kernel<T, 1><<<grid, 256, 0, st>>>(a);
}

}  // namespace

hipError_t rotate_rows(const Dims &d, int dtype, int R, int adjacent, const float *inv_freq, bool back, const void *Q,
                       const void *K, void *Qr, void *Kr, hipStream_t st) {
  const int W = chunk_width(dtype, R);
  RotateArgs a{};
  a.ro = {R, adjacent, inv_freq, back ? -1.f : 1.f};
  a.shape = make_turn_shape(d.A, R, W, 8 * (d.A / (2 * W)));
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
  const uint32_t tiles = a.side[0].tiles + a.side[1].tiles, each = heads_in_flight(dtype, W) * (256 / a.shape.lanes);
  const uint32_t x = tiles < (1u << 22) ? tiles : (1u << 22);  // (a dimension of a grid has less than 2^32 threads)
  const dim3 grid(x, (a.heads + each - 1) / each, (tiles + x - 1) / x);
  if (dtype == RSA_BF16) launch<bf16_t>(a, W, grid, st);
  else launch<float>(a, W, grid, st);
  return hipGetLastError();
}

}  // namespace rsa
