// Where the lanes of a rotation's work-group read, on the host: partners in LDS, angles, for every head size, turned part and type.
#include <cstdio>
#include <vector>

#include "rsa_rotate.hip"

using namespace rsa;

static int check(int dtype, int A, int R) {
  const int W = dtype == RSA_BF16 ? 8 : 4, es = 16 / W;
  const TurnShape s = make_turn_shape(A, R, dtype);
  if (s.chunks * W != A || s.rows * (int)s.by_half.d > kTurnAngles) return 1;
  std::vector<int> seen((size_t)(4 / s.waves * s.rows * s.chunks), 0);
  for (uint32_t thread = 0; thread < 256; ++thread) {
    const Place p(s, thread);
    const bool some = p.row < s.rows;
    if (p.lane != (int)(thread % 64) || p.row < 0 || p.group < 0 || p.group >= 4 / s.waves) return 2;
    if (some) ++seen[(size_t)((p.group * s.rows + p.row) * s.chunks + p.c)];
    for (int e = p.c * W; e < (p.c + 1) * W; ++e) {
      // bytes of the wave's 1 KB that the partner is read from: a place of the same row, or of the lane's own chunk
      const int from = partner_of(e, R), at = (p.lane - p.c) * 16 + from * es;
      const int first = some && e < R ? (p.lane - p.c) * 16 : p.lane * 16, size = some && e < R ? A * es : 16;
      if (p.lane < p.c || at < first || at + es > first + size || at + es > 1024) return 3;
      if (partner_of(from, R) != e || (e < R && (from == e || from >= R))) return 4;
      if (!some && e < R) return 5;  // (an angle would be read)
    }
  }
  for (int n : seen)
    if (n != 1) return 6;
  return 0;
}

int main() {
  int bad = 0;
  for (int dtype : {RSA_BF16, RSA_F32})
    for (int A = 64; A <= 256; A += 64)
      for (int R = 2; R <= A; R += 2)
        if (const int why = check(dtype, A, R)) {
          std::printf("dtype %d A %d R %d: %d\n", dtype, A, R, why);
          ++bad;
        }
  if (!bad) std::puts("TURNS_OK");
  return bad != 0;
}
