"""Several new tokens where infinite values lie in the first tile that a row walks, or beside keys of far larger scores than all before:
rows that see them get them, everything else is as without them, to the bit."""
import pytest
import torch

from cache8_helpers import i32
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu

INF = float("inf")
# A, sequences, query and key heads, tokens: four waves that share 32 rows, two (of up to 64, of up to 128), waves of their own, 256 rows a work-group
# (of 64 rows a wave, of eight waves), and few rows
FORMS = [(64, 2, 2, 2, 30), (64, 1, 4, 2, 9), (192, 1, 2, 2, 30), (256, 1, 2, 2, 32), (64, 1, 2, 2, 40), (64, 1, 4, 2, 40), (64, 1, 2, 1, 200), (64, 16, 32, 8, 200),
         (128, 1, 2, 2, 40), (128, 1, 4, 2, 40), (128, 1, 2, 1, 200), (128, 8, 32, 8, 500),
         (192, 1, 2, 2, 40), (192, 1, 4, 2, 40), (192, 1, 2, 1, 200),
         (256, 1, 2, 2, 40), (256, 1, 4, 2, 40), (256, 1, 2, 1, 200), (64, 2, 2, 2, 7), (128, 2, 2, 2, 30), (256, 2, 2, 2, 9)]
PAGE = 16


class Call:
    def __init__(self, A, B, Z, Zkv, T, n, causal=True, scale=0.0, holes=()):
        g = torch.Generator(device="cuda").manual_seed(51)
        W = -(-n // PAGE)
        self.K, self.V = (torch.randn(B * W, Zkv, PAGE, A, generator=g, device="cuda").bfloat16() for _ in range(2))
        self.table = torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).int()
        self.where = self.table.tolist()
        for p in holes:
            self.table[:, p] = -1
        self.Q = torch.randn(B, Z, T, A, generator=g, device="cuda").bfloat16()
        self.d, self.lengths, self.causal = rsa.make_cache_desc(self.K, self.table, Z, scale=scale), i32([n] * B), causal

    def __call__(self):
        return [x.clone() for x in rsa.cache_attend_chunk(self.d, self.Q, self.K, self.V, self.table, self.lengths, causal=self.causal)]

    def put(self, pool, b, h, slot, col, value):
        pool[self.where[b][slot // PAGE], h, slot % PAGE, col] = value


def same_but(got, ref, expected):
    """expected: (sequence, heads, rows, column, value).  (NaN for NaN)"""
    O, R = got[0], ref[0].clone()
    for b, heads, rows, col, value in expected:
        R[b, heads, rows, col] = value
    assert torch.equal(O.isnan(), R.isnan()), f"NaN in {(O.isnan() != R.isnan()).nonzero()[:4].tolist()}"
    bad = (O != R) & ~R.isnan()
    assert not bad.any(), f"{int(bad.sum())} differ, the first at {bad.nonzero()[0].tolist()}: {O[bad][0]} for {R[bad][0]}"
    assert torch.equal(got[1], ref[1])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("gone", [0, 1, 9])
def test_in_the_first_tile_of_a_fresh_prompt(form, gone):
    """... or of one behind pages that are no longer held."""
    A, B, Z, Zkv, T = form
    front = gone * PAGE
    c = Call(A, B, Z, Zkv, T, front + T, holes=range(gone))
    ref = c()
    b, h, group = B - 1, Zkv - 1, Z // Zkv
    heads = slice(h * group, Z)
    for slot, col, value in ((0, 5, INF), (1, 40, -INF), (3, A - 1, INF), (4, 6, INF), (5, 6, -INF), (5, 33, -INF)):
        c.put(c.V, b, h, front + slot, col, value)
    nan = float("nan")
    same_but(c(), ref, [(b, heads, slice(0, T), 5, INF), (b, heads, slice(1, T), 40, -INF), (b, heads, slice(3, T), A - 1, INF),
                        (b, heads, slice(4, 5), 6, INF), (b, heads, slice(5, T), 6, nan), (b, heads, slice(5, T), 33, -INF)])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("front", [128, 150, 160, 192])
def test_beside_scores_far_beyond_all_before(form, front):
    """The slots in front of the tokens have scores of -1000, the tokens' own 0: the first have probabilities of 0 in the end, whatever they
    were worth before the others came."""
    A, B, Z, Zkv, T = form
    n = front + T
    c = Call(A, B, Z, Zkv, T, n, scale=1.0)
    c.Q.zero_()
    c.Q[..., 0] = 8.0
    for b in range(B):
        for j in range(n):
            c.K[c.where[b][j // PAGE], :, j % PAGE, 0] = -125.0 if j < front else 0.0
    ref = c()
    b, group = B - 1, Z // Zkv
    heads = slice(0, group)
    c.put(c.V, b, 0, front + 2, 5, INF)
    c.put(c.V, b, 0, front, 7, -INF)
    same_but(c(), ref, [(b, heads, slice(2, T), 5, INF), (b, heads, slice(0, T), 7, -INF)])


@pytest.mark.parametrize("form", FORMS + [(64, 1, 2, 2, 64), (128, 1, 2, 1, 60), (192, 1, 2, 1, 100), (256, 1, 2, 1, 200)])
def test_in_every_tile_of_divided_walks(form):
    """A page of each tile is not held, an infinite value in each tile; all rows see all slots."""
    A, B, Z, Zkv, T = form
    n = 4000 if B == 1 else 700
    c = Call(A, B, Z, Zkv, T, n, causal=False, holes=range(2, -(-n // PAGE), 4))
    ref = c()
    group, expected = Z // Zkv, []
    for j, slot in enumerate(range(3, n, 64)):
        value = -INF if j % 2 else INF
        c.put(c.V, 0, 0, slot, j % A, value)
        expected.append((0, slice(0, group), slice(0, T), j % A, value))
    same_but(c(), ref, expected)
