"""Attention of several new tokens per sequence to the paged cache against the fp64 oracle, pools in the queries' type and in e4m3."""
import numpy as np
import pytest
import torch

from cache8_helpers import Cache8, chunk, compare_chunk, i32, scales_of, vectorised_chunk
from cache_helpers import DTYPES, F32, STEP, Cache, f64, frequencies, normal, within
from oracle import cache as oracle
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu

CASES = [  # dtype, Z, Zkv, A, page, T, lengths, counts, causal
    ("bf16", 4, 4, 64, 16, 1, [1, 17, 16, 0], None, True),
    ("bf16", 8, 2, 128, 16, 4, [100, 4, 37, 3, 0], None, True),               # tokens in front of slot 0
    ("bf16", 8, 2, 128, 16, 5, [100, 5, 37], [5, 3, 0], False),
    ("bf16", 6, 2, 64, 5, 9, [30, 9, 11], [9, 12, -1], True),                 # counts outside 0 .. T
    ("bf16", 32, 1, 64, 24, 1, [300, 5], None, True),
    ("bf16", 3, 1, 192, 7, 10, [40, 12], None, True),
    ("bf16", 2, 2, 256, 16, 17, [50, 17], [17, 9], True),
    ("bf16", 4, 4, 64, 16, 33, [33, 70, 200], None, True),                    # beyond 32 rows
    ("bf16", 4, 4, 64, 1, 40, [64, 40], [40, 1], True),                       # pages of one token
    ("bf16", 10, 2, 64, 24, 13, [13, 129, 64], [13, 7, 0], True),             # five heads a group, 65 rows
    ("bf16", 8, 2, 128, 16, 64, [64, 65, 190], None, True),
    ("bf16", 8, 2, 128, 100, 50, [200, 60, 20], [50, 50, 50], False),
    ("bf16", 3, 1, 192, 24, 70, [130, 71], [70, 33], True),
    ("bf16", 7, 1, 256, 16, 23, [90, 23], None, True),
    ("bf16", 48, 2, 128, 32, 3, [77, 3], None, True),                         # 72 rows of 24 heads
    ("bf16", 2, 2, 128, 16, 100, [50, 0, 300], [100, 100, 100], True),        # fewer slots than tokens
    ("f32", 4, 4, 64, 16, 1, [1, 17, 0], None, True),
    ("f32", 8, 2, 128, 24, 7, [100, 7, 3], [7, 7, 2], True),
    ("f32", 6, 3, 64, 16, 45, [45, 99], [45, 20], True),
    ("f32", 5, 1, 192, 7, 9, [33, 9], None, False),
    ("f32", 3, 3, 256, 16, 20, [60, 20], None, True),
]


@pytest.mark.parametrize("case", CASES)
def test_chunk(case):
    """The pools hold NaN wherever no sequence has a token."""
    dtype, Z, Zkv, A, page, T, lengths, counts, causal = case
    rng = np.random.default_rng(31)
    c = Cache(rng, lengths, Zkv, A, page, -(-max(lengths) // page) + 1, dtype)
    Q = normal(rng, (len(lengths), Z, T, A), dtype)
    compare_chunk(c, Q, chunk(c, Q, counts, causal), dtype, counts, causal)


@pytest.mark.parametrize("case", [c for c in CASES if c[0] == "bf16"])
def test_chunk_of_a_cache_in_8_bits(case):
    """... and 255 for the exponents there."""
    dtype, Z, Zkv, A, page, T, lengths, counts, causal = case
    rng = np.random.default_rng(32)
    c = Cache8(rng, lengths, Zkv, A, page, -(-max(lengths) // page) + 1)
    Q = normal(rng, (len(lengths), Z, T, A), dtype)
    compare_chunk(c, Q, chunk(c, Q, counts, causal), dtype, counts, causal)


@pytest.mark.parametrize("dtype,kind", [("bf16", Cache), ("f32", Cache), ("bf16", Cache8)])
@pytest.mark.parametrize("T", [3, 50])
@pytest.mark.parametrize("causal", [True, False])
def test_pages_that_are_not_held(dtype, kind, T, causal):
    """Entries outside the pool, at the front, in the middle, everywhere; a length beyond the table; below zero."""
    rng = np.random.default_rng(33)
    c = kind(rng, [200, 200, 200, 200, 200], 2, 64, 16, 13, dtype)
    c.table[0, :9] = -1
    c.table[1, 3:11:2] = 1 << 20
    c.table[2, :] = -2 ** 31
    c.lengths[3] = 2 ** 31 - 1
    c.table[3, 12] = 2 ** 31 - 1                      # (its last page holds NaN behind slot 200)
    c.lengths[4] = -7
    Q = normal(rng, (5, 4, T, 64), dtype)
    got = chunk(c, Q, None, causal)
    compare_chunk(c, Q, got, dtype, None, causal)
    for b in (2, 4):
        assert (got[0][b] == 0).all() and torch.isneginf(got[1][b]).all()


@pytest.mark.parametrize("dtype,T,kind", [("bf16", 7, Cache), ("bf16", 7, Cache8), ("f32", 40, Cache), ("bf16", 80, Cache), ("bf16", 80, Cache8)])
@pytest.mark.parametrize("A", [64, 128])
def test_infinite_and_nan_tokens_reach_the_rows_that_see_them_alone(dtype, T, kind, A):
    """Keys and values of one token, of one head, that are infinite or NaN: the rows in front of it as without it, to the bit."""
    rng = np.random.default_rng(34)
    n = 150
    c = kind(rng, [n, n], 2, A, 16, 10, dtype)
    Q = normal(rng, (2, 4, T, A), dtype)
    ref = chunk(c, Q)
    first = n - T

    def put(which, b, h, slot, col, value):
        at = c.table[b, slot // 16], h, slot % 16
        if kind is Cache8:
            c.bytes[which][at + (col,)] = 127
        else:
            (c.Vc if which else c.Kc)[at + (col,)] = value
    inf, nan = float("inf"), float("nan")
    eight = kind is Cache8
    put(1, 0, 0, first + 2, 5, inf)
    put(1, 0, 0, first + 4, 6, -inf)
    put(1, 0, 0, first + 5, 5, -inf)
    put(1, 0, 1, first + T // 2, A - 1, nan)
    put(0, 1, 1, first + 3, 0, nan)
    O, LSE = (x.clone() for x in chunk(c, Q))
    assert torch.equal(LSE[0], ref[1][0])
    seen = O[0, :2, 2:, 5]
    assert (seen.isnan() if eight else torch.isposinf(seen[:, :3])).all() and seen[:, 3:].isnan().all()
    assert (O[0, :2, 4:, 6].isnan() if eight else torch.isneginf(O[0, :2, 4:, 6])).all()
    assert O[0, 2:, T // 2:, A - 1].isnan().all() and O[1, 2:, 3:].isnan().all() and LSE[1, 2:, 3:].isnan().all()
    for x, r in ((O, ref[0]), (LSE, ref[1])):
        x[1, 2:, 3:] = r[1, 2:, 3:]
    O[0, :2, 2:, 5], O[0, :2, 4:, 6], O[0, 2:, T // 2:, A - 1] = ref[0][0, :2, 2:, 5], ref[0][0, :2, 4:, 6], ref[0][0, 2:, T // 2:, A - 1]
    assert torch.equal(O, ref[0]) and torch.equal(LSE, ref[1])


@pytest.mark.parametrize("A,B,Z,T,n", [(128, 8, 32, 512, 2048), (128, 2, 32, 1024, 4200), (192, 2, 2, 300, 700), (192, 1, 2, 200, 3000), (256, 1, 2, 90, 2000), (256, 2, 2, 300, 700), (256, 1, 8, 100, 3000), (64, 16, 32, 1000, 1000),
                                        (64, 2, 2, 33, 200), (128, 1, 2, 50, 700), (128, 1, 2, 64, 5000), (192, 2, 2, 50, 200), (192, 1, 2, 100, 3000), (256, 1, 2, 50, 600)])
@pytest.mark.parametrize("eight", [False, True])
def test_infinite_and_nan_tokens_of_large_work_groups(A, B, Z, T, n, eight):
    """The same where work-groups have 256 rows, waves share rows or walks are divided: one value of one slot NaN, another head's infinite, one key NaN."""
    g = torch.Generator(device="cuda").manual_seed(45)
    page, Zkv = 16, max(2, Z // 4)
    W = -(-n // page)
    Kc, Vc = (torch.randn(B * W, Zkv, page, A, generator=g, device="cuda").to(torch.float8_e4m3fn if eight else torch.bfloat16) for _ in range(2))
    s = {k: torch.full((B * W, Zkv, page), 127, dtype=torch.uint8, device="cuda") for k in ("Ks", "Vs")} if eight else {}
    table = torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).int()
    Q = torch.randn(B, Z, T, A, generator=g, device="cuda").bfloat16()
    d, lengths = rsa.make_cache_desc(Kc, table, Z), i32([n] * B)
    ref = rsa.cache_attend_chunk(d, Q, Kc, Vc, table, lengths, **s)
    nan = float("nan")
    group, b = Z // Zkv, B - 1
    first = n - T

    def put(pool, h, slot, col, value):
        at = (int(table[b, slot // page]), h, slot % page, col)
        if eight:
            pool.view(torch.uint8)[at] = 127
        else:
            pool[at] = value
    put(Vc, 0, first + T // 3, A - 3, nan)
    put(Vc, 1, first + T // 2, 7, float("inf"))
    put(Kc, 1, first + T - 5, 1, nan)
    O, LSE = (x.clone() for x in rsa.cache_attend_chunk(d, Q, Kc, Vc, table, lengths, **s))
    one, two = slice(0, group), slice(group, 2 * group)
    assert O[b, one, T // 3:, A - 3].isnan().all() and O[b, two, T - 5:].isnan().all() and LSE[b, two, T - 5:].isnan().all()
    seen = O[b, two, T // 2:T - 5, 7]
    assert (seen.isnan() if eight else torch.isposinf(seen)).all()
    O[b, one, T // 3:, A - 3] = ref[0][b, one, T // 3:, A - 3]
    O[b, two, T // 2:, 7] = ref[0][b, two, T // 2:, 7]
    O[b, two, T - 5:], LSE[b, two, T - 5:] = ref[0][b, two, T - 5:], ref[1][b, two, T - 5:]
    assert torch.equal(O, ref[0]) and torch.equal(LSE, ref[1])


@pytest.mark.parametrize("T", [6, 70])
@pytest.mark.parametrize("scale,spread", [(0.3, 1.0), (0.0, 8.0), (0.01, 1.0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales(T, scale, spread, dtype):
    rng = np.random.default_rng(35)
    c = Cache(rng, [200, 90], 2, 64, 16, 13, dtype, spread)
    Q = normal(rng, (2, 4, T, 64), dtype)
    compare_chunk(c, Q, chunk(c, Q, scale=scale), dtype, scale=scale or None)


@pytest.mark.parametrize("Z,T", [(2, 5), (2, 60), (1, 100), (1, 300)])
@pytest.mark.parametrize("A", [64, 192, 256])
def test_scores_that_grow_by_large_steps(Z, T, A):
    """Keys in ascending and in descending order of their scores, by hundreds."""
    n = 300
    for order in (np.arange(n), np.arange(n)[::-1]):
        rng = np.random.default_rng(36)
        c = Cache(rng, [n], 1, A, 16, 19, "bf16")
        Q = torch.zeros(1, Z, T, A, dtype=torch.bfloat16)
        Q[..., 0] = 8.0
        for j in range(n):
            c.Kc[c.table[0, j // 16], 0, j % 16, 0] = float(order[j] * 8 - 1000)
        compare_chunk(c, Q, chunk(c, Q), "bf16")


@pytest.mark.parametrize("dtype,Z,Zkv,A,page,T,lengths,counts,causal,eight", [
    ("bf16", 8, 2, 128, 64, 4, [20000], None, True, False), ("bf16", 8, 2, 128, 64, 4, [20000, 7], None, True, True),
    ("bf16", 8, 2, 128, 64, 100, [9000], None, True, False),                       # few work-groups: divided walks
    ("bf16", 8, 2, 128, 64, 100, [9000, 120], [100, 31], True, True),
    ("bf16", 4, 4, 64, 16, 500, [9000, 500, 5000], [500, 500, 123], True, False),
    ("bf16", 4, 1, 64, 16, 900, [900 + 77 * b for b in range(40)], None, True, False),     # many rows of heads of 64
    ("bf16", 4, 1, 64, 16, 900, [900 + 77 * b for b in range(40)], None, True, True),
    ("bf16", 6, 2, 256, 32, 200, [3000, 222], None, True, False), ("bf16", 6, 2, 256, 32, 200, [3000, 222], [200, 99], False, True),
    ("bf16", 5, 5, 192, 16, 130, [3001, 130], None, False, False), ("bf16", 5, 5, 192, 16, 130, [3001, 130], None, True, True),
    ("bf16", 3, 1, 192, 16, 20, [6001], None, True, True), ("bf16", 9, 9, 64, 16, 40, [7000], None, True, True),
    ("bf16", 16, 4, 128, 16, 1024, [4096, 2100, 1024, 3000], [1024, 500, 1024, 7], True, False),  # heads of 128 by 256 rows
    ("bf16", 32, 8, 128, 16, 520, [4500], None, True, True), ("bf16", 32, 8, 128, 16, 520, [4500, 600, 2000, 1], [520, 520, 0, 1], False, True),
    ("bf16", 8, 8, 128, 16, 500, [2000 + 31 * b for b in range(17)], None, True, False),   # ... one tile and a part of one, divided
    ("bf16", 4, 2, 192, 16, 300, [2000, 400], [300, 299], True, False), ("bf16", 4, 2, 192, 16, 300, [2000, 400], [300, 299], True, True),
    ("bf16", 4, 2, 256, 16, 300, [2000, 400], [300, 299], False, False), ("bf16", 3, 1, 256, 24, 331, [4000, 331, 1], None, True, True),
    ("f32", 6, 3, 64, 24, 300, [2000, 300], None, True, False), ("f32", 20, 1, 128, 16, 5, [6000] * 3, None, True, False),
    ("f32", 4, 2, 256, 16, 100, [3000], [77], True, False), ("bf16", 2, 1, 64, 16, 8, [50 + 3 * b for b in range(700)], None, True, False)])
def test_long_and_many(dtype, Z, Zkv, A, page, T, lengths, counts, causal, eight):
    g = torch.Generator(device="cuda").manual_seed(37)
    B, W = len(lengths), -(-max(lengths) // page)
    Kc, Vc = (torch.randn(B * W, Zkv, page, A, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    table = torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).to(torch.int32)
    Q = torch.randn(B, Z, T, A, generator=g, device="cuda").to(DTYPES[dtype])
    pools, kw = (Kc, Vc), {}
    if eight:                     # powers of two of their own per row, the numbers e4m3's
        e = torch.randint(-3, 3, (2, B * W, Zkv, page), generator=g, device="cuda")
        pools = [x.to(torch.float8_e4m3fn) for x in pools]
        kw = dict(zip(("Ks", "Vs"), (e + 127).to(torch.uint8)))
        two = torch.tensor([2.0 ** k for k in range(-3, 3)], device="cuda")
        Kc, Vc = (x.float() * two[k + 3][..., None] for x, k in zip(pools, e))
    d = rsa.make_cache_desc(pools[0], table, Z)
    ws = torch.full((max(16, rsa.cache_chunk_workspace_bytes(d, T)),), 0xFF, dtype=torch.uint8, device="cuda")
    call = lambda **k: rsa.cache_attend_chunk(d, Q, *pools, table, i32(lengths), None if counts is None else i32(counts), causal, **kw, **k)
    O, LSE = call(ws=ws)
    rO, rLSE, PV = vectorised_chunk(Q, Kc, Vc, table, lengths, counts, causal)
    few = dtype == "f32" or T * (Z // Zkv) <= 16
    # as in attend_bounds, with |q| |k| of these inputs for the sum of products (powers up to 4 in 8 bits)
    rel = 2 * (A + 4) * F32 * A ** 0.5 * (24 if eight else 6) + 2.0 ** -21 + 2 * max(lengths) * F32
    bound = (rel + (0.0 if dtype == "f32" else 2.0 ** -15 if few else 2.0 ** -8)) * PV + STEP[dtype] * rO.abs()
    within(O, f64(rO), f64(bound), "O")
    finite = f64(rLSE)
    within(LSE, finite, rel + 4 * F32 * np.abs(np.where(np.isfinite(finite), finite, 0.0)), "LSE")
    again = call()
    assert torch.equal(again[0], O) and torch.equal(again[1], LSE)            # sums in a fixed order


@pytest.mark.parametrize("dtype,T", [("bf16", 6), ("bf16", 70), ("f32", 30)])
def test_rows_of_no_token_are_left_as_they_are(dtype, T):
    """... in results that are given, and those of rows that see nothing in new ones."""
    rng = np.random.default_rng(38)
    lengths, counts = [100, 30, 5], [T, 2, 0]
    c = Cache(rng, lengths, 2, 64, 16, 8, dtype)
    Q = normal(rng, (3, 4, T, 64), dtype)
    O, LSE = torch.full(Q.shape, 3.0, dtype=Q.dtype, device="cuda"), torch.full((3, 4, T), 5.0, device="cuda")
    got = chunk(c, Q, counts, O=O, LSE=LSE)
    assert got[0].data_ptr() == O.data_ptr() and got[1].data_ptr() == LSE.data_ptr()
    Q[1, :, 2:], Q[2] = float("nan"), float("inf")              # what lies in rows of no token does not count
    new = chunk(c, Q, counts)
    half = chunk(c, Q, counts, O=torch.full_like(O, 3.0))
    assert torch.equal(half[0], O) and torch.equal(half[1], new[1])
    for b, n in enumerate(counts):
        assert torch.equal(O[b, :, :n], new[0][b, :, :n]) and torch.equal(LSE[b, :, :n], new[1][b, :, :n])
        assert (O[b, :, n:] == 3).all() and (LSE[b, :, n:] == 5).all() and torch.isfinite(LSE[b, :, :n]).all()
        assert (new[0][b, :, n:] == 0).all() and torch.isneginf(new[1][b, :, n:]).all()


@pytest.mark.parametrize("dtype,T,kind", [("bf16", 6, Cache), ("bf16", 70, Cache), ("bf16", 70, Cache8), ("f32", 30, Cache)])
def test_strided_queries_and_results(dtype, T, kind):
    """Queries as a slice of one projection output, results with their heads side by side."""
    rng = np.random.default_rng(39)
    B, Z, Zkv, A = 2, 6, 2, 64
    c = kind(rng, [100, T], Zkv, A, 16, 8, dtype)
    x = normal(rng, (B, T, Z + 2 * Zkv, A), dtype).cuda().permute(0, 2, 1, 3)
    Q, O = x[:, :Z], torch.zeros(B, T, Z, A, dtype=DTYPES[dtype], device="cuda").permute(0, 2, 1, 3)
    Kc, Vc, table, n = c.gpu()
    ref = rsa.cache_attend_chunk(rsa.make_cache_desc(Kc, table, Z), Q.contiguous(), Kc, Vc, table, n, **scales_of(c))
    d = rsa.make_cache_desc(Kc, table, Z, Q=Q, O=O)
    got = rsa.cache_attend_chunk(d, Q, Kc, Vc, table, n, O=O, **scales_of(c))
    assert torch.equal(O, ref[0]) and torch.equal(got[1], ref[1]) and (O != 0).any()


@pytest.mark.parametrize("T", [5, 60])
def test_a_prompt_over_ranks_shares_of_the_cache(T):
    """Two ranks hold the slots in front of the tokens, a third the tokens' own: joined, they are the whole."""
    rng = np.random.default_rng(40)
    Z, Zkv, A, page = 4, 2, 64, 16
    c = Cache(rng, [128 + T], Zkv, A, page, -(-(128 + T) // page), "f32")
    Q = normal(rng, (1, Z, T, A), "f32").cuda()
    Kc, Vc, table, _ = c.gpu()
    call = lambda t, n, causal: rsa.cache_attend_chunk(rsa.make_cache_desc(Kc, t, Z), Q, Kc, Vc, t, i32([n]), causal=causal)
    whole = call(table, 128 + T, True)
    parts = [call(table[:, :5].contiguous(), 80, False), call(table[:, 5:8].contiguous(), 48, False), call(table[:, 8:].contiguous(), T, True)]
    rows = rsa.make_cache_desc(Kc, table, Z * T)
    O, LSE = rsa.cache_join(rows, *(torch.stack([p[i].reshape(1, Z * T, 1, *p[i].shape[3:]) for p in parts]) for i in range(2)))
    ref = oracle.attend_chunk(f64(Q), f64(c.Kc), f64(c.Vc), c.table, [128 + T])
    for got, w, r in ((O, whole[0], ref[0]), (LSE, whole[1], ref[1])):
        # fp32 sums of some hundred terms and a join: 2^-24 times as many, of values below 4
        assert np.abs(f64(got).reshape(r.shape) - r).max() < 4 * 300 * F32 and np.abs(f64(w) - r).max() < 4 * 300 * F32


@pytest.mark.parametrize("eight", [False, True])
def test_a_pool_beyond_32_bits(eight):
    """Pages whose rows lie more than 2^32 bytes into the pool."""
    A, page, Zkv, T = 256, 64, 8, 50
    pages = (1 << 32) // (A * page * Zkv * (1 if eight else 2)) + 3
    g = torch.Generator(device="cuda").manual_seed(41)
    dt = torch.float8_e4m3fn if eight else torch.bfloat16
    Kc, Vc = (torch.zeros(pages, Zkv, page, A, dtype=torch.uint8 if eight else dt, device="cuda").view(dt) for _ in range(2))
    for x in (Kc, Vc):
        x[-2:] = torch.randn(2, Zkv, page, A, generator=g, device="cuda").to(dt)
    Q = torch.randn(1, Zkv, T, A, generator=g, device="cuda").bfloat16()
    kw = {k: torch.full((pages, Zkv, page), 127, dtype=torch.uint8, device="cuda") for k in ("Ks", "Vs")} if eight else {}
    small = {k: v[-2:].contiguous() for k, v in kw.items()}
    for t in (T, 3):
        q = Q[:, :, :t].contiguous()
        table = i32([[pages - 1, pages - 2]])
        O, LSE = rsa.cache_attend_chunk(rsa.make_cache_desc(Kc, table, Zkv), q, Kc, Vc, table, i32([100]), **kw)
        k, v = (x.view(torch.uint8)[-2:].clone().view(dt) if eight else x[-2:].contiguous() for x in (Kc, Vc))
        table = i32([[1, 0]])
        O2, LSE2 = rsa.cache_attend_chunk(rsa.make_cache_desc(k, table, Zkv), q, k, v, table, i32([100]), **small)
        assert torch.equal(O, O2) and torch.equal(LSE, LSE2) and (O != 0).any()


@pytest.mark.parametrize("kind", [Cache, Cache8])
@pytest.mark.parametrize("T", [4, 40])
def test_captured_and_replayed_with_other_lengths(kind, T):
    rng = np.random.default_rng(42)
    c = kind(rng, [900, 700], 2, 64, 16, 64, "bf16")
    Kc, Vc, table, n = c.gpu()
    Q = normal(rng, (2, 4, T, 64), "bf16").cuda()
    d = rsa.make_cache_desc(Kc, table, 4)
    counts = i32([T, T])
    O, LSE = torch.zeros_like(Q), torch.zeros(2, 4, T, device="cuda")
    ws = torch.zeros(max(16, rsa.cache_chunk_workspace_bytes(d, T)), dtype=torch.uint8, device="cuda")
    s = scales_of(c)
    rsa.cache_attend_chunk(d, Q, Kc, Vc, table, n, counts, O=O, LSE=LSE, ws=ws, **s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rsa.cache_attend_chunk(d, Q, Kc, Vc, table, n, counts, O=O, LSE=LSE, ws=ws, **s)
    for lengths, have in (([900, 700], [T, T]), ([30, 0], [T, 1]), ([900, T], [2, T]), ([1, 512], [0, T])):
        n.copy_(i32(lengths))
        counts.copy_(i32(have))
        O.fill_(7.0)
        LSE.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = rsa.cache_attend_chunk(d, Q, Kc, Vc, table, n, counts, O=torch.full_like(O, 7.0), LSE=torch.full_like(LSE, 7.0), **s)
        assert torch.equal(O, eager[0]) and torch.equal(LSE, eager[1])


@pytest.mark.parametrize("T", [4, 64])
def test_two_streams(T):
    """Calls on streams of their own, each with its workspace, beside each other."""
    rng = np.random.default_rng(43)
    c = Cache(rng, [1500], 2, 128, 16, 100, "bf16")
    Kc, Vc, table, n = c.gpu()
    Q = [normal(rng, (1, 4, T, 128), "bf16").cuda() for _ in range(2)]
    d = rsa.make_cache_desc(Kc, table, 4)
    ref = [rsa.cache_attend_chunk(d, q, Kc, Vc, table, n) for q in Q]
    streams = [torch.cuda.Stream() for _ in Q]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(rsa.cache_attend_chunk(d, Q[i], Kc, Vc, table, n))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, ref[i][0]) and torch.equal(l, ref[i][1]) for o, l in got[i])


@pytest.mark.parametrize("eight", [False, True])
def test_a_prompt_in_chunks_and_then_token_by_token(eight):
    """A prompt appended and attended to in pieces of uneven lengths, then single tokens, as a program answers: every row is the
    attention to what the cache holds (read back) of its sequence."""
    rng = np.random.default_rng(44)
    B, Z, Zkv, A, page, width = 2, 4, 2, 64, 16, 8
    f = frequencies(A).cuda()
    table = torch.randperm(B * width, generator=torch.Generator().manual_seed(3)).reshape(B, width).int().cuda()
    dt = torch.float8_e4m3fn if eight else torch.bfloat16
    Kc, Vc = (torch.full((B * width, Zkv, page, A), 255 if eight else float("nan"), dtype=torch.uint8 if eight else dt, device="cuda").view(dt) for _ in range(2))
    s = {k: torch.full((B * width, Zkv, page), 255, dtype=torch.uint8, device="cuda") for k in ("Ks", "Vs")} if eight else {}
    d = rsa.make_cache_desc(Kc, table, Z)
    lengths = i32([0, 0])
    rows = []
    for counts in ([40, 7], [1, 33], [0, 40], [9, 2], [1, 1], [1, 1]):
        T = max(counts)
        q, k, v = (normal(rng, (B, z, T, A), "bf16").cuda() for z in (Z, Zkv, Zkv))
        n = i32(counts)
        lengths += n
        q = rsa.cache_append(d, k, v, Kc, Vc, table, lengths, n, None, f, Q=q, **s)
        if T == 1:
            O, LSE = rsa.cache_attend(d, q, Kc, Vc, table, lengths, **s)
        else:
            O, LSE = rsa.cache_attend_chunk(d, q, Kc, Vc, table, lengths, n, **s)
        rows.append((q, O, LSE, counts, lengths.tolist()))
    K, V = (f64(x) for x in rsa.cache_read(d, 64, Kc, Vc, table, lengths, lengths, **s))
    wide = [np.concatenate([x, np.zeros((B, Zkv, 64, A))], 2) for x in (K, V)]          # dense: pages of 128 tokens
    if max(lengths.tolist()) > 64:
        wide = [f64(x) for x in rsa.cache_read(d, 128, Kc, Vc, table, lengths, lengths, **s)]
    one = np.arange(B)[:, None]
    for q, O, LSE, counts, n in rows:
        class Dense:
            Kc, Vc, table, lengths = torch.from_numpy(wide[0]), torch.from_numpy(wide[1]), one, n
        ref = compare_chunk if q.shape[2] > 1 else None
        if ref:
            compare_chunk(Dense, q.cpu(), (O, LSE), "bf16", counts)
        else:
            compare_chunk(Dense, q.cpu(), (O, LSE), "bf16", [1] * B)


@pytest.mark.parametrize("seed", range(18))
def test_uneven_sequences(seed):
    """Random lengths and counts, empty sequences and tokens in front of slot 0 among them: the order in which work-groups take them, walks
    that are divided and such that are not; more sequences than are put in order."""
    r = np.random.default_rng(100 + seed)
    B = [1, 2, 3, 5, 8, 13, 31, 32, 33, 70, 4, 6, 7, 1, 2, 64, 65, 130][seed]
    Zkv, group, A = int(r.integers(1, 4)), int(r.choice([1, 2, 3, 8])), int(r.choice([64, 64, 128]))
    T, most, page = int(r.integers(33, 400)), int(r.choice([200, 1500, 6000])), int(r.choice([5, 16, 64]))
    causal, eight = bool(r.random() < 0.75), bool(r.random() < 0.5)
    Z = Zkv * group
    lengths = [int(most ** x) if r.random() > 0.15 else int(r.integers(-5, 5)) for x in r.random(B)]
    lengths[0] = most
    counts = [int(r.integers(-2, T + 3)) if r.random() < 0.6 else T for _ in range(B)]
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = -(-most // page)
    K, V = (torch.randn(B * W, Zkv, page, A, generator=g, device="cuda").bfloat16() for _ in range(2))
    pools, kw = (K, V), {}
    if eight:
        pools = [x.to(torch.float8_e4m3fn) for x in pools]
        K, V = (x.float() for x in pools)
        kw = {k: torch.full((B * W, Zkv, page), 127, dtype=torch.uint8, device="cuda") for k in ("Ks", "Vs")}
    table = torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).int()
    Q = torch.randn(B, Z, T, A, generator=g, device="cuda").bfloat16()
    d = rsa.make_cache_desc(pools[0], table, Z)
    ws = torch.full((max(16, rsa.cache_chunk_workspace_bytes(d, T)),), 0xFF, dtype=torch.uint8, device="cuda")
    O, LSE = rsa.cache_attend_chunk(d, Q, *pools, table, i32(lengths), i32(counts), causal, ws=ws, **kw)
    mine = rsa.cache_attend_chunk(d, Q, *pools, table, i32(lengths), i32(counts), causal, torch.full_like(Q, 9.0), torch.full_like(LSE, 9.0), **kw)
    there = torch.arange(T, device="cuda")[None] < i32(counts)[:, None]
    assert torch.equal(mine[0], torch.where(there[:, None, :, None], O, 9.0)) and torch.equal(mine[1], torch.where(there[:, None], LSE, 9.0))
    have = [max(0, min(c, T)) for c in counts]
    rO, rLSE, PV = vectorised_chunk(Q, K, V, table, lengths, have, causal)
    rel = 2 * (A + 4) * F32 * A ** 0.5 * 6 + 2.0 ** -21 + 2 * most * F32
    within(O, f64(rO), f64((rel + 2.0 ** -8) * PV + STEP["bf16"] * rO.abs()), "O")
    ref = f64(rLSE)
    within(LSE, ref, rel + 4 * F32 * np.abs(np.where(np.isfinite(ref), ref, 0.0)), "LSE")
