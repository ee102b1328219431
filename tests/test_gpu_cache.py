"""The paged cache against the fp64 oracle: appending to it, attention of one token per sequence, the join of shares."""
import numpy as np
import pytest
import torch

from cache_helpers import DTYPES, F32, STEP, Cache, attend_bounds, f64, frequencies, normal, rotated_bound, within
from oracle import cache as oracle
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- append ----
APPEND = [  # dtype, Z, Zkv, A, page, T, R, adjacent, lengths, counts
    ("bf16", 4, 2, 64, 16, 1, 64, False, [1, 17, 16, 100], None),
    ("bf16", 8, 1, 128, 24, 1, 128, True, [5], None),                       # one sequence
    ("bf16", 6, 6, 64, 5, 9, 32, False, [9, 30, 14], [9, 4, 0]),            # pages that end inside a call, a sequence without tokens
    ("bf16", 2, 2, 128, 1, 7, 20, False, [7, 9], [7, 3]),                   # pages of one token
    ("bf16", 3, 1, 192, 64, 5, 192, True, [5, 70], [12, 5]),                # counts above T
    ("bf16", 4, 4, 64, 16, 3, 0, False, [3, 20], [3, 2]),                   # no rotation
    ("bf16", 5, 5, 256, 16, 2, 62, True, [2, 18], [2, -3]),
    ("bf16", 40, 8, 128, 16, 33, 128, False, [40, 33], [33, 21]),
    ("f32", 4, 2, 64, 16, 1, 64, False, [1, 17, 16, 100], None),
    ("f32", 3, 3, 192, 7, 6, 192, True, [6, 20], [6, 5]),
    ("f32", 2, 1, 256, 16, 5, 250, False, [9, 5], [5, 5]),
    ("f32", 9, 3, 128, 32, 4, 40, True, [70, 4, 33], [1, 4, 2]),
    # more sequences than lanes, many of them without tokens, tiles that end inside a sequence
    ("bf16", 2, 1, 64, 16, 21, 64, False, [21 + 7 * b % 50 for b in range(150)], [(13 * b) % 29 - 4 for b in range(150)]),
    ("f32", 1, 1, 64, 4, 6, 64, True, [6 + b % 9 for b in range(70)], [6 if b in (0, 69) else 0 for b in range(70)]),
    ("bf16", 2, 2, 128, 16, 9, 24, True, [9, 9, 9], [0, 0, 0]),             # no tokens at all
]


def append_case(case, seed=0, width=8):
    dtype, Z, Zkv, A, page, T, R, adjacent, lengths, counts = case
    rng = np.random.default_rng(seed)
    B = len(lengths)
    c = Cache(rng, lengths, Zkv, A, page, max(width, -(-max(lengths) // page)), dtype, junk=7.0)
    Q = normal(rng, (B, Z, T, A), dtype)
    K, V = normal(rng, (B, Zkv, T, A), dtype), normal(rng, (B, Zkv, T, A), dtype)
    return c, Q, K, V, frequencies(R) if R else None


@pytest.mark.parametrize("case", APPEND)
@pytest.mark.parametrize("first", [None, 70000, 2 ** 31 - 100])          # (fp32 holds the last one's turns to a few hundred)
def test_append(case, first):
    dtype, Z, Zkv, A, page, T, R, adjacent, lengths, counts = case
    c, Q, K, V, f = append_case(case)
    B = len(lengths)
    base = None if first is None else [min(first + 3 * b, 2 ** 31 - 1) for b in range(B)]      # (int32)
    Kc, Vc, table, n = c.gpu()
    d = rsa.make_cache_desc(Kc, table, Z)
    Qr = torch.full_like(Q, 5.0).cuda()
    got = rsa.cache_append(d, K.cuda(), V.cuda(), Kc, Vc, table, n, None if counts is None else i32(counts),
                           None if base is None else i32(base), None if f is None else f.cuda(), adjacent, Q.cuda(), Qr)
    assert got.data_ptr() == Qr.data_ptr()
    freq = None if f is None else f.numpy()
    cnt = None if counts is None else [max(0, x) for x in counts]
    rQ, rK, rV = oracle.append(f64(K), f64(V), f64(c.Kc), f64(c.Vc), c.table, lengths, cnt, base, freq, adjacent, f64(Q), np.full(Q.shape, 5.0))
    # the same by which every element is allowed its own bound: inputs in the places of their results
    xQ, xK, _ = oracle.append(f64(K), f64(V), f64(c.Kc), f64(c.Vc), c.table, lengths, cnt, base, None, adjacent, f64(Q), np.full(Q.shape, 5.0))
    for name, y, ref, x in (("Qr", got, rQ, xQ), ("Kc", Kc, rK, xK)):
        bound = rotated_bound(x, ref, R, adjacent, dtype) if R else np.zeros(x.shape)
        within(y, ref, np.where(ref == x, 0.0, bound), name)              # what was not written is as it was, to the bit
    assert np.array_equal(f64(Vc), rV)


def test_append_leaves_what_is_not_held():
    """Slots below 0, behind the table and on pages that are not held: nothing is written, queries are rotated all the same."""
    Zkv, A, page, T = 2, 64, 4, 3
    rng = np.random.default_rng(1)
    K, V, Q = (normal(rng, (4, Zkv, T, A), "bf16").cuda() for _ in range(3))
    Kc = torch.full((3, Zkv, page, A), 7.0, dtype=torch.bfloat16, device="cuda")
    Vc = Kc.clone()
    table = i32([[0, -1], [3, 1], [2, 2 ** 31 - 1], [-2 ** 31, 1]])
    n = i32([6, 10, 1, 3])                   # slots 3, 4, 5; 7, 8, 9; -2, -1, 0; 0, 1, 2
    d = rsa.make_cache_desc(Kc, table, Zkv)
    f = frequencies(A)
    Qr = rsa.cache_append(d, K, V, Kc, Vc, table, n, inv_freq=f.cuda(), Q=Q)
    want = torch.full((3, Zkv, page, A), 7.0, dtype=torch.bfloat16, device="cuda")
    want[0, :, 3], want[1, :, 3], want[2, :, 0] = V[0, :, 0], V[1, :, 0], V[2, :, 2]
    assert torch.equal(Vc, want)
    assert torch.equal((Kc == 7.0).all(-1), (want == 7.0).all(-1))
    for b, slot in enumerate((3, 7, -2, 0)):
        ref = oracle.rotate(f64(Q[b]), np.arange(slot, slot + T), f.numpy())
        within(Qr[b], ref, rotated_bound(f64(Q[b]), ref, A, False, "bf16"), f"Qr[{b}]")


def test_append_by_shares_of_strided_tensors():
    """Q, K, V as slices of one projection output; Qr over Q; new tensors' rows behind a count are zero."""
    B, Z, Zkv, T, A = 3, 4, 2, 5, 64
    x = torch.randn(B, T, Z + 2 * Zkv, A, generator=torch.Generator().manual_seed(2)).bfloat16().cuda().permute(0, 2, 1, 3)
    Q, K, V = x[:, :Z], x[:, Z:Z + Zkv], x[:, Z + Zkv:]
    lengths, counts, f = i32([5, 9, 4]), i32([5, 2, 0]), frequencies(A).cuda()
    table = i32(np.arange(9).reshape(3, 3))
    pools = [torch.zeros(9, Zkv, 4, A, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    dense = rsa.make_cache_desc(pools[0], table, Z)
    ref = rsa.cache_append(dense, K.contiguous(), V.contiguous(), pools[0], pools[1], table, lengths, counts, None, f, Q=Q.contiguous())
    assert (ref[1, :, 2:] == 0).all() and (ref[2] == 0).all() and (ref[0] != 0).any()
    d = rsa.make_cache_desc(pools[0], table, Z, Q=Q, K=K)
    before = x.clone()
    with pytest.raises(ValueError, match="has to be given"):
        rsa.cache_append(d, K, V, pools[2], pools[3], table, lengths, counts, None, f, Q=Q)
    rsa.cache_append(d, K, V, pools[2], pools[3], table, lengths, counts, None, f, Q=Q, Qr=Q)
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    there = torch.arange(T, device="cuda")[None] < counts[:, None]
    assert torch.equal(Q, torch.where(there[:, None, :, None], ref, before[:, :Z])) and torch.equal(x[:, Z:], before[:, Z:])
    assert rsa.cache_append(d, K, V, pools[2], pools[3], table, lengths, counts, None, f) is None


@pytest.mark.parametrize("B,T", [(4096, 9), (4097, 9), (5000, 1)])
def test_append_for_many_sequences(B, T):
    """... against calls for a few of them at a time."""
    Zkv, A, page, W, pages = 1, 64, 8, 3, 3 * 5000
    g = torch.Generator(device="cuda").manual_seed(23)
    rng = np.random.default_rng(24)
    Q, K, V = (torch.randn(B, Zkv, T, A, generator=g, device="cuda").bfloat16() for _ in range(3))
    table = torch.randperm(pages, generator=g, device="cuda")[:B * W].reshape(B, W).int()
    counts = np.where(rng.random(B) < 0.7, 0, rng.integers(-1, T + 2, B))
    n, c = i32(rng.integers(0, W * page + 3, B)), i32(counts)
    f = frequencies(A).cuda()

    def run(step):
        Kc = torch.zeros(pages, Zkv, page, A, dtype=torch.bfloat16, device="cuda")
        Vc, Qr = torch.zeros_like(Kc), torch.full_like(Q, 3.0)
        for b in range(0, B, step):
            s = slice(b, b + step)
            rsa.cache_append(rsa.make_cache_desc(Kc, table[s], Zkv), K[s], V[s], Kc, Vc, table[s], n[s], c[s], None, f, Q=Q[s], Qr=Qr[s])
        return Kc, Vc, Qr
    for x, y in zip(run(B), run(61)):
        assert torch.equal(x, y) and (x != 0).any()


def test_append_in_a_pool_beyond_32_bits():
    """A page whose elements lie more than 2^31 elements (4 GB) into the pool."""
    A, page, Zkv = 256, 64, 8
    pages = (1 << 31) // (A * page * Zkv) + 3
    Kc = torch.zeros(pages, Zkv, page, A, dtype=torch.bfloat16, device="cuda")
    Vc = torch.zeros_like(Kc)
    K, V, Q = (torch.randn(1, Zkv, 100, A, device="cuda").bfloat16() for _ in range(3))
    table = i32([[pages - 1, pages - 2]])
    d = rsa.make_cache_desc(Kc, table, Zkv)
    rsa.cache_append(d, K, V, Kc, Vc, table, i32([100]))
    assert torch.equal(Kc[-1], K[0, :, :64]) and torch.equal(Vc[-2, :, :36], V[0, :, 64:]) and (Kc[:-2] == 0).all()
    O, LSE = rsa.cache_attend(d, Q[:, :, :1].contiguous(), Kc, Vc, table, i32([100]))
    small = rsa.make_cache_desc(Kc[-2:], table, Zkv)
    O2, LSE2 = rsa.cache_attend(small, Q[:, :, :1].contiguous(), Kc[-2:].contiguous(), Vc[-2:].contiguous(), i32([[1, 0]]), i32([100]))
    assert torch.equal(O, O2) and torch.equal(LSE, LSE2) and (O != 0).any()


# ---------------------------------------------------------------- attend ----
ATTEND = [  # dtype, Z, Zkv, A, page, lengths
    ("bf16", 4, 4, 64, 16, [1, 2, 15, 16, 17, 0]),
    ("bf16", 8, 2, 128, 16, [300, 0, 31, 32, 33, 700]),
    ("bf16", 2, 2, 64, 1, [70, 129]),                          # pages of one token
    ("bf16", 6, 2, 64, 24, [127, 128, 129, 25]),
    ("bf16", 16, 1, 128, 100, [511, 99]),                      # sixteen queries a key head
    ("bf16", 17, 1, 64, 16, [200, 64]),                        # one more
    ("bf16", 33, 1, 128, 64, [400]),
    ("bf16", 48, 2, 64, 16, [90, 0, 260]),
    ("bf16", 3, 3, 192, 32, [65, 190]),
    ("bf16", 10, 2, 256, 16, [33, 600]),
    ("bf16", 20, 1, 256, 7, [333]),
    ("bf16", 12, 12, 64, 256, [1025]),
    ("f32", 4, 4, 64, 16, [1, 2, 15, 16, 17, 0]),
    ("f32", 8, 2, 128, 24, [300, 31, 500]),
    ("f32", 17, 1, 192, 16, [65, 190]),
    ("f32", 36, 2, 256, 5, [33, 260]),
    ("f32", 1, 1, 64, 1, [77]),
]


def attend(c, Q, **kw):
    Kc, Vc, table, n = c.gpu()
    d = rsa.make_cache_desc(Kc, table, Q.shape[1], scale=kw.pop("scale", 0.0))
    return rsa.cache_attend(d, Q.cuda(), Kc, Vc, table, n, **kw)


def compare(c, Q, got, dtype, scale=None):
    Kc, Vc = f64(c.Kc), f64(c.Vc)
    O, LSE = oracle.attend(f64(Q), Kc, Vc, c.table, c.lengths, scale)
    bO, bL = attend_bounds(f64(Q), Kc, Vc, c.table, c.lengths, O, LSE, dtype, scale)
    within(got[0], O, bO, "O")
    within(got[1], LSE, bL, "LSE")


@pytest.mark.parametrize("case", ATTEND)
def test_attend(case):
    """The pools hold NaN wherever no sequence has a token."""
    dtype, Z, Zkv, A, page, lengths = case
    rng = np.random.default_rng(3)
    c = Cache(rng, lengths, Zkv, A, page, -(-max(lengths) // page) + 1, dtype)
    Q = normal(rng, (len(lengths), Z, 1, A), dtype)
    compare(c, Q, attend(c, Q), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,spread", [(0.3, 1.0), (0.0, 8.0), (0.01, 1.0)])
def test_attend_scales(dtype, scale, spread):
    rng = np.random.default_rng(4)
    c = Cache(rng, [400, 37], 2, 64, 16, 30, dtype, spread)
    Q = normal(rng, (2, 6, 1, 64), dtype)
    compare(c, Q, attend(c, Q, scale=scale), dtype, scale or None)


def test_attend_rows_that_grow_by_large_steps():
    """Keys in ascending and in descending order of their scores, by hundreds: the running maximum moves with every key, or never."""
    n, A = 600, 64
    for order in (np.arange(n), np.arange(n)[::-1]):
        rng = np.random.default_rng(5)
        c = Cache(rng, [n], 1, A, 16, 38, "f32")
        Q = torch.zeros(1, 1, 1, A)
        Q[..., 0] = 8.0
        for j in range(n):
            c.Kc[c.table[0, j // 16], 0, j % 16, 0] = float(order[j] * 7 - 2000)
        compare(c, Q, attend(c, Q), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Z", [2, 20])
def test_pages_that_are_not_held(dtype, Z):
    """Entries outside the pool, at the front, in the middle, behind, everywhere; a length beyond the table; below zero."""
    rng = np.random.default_rng(6)
    c = Cache(rng, [200, 200, 200, 200, 200, 200], 2, 64, 16, 13, dtype)
    pages = c.Kc.shape[0]
    c.table[0, :9] = -1
    c.table[1, 3:11:2] = pages
    c.table[2, 12] = 2 ** 31 - 1
    c.table[3, :] = -2 ** 31
    c.lengths[4] = 2 ** 31 - 1
    c.table[4, 12] = -5                      # (its last page holds NaN behind slot 200)
    c.lengths[5] = -7
    Q = normal(rng, (6, Z, 1, 64), dtype)
    got = attend(c, Q)
    compare(c, Q, got, dtype)
    for b in (3, 5):
        assert (got[0][b] == 0).all() and torch.isneginf(got[1][b]).all()


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_what_lies_behind_a_sequence_does_not_reach_it(junk):
    rng = np.random.default_rng(7)
    lengths = [1, 5, 33, 130]
    clean = Cache(rng, lengths, 2, 128, 16, 9, "bf16", junk=0.0)
    Q = normal(rng, (4, 8, 1, 128), "bf16")
    ref = attend(clean, Q)
    rng = np.random.default_rng(7)
    dirty = Cache(rng, lengths, 2, 128, 16, 9, "bf16", junk=junk)
    got = attend(dirty, Q)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_infinite_and_nan_keys_reach_their_own_heads_alone():
    rng = np.random.default_rng(8)
    c = Cache(rng, [50, 50, 50], 2, 64, 16, 4, "bf16")
    Q = normal(rng, (3, 4, 1, 64), "bf16")
    ref = attend(c, Q)
    c.Vc[c.table[0, 1], 0, 3, 5] = float("inf")
    c.Kc[c.table[1, 2], 1, 0, 0] = float("nan")
    O, LSE = attend(c, Q)
    assert torch.isinf(O[0, :2, 0, 5]).all() and O[1, 2:].isnan().all() and LSE[1, 2:].isnan().all()
    O[0, :2, 0, 5], O[1, 2:], LSE[1, 2:] = ref[0][0, :2, 0, 5], ref[0][1, 2:], ref[1][1, 2:]
    assert torch.equal(O, ref[0]) and torch.equal(LSE, ref[1])


def test_sequences_that_share_pages():
    """The same pages in several rows of the table, as sequences with one beginning have them: rows of one length agree."""
    rng = np.random.default_rng(9)
    c = Cache(rng, [100], 2, 64, 16, 7, "bf16")
    c.table, c.lengths = np.repeat(c.table, 4, 0), np.array([100, 60, 100, 1], np.int32)
    Q = normal(rng, (1, 4, 1, 64), "bf16").repeat(4, 1, 1, 1)
    got = attend(c, Q)
    compare(c, Q, got, "bf16")
    one = Cache(np.random.default_rng(9), [100], 2, 64, 16, 7, "bf16")
    alone = attend(one, Q[:1])
    for b in (0, 2):
        assert (got[0][b] - alone[0][0]).abs().max() <= 2 * 2.0 ** -8 * alone[0].abs().max()


def vectorised(Q, Kc, Vc, table, lengths):
    """The definition in fp64 on the GPU, for caches that are too long for loops."""
    B, Z, _, A = Q.shape
    Zkv, page = Kc.shape[1:3]
    O, LSE, PV = [], [], []
    for b in range(B):
        n = int(lengths[b])
        rows = table[b, :-(-n // page)].long()
        k, v = (x[rows].transpose(0, 1).reshape(Zkv, -1, A)[:, :n].double() for x in (Kc, Vc))
        S = Q[b].double().reshape(Zkv, Z // Zkv, A) @ k.transpose(1, 2) / A ** 0.5
        P = S.softmax(-1)
        O.append((P @ v).reshape(Z, 1, A))
        LSE.append(S.logsumexp(-1).reshape(Z, 1))
        PV.append((P @ v.abs()).reshape(Z, 1, A))
    return (torch.stack(x) for x in (O, LSE, PV))


@pytest.mark.parametrize("dtype,Z,Zkv,A,page,lengths", [
    ("bf16", 8, 2, 128, 64, [20000]), ("bf16", 4, 4, 64, 16, [9000, 1, 5000, 33]), ("bf16", 32, 1, 64, 16, [40000, 700]),
    ("bf16", 20, 4, 128, 48, [3000 + 61 * b for b in range(40)]), ("bf16", 6, 2, 256, 32, [7000, 8192, 12]),
    ("bf16", 5, 5, 192, 16, [6001, 2]), ("f32", 6, 3, 64, 24, [9000, 300, 4096]), ("f32", 20, 1, 128, 16, [6000] * 3),
    ("bf16", 2, 1, 64, 16, [50 + 3 * b for b in range(700)]), ("bf16", 16, 1, 256, 16, [9000]), ("f32", 3, 1, 192, 16, [5001]),
    ("f32", 20, 1, 64, 16, [9999]), ("bf16", 3, 3, 192, 16, [300 + 5 * b for b in range(200)])])
def test_long_and_many_sequences(dtype, Z, Zkv, A, page, lengths):
    g = torch.Generator(device="cuda").manual_seed(11)
    B, W = len(lengths), -(-max(lengths) // page)
    Kc, Vc = (torch.randn(B * W, Zkv, page, A, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    table = torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).to(torch.int32)
    Q = torch.randn(B, Z, 1, A, generator=g, device="cuda").to(DTYPES[dtype])
    d = rsa.make_cache_desc(Kc, table, Z)
    ws = torch.full((max(16, rsa.cache_workspace_bytes(d)),), 0xFF, dtype=torch.uint8, device="cuda")
    O, LSE = rsa.cache_attend(d, Q, Kc, Vc, table, i32(lengths), ws=ws)
    rO, rLSE, PV = vectorised(Q, Kc, Vc, table, lengths)
    # as in attend_bounds, with |q| |k| of these inputs for the sum of products (below A times 5 times 5, and s = A^-1/2)
    rel = 2 * (A + 4) * F32 * A ** 0.5 * 6 + 2.0 ** -21 + 2 * max(lengths) * F32
    bound = (rel + (2.0 ** -15 if dtype == "bf16" else 0.0)) * PV + STEP[dtype] * rO.abs()
    within(O, f64(rO), f64(bound), "O")
    within(LSE, f64(rLSE), rel + 4 * F32 * np.abs(f64(rLSE)), "LSE")
    again = rsa.cache_attend(d, Q, Kc, Vc, table, i32(lengths))
    assert torch.equal(again[0], O) and torch.equal(again[1], LSE)            # sums in a fixed order


@pytest.mark.parametrize("dtype,Z,Zkv,A,B", [
    ("bf16", 16, 1, 256, 1), ("bf16", 32, 1, 128, 2), ("f32", 2, 1, 64, 3),                # segments of many parts
    ("bf16", 8, 2, 128, 5), ("f32", 6, 3, 64, 4), ("bf16", 40, 40, 64, 30)])               # of fewer; more segments than shares
def test_a_workspace_in_which_a_longer_call_has_left_its_notes(dtype, Z, Zkv, A, B):
    """Every call of one workspace against the same call of its own: what lies there does not count."""
    page, W = 16, 2048 if B < 30 else 256
    g = torch.Generator(device="cuda").manual_seed(23)
    pages = W if B < 30 else 1000
    Kc, Vc = (torch.randn(pages, Zkv, page, A, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    table = torch.randint(pages, (B, W), generator=g, device="cuda", dtype=torch.int32)
    Q = torch.randn(B, Z, 1, A, generator=g, device="cuda").to(DTYPES[dtype])
    d = rsa.make_cache_desc(Kc, table, Z)
    n = rsa.cache_workspace_bytes(d)
    assert n > 0
    used = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    most = W * page
    for lengths in ([most] * B, [most - 1 - 37 * b for b in range(B)], [0] * (B - 1) + [1], [0] * B, [most // 2] + [0] * (B - 1),
                    [most if b % 2 else 0 for b in range(B)], [1] * B, [0] * B, [700 - 23 * b for b in range(B)]):
        O, LSE = rsa.cache_attend(d, Q, Kc, Vc, table, i32(lengths), ws=used)
        fresh = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        own = rsa.cache_attend(d, Q, Kc, Vc, table, i32(lengths), ws=fresh)
        assert torch.equal(O, own[0]) and torch.equal(LSE, own[1])
        none = i32(lengths) <= 0
        assert (O[none] == 0).all() and torch.isneginf(LSE[none]).all()
        assert torch.isfinite(LSE[~none]).all()
        # (a row of the first slot alone is its value)
        if lengths == [1] * B:
            v = Vc[table[:, 0].long(), :, 0].repeat_interleave(Z // Zkv, 1).unsqueeze(2)
            within(O, f64(v), f64(v.abs().double() * (STEP[dtype] + 2.0 ** -15 + 2.0 ** -20)), "O")


@pytest.mark.parametrize("B", [65, 4096, 4097])
def test_more_sequences_than_lanes(B):
    """Most of them empty or short, on pages that they share, in tables with room for long ones."""
    Z, Zkv, A, page, W, pages = 2, 1, 64, 16, 64, 300
    g = torch.Generator(device="cuda").manual_seed(18)
    Kc, Vc = (torch.randn(pages, Zkv, page, A, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(pages, (B, W), generator=g, device="cuda", dtype=torch.int32)
    rng = np.random.default_rng(19)
    lengths = np.where(rng.random(B) < 0.4, 0, rng.integers(1, 1025, B) ** 2 // 1024)
    lengths[0], lengths[-1] = 0, 1024
    Q = torch.randn(B, Z, 1, A, generator=g, device="cuda").bfloat16()
    O, LSE = rsa.cache_attend(rsa.make_cache_desc(Kc, table, Z), Q, Kc, Vc, table, i32(lengths))
    none = torch.from_numpy(lengths == 0).cuda()
    assert (O[none] == 0).all() and torch.isneginf(LSE[none]).all()
    some = np.flatnonzero(lengths)
    rO, rLSE, PV = vectorised(Q[~none], Kc, Vc, table[~none], lengths[some])
    # as in test_long_and_many_sequences
    rel = 2 * (A + 4) * F32 * A ** 0.5 * 6 + 2.0 ** -21 + 2 * 1024 * F32
    bound = (rel + 2.0 ** -15) * PV + STEP["bf16"] * rO.abs()
    within(O[~none], f64(rO), f64(bound), "O")
    within(LSE[~none], f64(rLSE), rel + 4 * F32 * np.abs(f64(rLSE)), "LSE")


def test_strided_queries_and_results():
    """Q and O as a projection's rows of one token per sequence, (1, Z, B, A) seen as (B, Z, 1, A)."""
    rng = np.random.default_rng(12)
    c = Cache(rng, [40, 3, 90], 2, 64, 16, 6, "bf16")
    Kc, Vc, table, n = c.gpu()
    x = torch.randn(1, 4, 64, 64, device="cuda").bfloat16()
    Q = x.permute(2, 1, 0, 3)[:3]
    y = torch.full_like(x, 9.0)
    O = y.permute(2, 1, 0, 3)[:3]
    ref = rsa.cache_attend(rsa.make_cache_desc(Kc, table, 4), Q.contiguous(), Kc, Vc, table, n)
    got = rsa.cache_attend(rsa.make_cache_desc(Kc, table, 4, Q=Q, O=O), Q, Kc, Vc, table, n, O=O)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1]) and (y[:, :, 3:] == 9).all()
    need = rsa.cache_workspace_bytes(rsa.make_cache_desc(Kc, table, 4))
    if need:
        with pytest.raises(rsa.RSAError, match="workspace"):
            rsa.cache_attend(rsa.make_cache_desc(Kc, table, 4), Q.contiguous(), Kc, Vc, table, n,
                             ws=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------ join ----
@pytest.mark.parametrize("dtype,N,B,Z,A", [("bf16", 1, 1, 1, 64), ("bf16", 8, 3, 5, 128), ("bf16", 3, 70, 2, 192), ("f32", 5, 2, 3, 256),
                                           ("f32", 2, 9, 7, 64), ("bf16", 17, 2, 2, 64)])
def test_join(dtype, N, B, Z, A):
    rng = np.random.default_rng(13)
    Op, LSEp = normal(rng, (N, B, Z, 1, A), dtype), normal(rng, (N, B, Z, 1), "f32", 20.0)
    gone = torch.from_numpy(rng.random((N, B, Z, 1)) < 0.3)
    gone[:, 0, 0] = True                                # a row that no share sees
    LSEp[gone] = -float("inf")
    Op[gone] = float("nan")
    pool = torch.zeros(1, 1, 16, A, dtype=DTYPES[dtype], device="cuda")
    d = rsa.make_cache_desc(pool, torch.zeros(B, 1, dtype=torch.int32, device="cuda"), Z)
    O, LSE = rsa.cache_join(d, Op.cuda(), LSEp.cuda())
    rO, rLSE = oracle.join(f64(Op), f64(LSEp))
    # the exponent's argument errs by 2^-24 of its size (below 200), exp by 2^-22, N terms' sum by N 2^-24
    rel = 200 * F32 + 2.0 ** -21 + 2 * N * F32
    size = np.abs(np.where(f64(gone.float())[..., None] > 0, 0.0, f64(Op))).max(0)
    within(O, rO, rel * size + STEP[dtype] * np.abs(rO), "O")
    within(LSE, rLSE, rel + 4 * F32 * np.abs(np.where(np.isinf(rLSE), 0, rLSE)), "LSE")
    assert (O[0, 0] == 0).all() and torch.isneginf(LSE[0, 0]).all()


def test_join_into_a_projections_rows():
    g = torch.Generator(device="cuda").manual_seed(22)
    Op = torch.randn(3, 5, 4, 1, 64, generator=g, device="cuda").bfloat16()
    LSEp = torch.randn(3, 5, 4, 1, generator=g, device="cuda")
    pool, table = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16, device="cuda"), i32(np.zeros((5, 1)))
    ref = rsa.cache_join(rsa.make_cache_desc(pool, table, 4), Op, LSEp)
    y = torch.full((1, 4, 64, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    O = y.permute(2, 1, 0, 3)[:5]
    got = rsa.cache_join(rsa.make_cache_desc(pool, table, 4, O=O), Op, LSEp, O)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1]) and (y[:, :, 5:] == 9).all()


def test_join_of_ranks_that_share_a_cache():
    """Each of four ranks holds a run of the tokens (first: its beginning) and answers for it; joined, that is the whole cache's answer."""
    B, Z, Zkv, A, page, L, N = 2, 8, 2, 64, 16, 300, 4
    rng = np.random.default_rng(14)
    K, V = normal(rng, (B, Zkv, L, A), "f32").cuda(), normal(rng, (B, Zkv, L, A), "f32").cuda()
    Q = normal(rng, (B, Z, 1, A), "f32").cuda()
    f = frequencies(A).cuda()

    def cache(b, e):
        pools = [torch.full((40, Zkv, page, A), float("nan"), device="cuda") for _ in range(2)]
        table = i32(np.random.default_rng(b).permutation(40).reshape(2, 20))
        d = rsa.make_cache_desc(pools[0], table, Z)
        n = i32([e - b] * B)
        rsa.cache_append(d, K[:, :, b:e].contiguous(), V[:, :, b:e].contiguous(), *pools, table, n, first=i32([b] * B), inv_freq=f)
        return d, pools, table, n
    d, pools, table, n = cache(0, L)
    O, LSE = rsa.cache_attend(d, Q, *pools, table, n)
    Op, LSEp = torch.empty(N, B, Z, 1, A, device="cuda"), torch.empty(N, B, Z, 1, device="cuda")
    for r in range(N):
        d, pools, table, n = cache(r * 75, (r + 1) * 75)
        rsa.cache_attend(d, Q, *pools, table, n, Op[r], LSEp[r])
    Oj, LSEj = rsa.cache_join(d, Op, LSEp)
    # two fp32 results of one value: twice the bound of attend_bounds with scores below 6 and sums of 300
    tol = 2 * (2 * 68 * F32 * 8 * 6 + 2.0 ** -21 + 2 * L * F32)
    assert (Oj - O).abs().max() <= 4 * tol and (LSEj - LSE).abs().max() <= tol


# ------------------------------------------------- together, as they are used ----
def test_a_prompt_and_decoding_steps():
    """Prompt by the ring's causal forward, its keys into the cache, then tokens one by one through projections, append and
    attention: every step's answer is that of attention to the whole sequence in fp64."""
    H = Z = 4
    A, page, B, P, steps = 64, 16, 3, 64, 4
    H = Z * A
    g = torch.Generator(device="cuda").manual_seed(15)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()
    Wqkv, Wo = rnd(H, 3 * H, std=H ** -0.5), rnd(H, H, std=H ** -0.5)
    X = rnd(B, P + steps, H)
    f = frequencies(A).cuda()
    Kc, Vc = torch.full((3 * 5 + 1, Z, page, A), float("nan"), dtype=torch.bfloat16, device="cuda"), None
    Vc = Kc.clone()
    table = torch.randperm(16, generator=g, device="cuda")[:15].reshape(3, 5).to(torch.int32)
    # the prompt
    ring = rsa.make_desc(torch.empty(B, Z, P, A, dtype=torch.bfloat16, device="cuda"), 1, causal=True)
    Q, K, V = rsa.qkv_proj(ring, X[:, :P].contiguous(), Wqkv)
    cd = rsa.make_cache_desc(Kc, table, Z)
    n = i32([P] * B)
    rsa.cache_append(cd, K, V, Kc, Vc, table, n, inv_freq=f)
    Qr, Kr = rsa.rotate(ring, f, Q, K)
    assert torch.equal(Kc[table[:, :4].long()].permute(0, 2, 1, 3, 4).reshape(B, Z, P, A), Kr)
    O, _ = rsa.forward(ring, Qr, Kr, V)
    # rows of the padded step: B tokens, one of each sequence, and 61 that are not used
    row = rsa.make_desc(torch.empty(1, Z, 64, A, dtype=torch.bfloat16, device="cuda"), 1)
    pad = torch.zeros(1, 64, H, dtype=torch.bfloat16, device="cuda")
    keys, values = [K], [V]
    for t in range(steps):
        pad[0, :B] = X[:, P + t]
        q, k, v = (y.permute(2, 1, 0, 3)[:B] for y in rsa.qkv_proj(row, pad, Wqkv))
        o = torch.zeros(1, Z, 64, A, dtype=torch.bfloat16, device="cuda")
        ov = o.permute(2, 1, 0, 3)[:B]
        cd = rsa.make_cache_desc(Kc, table, Z, Q=q, K=k, O=ov)
        n += 1
        keys.append(k.clone())
        values.append(v.clone())
        q0 = q.clone()
        rsa.cache_append(cd, k, v, Kc, Vc, table, n, inv_freq=f, Q=q, Qr=q)
        rsa.cache_attend(cd, q, Kc, Vc, table, n, O=ov)
        Y = rsa.out_proj(row, o, Wo)
        kk, vv = torch.cat(keys, 2), torch.cat(values, 2)
        L = P + t + 1
        ref_k = oracle.rotate(f64(kk), np.arange(L), f.cpu().numpy())
        ref_q = oracle.rotate(f64(q0), [L - 1], f.cpu().numpy())
        S = (ref_q * ref_k).sum(-1) / 8
        p = np.exp(S - S.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        want = (p[..., None] * f64(vv)).sum(2)
        # stored q and k: scores off by 2^-8 / sqrt 3 of sum |q k| / 8 terms each, independent (below 0.04); then as attend_bounds
        err = np.abs(f64(ov)[:, :, 0] - want)
        dS = 2.0 ** -8 / 3 ** 0.5 * np.sqrt(2 * ((ref_q * ref_k) ** 2).sum(-1)) / 8
        spread = np.sqrt((p ** 2 * dS ** 2)[..., None] * f64(vv) ** 2).sum(2)
        assert (err <= 6 * spread + 2.0 ** -8 * np.abs(want) + 1e-4).all(), t
        wy = torch.from_numpy(f64(ov)[:, :, 0].reshape(B, H)).cuda() @ Wo.double()
        assert (Y[0, :B].double() - wy).abs().max() <= 2.0 ** -8 * wy.abs().max() + H * F32 * 16


def step(d, x, out):
    rsa.cache_append(d, x["K"], x["V"], x["Kc"], x["Vc"], x["table"], x["n"], inv_freq=x["f"], Q=x["Q"], Qr=out["Qr"])
    rsa.cache_attend(d, out["Qr"], x["Kc"], x["Vc"], x["table"], x["n"], out["O"], out["LSE"], x["ws"])


def test_a_captured_step_replays_with_new_lengths_and_tables():
    """Two graphs on one workspace, replayed in turn with tokens, lengths and tables that change, against eager calls."""
    B, Z, Zkv, A, page, W = 3, 8, 2, 128, 16, 200
    g = torch.Generator(device="cuda").manual_seed(16)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()

    def state():
        x = dict(Kc=rnd(B * W, Zkv, page, A), Vc=rnd(B * W, Zkv, page, A), Q=rnd(B, Z, 1, A), K=rnd(B, Zkv, 1, A), V=rnd(B, Zkv, 1, A),
                 table=torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).to(torch.int32), n=i32([1, 1, 1]), f=frequencies(A).cuda())
        return x, dict(Qr=torch.empty_like(x["Q"]), O=torch.empty_like(x["Q"]), LSE=torch.empty(B, Z, 1, device="cuda"))
    states = [state(), state()]
    d = rsa.make_cache_desc(states[0][0]["Kc"], states[0][0]["table"], Z)
    ws = torch.empty(max(16, rsa.cache_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    graphs = []
    for x, out in states:
        x["ws"] = ws
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(d, x, out)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(d, x, out)
        graphs.append(graph)
    for lengths in ([1, 2, 3], [3200, 5, 0], [40, 3199, 2000], [16, 17, 3200]):
        for (x, out), graph in zip(states, graphs):
            x["n"].copy_(i32(lengths))
            x["table"].copy_(x["table"].flip(0))
            for k in "QKV":
                x[k].normal_(generator=g)
            ref = {k: torch.empty_like(v) for k, v in out.items()}
            mine = dict(x, Kc=x["Kc"].clone(), Vc=x["Vc"].clone(), ws=None)
            step(d, mine, ref)
            for v in out.values():
                v.fill_(float("nan"))
            ws.fill_(0xFF)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for k in ref:
                assert torch.equal(out[k], ref[k]), (lengths, k)
            assert torch.equal(mine["Kc"], x["Kc"]) and torch.equal(mine["Vc"], x["Vc"])


def test_two_streams_at_once():
    rng = np.random.default_rng(17)
    c = [Cache(rng, [900, 20, 450], 2, 64, 16, 60, "bf16", junk=0.0) for _ in range(2)]
    Q = [normal(rng, (3, 8, 1, 64), "bf16").cuda() for _ in range(2)]
    gpu = [x.gpu() for x in c]
    d = [rsa.make_cache_desc(x[0], x[2], 8) for x in gpu]
    ref = [rsa.cache_attend(d[i], Q[i], *gpu[i]) for i in range(2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(rsa.cache_attend(d[i], Q[i], *gpu[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for O, LSE in got[i]:
            assert torch.equal(O, ref[i][0]) and torch.equal(LSE, ref[i][1])
