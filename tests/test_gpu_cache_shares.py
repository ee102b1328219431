"""Attention of a new token where its work is divided into shares: every slot counts once, wherever shares begin and end."""
import numpy as np
import pytest
import torch

from cache_helpers import DTYPES, F32, STEP, f64, within
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def apart(lengths, B, where, A=128, page=16):
    """Sequences of these lengths at the given places among B, the others empty; queries of zeros, so that every slot has the same weight."""
    n = np.zeros(B, np.int32)
    n[where] = lengths
    width = -(-max(lengths) // page)
    g = torch.Generator(device="cuda").manual_seed(50)
    pages = 512
    Kc, Vc = (torch.randn(pages, 1, page, A, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(pages, (B, width), generator=g, device="cuda", dtype=torch.int32)
    return torch.zeros(B, 4, 1, A, dtype=torch.bfloat16, device="cuda"), Kc, Vc, table, i32(n)


def time_of(call):
    """The shortest of ten in us, captured."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            call()
    best = float("inf")
    for _ in range(10):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        best = min(best, begin.elapsed_time(end) * 100)
    return best


def test_empty_sequences_between_long_ones():
    """A share that begins in one sequence and ends in one 2000 rows of the table behind it, in at most three times the time that it takes
    with the empty rows at the table's end (about as long; each empty row looked at alone takes five times as long)."""
    lengths, where = [35001, 7777, 16500], [0, 2000, 4095]
    Q, Kc, Vc, table, n = apart(lengths, 4096, where)
    all_of = rsa.make_cache_desc(Kc, table, 4)
    O, LSE = rsa.cache_attend(all_of, Q, Kc, Vc, table, n)
    for b, count in zip(where, lengths):
        v = Vc[table[b].long(), 0].reshape(-1, Vc.shape[-1])[:count].double()
        # equal weights: exp(0) is 1, their sum exact, log and its product off by 2^-22 and a rounding; sums of values by 2^-24 of their size a step of
        # the walk, 64 at most, the waves and the shares
        within(LSE[b], np.full((4, 1), np.log(count)), 2.0 ** -22 + 2 * F32 * np.log(count), "LSE")
        mean = f64(v.mean(0)).reshape(1, 1, -1)
        within(O[b], np.broadcast_to(mean, O[b].shape), STEP["bf16"] * np.abs(mean) + 400 * F32 * f64(v.abs().mean(0)), "O")
    none = torch.ones(4096, dtype=torch.bool)
    none[where] = False
    assert (O[none.cuda()] == 0).all() and torch.isneginf(LSE[none.cuda()]).all()
    ws = torch.empty(rsa.cache_workspace_bytes(all_of), dtype=torch.uint8, device="cuda")
    together = apart(lengths, 4096, [0, 1, 2])[-1]
    long, short = (time_of(lambda: rsa.cache_attend(all_of, Q, Kc, Vc, table, m, O, LSE, ws)) for m in (n, together))
    assert long <= 3 * short, (long, short)


def random_tables(rng, lengths, Zkv, A, page, dtype, junk=float("nan"), spare=1):
    """Pools of `junk` and a table whose sequences have pages of their own; keys and values are to be filled in."""
    B, W = len(lengths), -(-max(lengths) // page) + spare
    table = rng.permutation(B * W).reshape(B, W)
    Kc = torch.full((B * W, Zkv, page, A), junk, dtype=DTYPES[dtype], device="cuda")
    return Kc, Kc.clone(), torch.from_numpy(table).cuda()


def without_pages(table, kind, lengths, page, pages):
    """The table with pages that are not held, and their number of slots for each sequence."""
    t = table.clone()
    for b, n in enumerate(lengths):
        held = -(-n // page)
        if kind == "front":
            t[b, :held // 2] = -1
        elif kind == "all but the last":
            t[b, :max(0, held - 1)] = pages
        elif kind == "middle":
            t[b, held // 4:held - held // 4] = 2 ** 31 - 1
        elif kind == "one in three":
            t[b, b % 3::3] = -2 ** 31
        elif kind == "everywhere":
            t[b] = -1 if b % 2 == 0 else t[b]
    return t.to(torch.int32)


def slots_of(table, lengths, b, page, pages):
    """The slots of sequence b that are seen, with their pages and places."""
    s = torch.arange(min(max(0, int(lengths[b])), table.shape[1] * page), device="cuda")
    p = table[b, s // page].long()
    seen = (p >= 0) & (p < pages)
    return s[seen], p[seen], (s % page)[seen]


# dtype, Z, Zkv, A, page, lengths: segments of many parts, joined by 32 columns; notes by segment; notes by share; queries of two and of several tiles
FORMS = [
    ("bf16", 32, 1, 128, 16, [40000]), ("f32", 3, 1, 64, 64, [33001]), ("bf16", 16, 1, 256, 16, [9000]),
    ("bf16", 8, 2, 128, 64, [20000, 0, 129, 6000]), ("bf16", 4, 4, 64, 16, [9000, 1, 5000, 33]), ("f32", 6, 3, 192, 24, [4100, 300, 2000]),
    ("bf16", 68, 1, 64, 24, [3000, 1100]), ("f32", 20, 1, 128, 16, [6000] * 3),
    ("bf16", 40, 40, 64, 16, [800 + 13 * b for b in range(25)]), ("f32", 24, 24, 64, 8, [400 + 17 * b for b in range(33)]),
    ("bf16", 1, 1, 64, 16, [50 + 3 * b for b in range(900)])]
HOLES = [None, "front", "all but the last", "middle", "one in three", "everywhere"]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("holes", HOLES)
def test_every_slot_counts_once(form, holes):
    """Queries of zeros: every probability is 1, their sum the number of slots, exactly, so LSE = log n, where a slot that is lost or counted twice shows
    as 1 / n; the logarithm's last bit, ln 2 and the product are 4 x 2^-24 of it.  Every column's values are zeros but for one slot's 1, at the
    edges of tiles, units and pages and anywhere: 1 / n, rounded twice in fp32 and once when it is stored."""
    dtype, Z, Zkv, A, page, lengths = form
    rng = np.random.default_rng(51)
    Kc, Vc, table = random_tables(rng, lengths, Zkv, A, page, dtype)
    pages = Kc.shape[0]
    cut = without_pages(table, holes, lengths, page, pages)
    want = torch.zeros(len(lengths), Zkv, A, dtype=torch.float64, device="cuda")
    count = torch.zeros(len(lengths), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths):
        s, p, at = slots_of(cut, lengths, b, page, pages)
        Kc[p, :, at] = 3.0
        Vc[p, :, at] = 0.0
        count[b] = len(s)
        if len(s) == 0:
            continue
        edges = np.concatenate([np.arange(0, n, e) for e in (16, 64, 128, page)])
        near = torch.from_numpy(np.unique(np.concatenate([[0, n - 1], edges, edges - 1])).clip(0, n - 1)).cuda()
        near = torch.searchsorted(s, near).clamp(max=len(s) - 1).cpu().numpy()
        for h in range(Zkv):
            some = np.concatenate([rng.choice(near, A // 2), rng.integers(0, len(s), A - A // 2 - 2), [0, len(s) - 1]])
            some = torch.from_numpy(some).cuda()
            Vc[p[some], h, at[some], torch.arange(A, device="cuda")] = 1.0
        want[b] = 1.0 / len(s)
    Q = torch.zeros(len(lengths), Z, 1, A, dtype=DTYPES[dtype], device="cuda")
    d = rsa.make_cache_desc(Kc, cut, Z)
    need = rsa.cache_workspace_bytes(d)
    assert need > 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    O, LSE = rsa.cache_attend(d, Q, Kc, Vc, cut, i32(lengths), ws=ws)
    ref = f64(torch.log(count))[:, None, None]
    within(LSE, np.broadcast_to(ref, LSE.shape), 2.0 ** -22 + 4 * F32 * np.where(np.isinf(ref), 0, ref), "LSE")
    mean = f64(want.repeat_interleave(Z // Zkv, 1))[:, :, None]
    within(O, mean, (STEP[dtype] + 2 * F32) * mean, "O")


def reference(Q, Kc, Vc, table, lengths):
    """The definition in fp64, and by which it is allowed: sum of P |v|, the largest sum of |q k|, the number of slots."""
    B, Z, _, A = Q.shape
    pages, Zkv, page, _ = Kc.shape
    O, PV = (torch.zeros(B, Z, 1, A, dtype=torch.float64, device="cuda") for _ in range(2))
    LSE = torch.full((B, Z, 1), -float("inf"), dtype=torch.float64, device="cuda")
    S = torch.zeros_like(LSE)
    for b in range(B):
        _, p, at = slots_of(table, lengths, b, page, pages)
        if len(p) == 0:
            continue
        k, v = (x[p, :, at].transpose(0, 1).double() for x in (Kc, Vc))
        q = Q[b].double().reshape(Zkv, Z // Zkv, A)
        kt = k.transpose(1, 2).contiguous()
        s = q @ kt / A ** 0.5
        P = s.softmax(-1)
        O[b], PV[b] = (P @ v).reshape(Z, 1, A), (P @ v.abs()).reshape(Z, 1, A)
        LSE[b] = s.logsumexp(-1).reshape(Z, 1)
        S[b] = (q.abs() @ kt.abs() / A ** 0.5).amax(-1).reshape(Z, 1)
    return O, LSE, PV, S


def compare(Q, Kc, Vc, table, lengths, got, dtype):
    """A score is a sum of A products, off by (A + 4) 2^-24 of the sum of their sizes at most; exp and the exponents of the joins add 2^-20.  A
    wave takes a tile of 32 slots (16) of every unit of a share; its sum is 8 adds a tile, a matrix product's 96 at most.  Shares have
    at most units / 256 + 1 units or, of some hundred segments and more, 16 here; the waves and a segment's parts are joined one after the other."""
    O, LSE, PV, S = (f64(x) for x in reference(Q, Kc, Vc, table, lengths))
    A, tiles = Q.shape[-1], 16
    parts = np.minimum(256, -(-np.maximum(1, np.asarray(lengths)) // 64) + 1)[:, None, None]
    score = 2 * (A + 4) * F32 * S + 2.0 ** -20
    depth = (96 * tiles + 4 + parts) * F32
    within(got[0], O, (score + depth)[..., None] * PV + STEP[dtype] * np.abs(O), "O")
    within(got[1], LSE, score + (8 * tiles + 6 + parts) * F32 + 4 * F32 * np.abs(np.where(np.isinf(LSE), 0, LSE)), "LSE")


def filled(form, holes=None, seed=52, spare=1):
    dtype, Z, Zkv, A, page, lengths = form
    rng = np.random.default_rng(seed)
    Kc, Vc, table = random_tables(rng, lengths, Zkv, A, page, dtype, spare=spare)
    cut = without_pages(table, holes, lengths, page, Kc.shape[0])
    g = torch.Generator(device="cuda").manual_seed(seed)
    for b in range(len(lengths)):
        _, p, at = slots_of(cut, lengths, b, page, Kc.shape[0])
        for x in (Kc, Vc):
            x[p, :, at] = torch.randn(len(p), Zkv, A, generator=g, device="cuda").to(x.dtype)
    Q = torch.randn(len(lengths), Z, 1, A, generator=g, device="cuda").to(Kc.dtype)
    return Q, Kc, Vc, cut


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("holes", HOLES)
def test_shares_against_the_definition(form, holes):
    """Parts that see nothing (their maximum is -inf) among parts that do, in the front, the middle and everywhere."""
    dtype, Z, *_, lengths = form
    Q, Kc, Vc, table = filled(form, holes)
    d = rsa.make_cache_desc(Kc, table, Z)
    assert rsa.cache_workspace_bytes(d) > 0
    compare(Q, Kc, Vc, table, lengths, rsa.cache_attend(d, Q, Kc, Vc, table, i32(lengths)), dtype)


def test_lengths_beyond_the_table_and_below_zero():
    for form in (FORMS[3], FORMS[4]):
        dtype, Z, Zkv, A, page, lengths = form
        Q, Kc, Vc, table = filled(form, spare=0)
        n = list(lengths)
        n[0], n[1], n[2] = 2 ** 31 - 1, -2 ** 31, -5
        full = table.shape[1] * page
        Kc[table[0].long()] = 0.5
        Vc[table[0].long()] = 0.25
        got = rsa.cache_attend(rsa.make_cache_desc(Kc, table, Z), Q, Kc, Vc, table, i32(n))
        n = [full, 0, 0] + n[3:]
        compare(Q, Kc, Vc, table, n, got, dtype)
        assert (got[0][1:3] == 0).all() and torch.isneginf(got[1][1:3]).all()


@pytest.mark.parametrize("form", [FORMS[0], FORMS[3], FORMS[6], FORMS[8], FORMS[9]])
def test_strided_queries_and_results_of_shares(form):
    """Q and O as rows of a projection, (1, Z, rows, A) seen as (B, Z, 1, A): whole segments and divided ones, joined in either way."""
    dtype, Z, Zkv, A, page, lengths = form
    Q, Kc, Vc, table = filled(form)
    B = len(lengths)
    ref = rsa.cache_attend(rsa.make_cache_desc(Kc, table, Z), Q, Kc, Vc, table, i32(lengths))
    x, y = torch.full((1, Z, 64, A), 7.0, dtype=Q.dtype, device="cuda"), torch.full((1, Z, 64, A), 9.0, dtype=Q.dtype, device="cuda")
    q, o = (t.permute(2, 1, 0, 3)[:B] for t in (x, y))
    q.copy_(Q)
    d = rsa.make_cache_desc(Kc, table, Z, Q=q, O=o)
    got = rsa.cache_attend(d, q, Kc, Vc, table, i32(lengths), O=o)
    assert got[0].data_ptr() == y.data_ptr() and torch.equal(o, ref[0]) and torch.equal(got[1], ref[1]) and (y[:, :, B:] == 9).all()


@pytest.mark.parametrize("form", [FORMS[0], FORMS[3], FORMS[8]])
def test_infinite_and_nan_keys_in_shares(form):
    dtype, Z, Zkv, A, page, lengths = form
    Q, Kc, Vc, table = filled(form)
    d, n = rsa.make_cache_desc(Kc, table, Z), i32(lengths)
    ref = rsa.cache_attend(d, Q, Kc, Vc, table, n)
    slot, group, last = lengths[0] * 2 // 3, Z // Zkv, len(lengths) - 1
    Vc[table[0, slot // page].long(), 0, slot % page, 5] = float("inf")
    Kc[table[last, 1].long(), Zkv - 1, 3] = float("nan")
    O, LSE = rsa.cache_attend(d, Q, Kc, Vc, table, n)
    nan = O[last, Z - group:].isnan().all() and LSE[last, Z - group:].isnan().all()
    assert nan and (last == 0 or torch.isposinf(O[0, :group, 0, 5]).all())
    for x, r in ((O, ref[0]), (LSE, ref[1])):
        x[last, Z - group:] = r[last, Z - group:]
    O[0, :group, 0, 5] = ref[0][0, :group, 0, 5]
    assert torch.equal(O, ref[0]) and torch.equal(LSE, ref[1])


def test_a_workspace_that_is_too_small_is_refused():
    Q, Kc, Vc, table = filled(FORMS[4])
    d = rsa.make_cache_desc(Kc, table, 4)
    need = rsa.cache_workspace_bytes(d)
    assert need > 0
    for ws in (torch.empty(need - 1, dtype=torch.uint8, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")):
        with pytest.raises(rsa.RSAError, match="workspace"):
            rsa.cache_attend(d, Q, Kc, Vc, table, i32(FORMS[4][-1]), ws=ws)
