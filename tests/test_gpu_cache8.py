"""The cache in 8 bits against the fp64 oracle: what is stored, to the bit; reading it back; attention of one new token to it."""
import numpy as np
import pytest
import torch

from cache8_helpers import Cache8, i32
from cache_helpers import DTYPES, Cache, attend_bounds, f64, frequencies, normal, rotated_bound, within
from oracle import cache as oracle
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu

APPEND = [  # Z, Zkv, A, page, T, R, adjacent, lengths, counts
    (4, 2, 64, 16, 1, 64, False, [1, 17, 16, 100], None),
    (8, 1, 128, 24, 1, 128, True, [5], None),
    (6, 6, 64, 5, 9, 32, False, [9, 30, 14], [9, 4, 0]),
    (2, 2, 128, 1, 7, 20, False, [7, 9], [7, 3]),                     # partners over two lanes' pieces
    (3, 1, 192, 64, 5, 192, True, [5, 70], [12, 5]),
    (4, 2, 192, 64, 5, 192, False, [5, 70], [12, 5]),
    (4, 4, 64, 16, 3, 0, False, [3, 20], [3, 2]),
    (5, 5, 256, 16, 2, 62, True, [2, 18], [2, -3]),
    (5, 5, 256, 16, 2, 250, False, [2, 18], [2, 1]),
    (40, 8, 128, 16, 33, 128, False, [40, 33], [33, 21]),
    (2, 1, 64, 16, 21, 64, False, [21 + 7 * b % 50 for b in range(150)], [(13 * b) % 29 - 4 for b in range(150)]),
    (2, 2, 128, 16, 9, 2, True, [9, 9, 9], [0, 0, 0]),
]


def pools(table, Zkv, page, A, pages):
    Kc = torch.full((pages, Zkv, page, A), 0x11, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    Ks = torch.full((pages, Zkv, page), 99, dtype=torch.uint8, device="cuda")
    return Kc, Kc.view(torch.uint8).clone().view(torch.float8_e4m3fn), Ks, Ks.clone()


@pytest.mark.parametrize("case", APPEND)
@pytest.mark.parametrize("first", [None, 70000, 2 ** 31 - 100])
@pytest.mark.parametrize("spread", [1.0, 300.0])
def test_append(case, first, spread):
    """Bytes and exponents are those of the definition; what was not written is as it was."""
    Z, Zkv, A, page, T, R, adjacent, lengths, counts = case
    rng = np.random.default_rng(51)
    B = len(lengths)
    width = max(8, -(-max(lengths) // page))
    pages = B * width + 2
    table = rng.permutation(pages)[:B * width].reshape(B, width)
    table[:, -1] = -1
    Q, K, V = (normal(rng, (B, z, T, A), "bf16") for z in (Z, Zkv, Zkv))
    K, V = (x * torch.from_numpy(spread ** rng.uniform(-1, 1, (B, Zkv, T, 1))).bfloat16() for x in (K, V))
    f = frequencies(R) if R else None
    base = None if first is None else [min(first + 3 * b, 2 ** 31 - 1) for b in range(B)]
    Kc, Vc, Ks, Vs = pools(table, Zkv, page, A, pages)
    d = rsa.make_cache_desc(Kc, i32(table), Z)
    Qr = torch.full_like(Q, 5.0).cuda()
    got = rsa.cache_append(d, K.cuda(), V.cuda(), Kc, Vc, i32(table), i32(lengths), None if counts is None else i32(counts),
                           None if base is None else i32(base), None if f is None else f.cuda(), adjacent, Q.cuda(), Qr, Ks, Vs)
    assert got.data_ptr() == Qr.data_ptr()
    cnt = None if counts is None else [max(0, x) for x in counts]
    freq = None if f is None else f.numpy()
    start = [np.full((pages, Zkv, page, A), 0x11)] * 2 + [np.full((pages, Zkv, page), 99)] * 2
    rQ, *want = oracle.append8(f64(K), f64(V), *start, table, lengths, cnt, base, freq, adjacent, f64(Q), np.full(Q.shape, 5.0))
    for name, x, ref in zip(("Kc", "Vc", "Ks", "Vs"), (Kc.view(torch.uint8), Vc.view(torch.uint8), Ks, Vs), want):
        assert np.array_equal(x.cpu().numpy(), ref), name
    xQ = oracle.append(f64(K), f64(V), start[0], start[0], table, lengths, cnt, base, None, adjacent, f64(Q), np.full(Q.shape, 5.0))[0]
    bound = rotated_bound(xQ, rQ, R, adjacent, "bf16") if R else np.zeros(xQ.shape)
    within(got, rQ, np.where(rQ == xQ, 0.0, bound), "Qr")


def test_every_bf16_value_is_stored_as_the_definition_says():
    """All 2^16 numbers, infinite and NaN ones among them, 64 a row, beside a large element and without; 0 and the smallest ones."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    rows = torch.cat([x.reshape(-1, 64), x.reshape(64, -1).T.contiguous().reshape(-1, 64)])
    tall = rows.clone()
    tall[:, 0] = 448.0 * 2.0 ** torch.arange(len(rows)).remainder(9).sub(4).float()
    V = torch.cat([rows, tall, torch.zeros(1, 64, dtype=torch.bfloat16)])[None, None]
    n = V.shape[2]
    page, table = 64, torch.arange(-(-n // 64), dtype=torch.int32, device="cuda")[None]
    Kc, Vc, Ks, Vs = pools(table, 1, page, 64, table.shape[1])
    d = rsa.make_cache_desc(Kc, table, 1)
    rsa.cache_append(d, V.cuda().clone(), V.cuda(), Kc, Vc, table, i32([n]), Ks=Ks, Vs=Vs)
    byte, e = oracle.to_e4m3(f64(V)[0, 0])
    for pool, exps in ((Kc, Ks), (Vc, Vs)):
        got = pool.view(torch.uint8).cpu().numpy().reshape(-1, 64)[:n]
        nan = np.isnan(f64(V)[0, 0]) | np.isinf(f64(V)[0, 0])
        assert np.array_equal(exps.cpu().numpy().reshape(-1)[:n], e)
        assert np.array_equal(got[~nan], byte[~nan]) and ((got[nan] & 127) == 127).all()


def test_turned_pairs_of_large_and_tiny_numbers():
    """Pairs whose turn is larger than any bf16 number, and rows below the least power."""
    A, n = 64, 40
    K = torch.empty(1, 1, n, A, dtype=torch.bfloat16)
    K[:, :, :20], K[:, :, 20:] = 3.3e38, 2.0 ** -70
    table = torch.arange(3, dtype=torch.int32, device="cuda")[None]
    Kc, Vc, Ks, Vs = pools(table, 1, 16, A, 3)
    f = frequencies(A, 3.0)
    rsa.cache_append(rsa.make_cache_desc(Kc, table, 1), K.cuda(), K.cuda().clone(), Kc, Vc, table, i32([n]), inv_freq=f.cuda(), Ks=Ks, Vs=Vs)
    _, kc, vc, ks, vs = oracle.append8(f64(K), f64(K), *[np.full((3, 1, 16, A), 0x11)] * 2, *[np.full((3, 1, 16), 99)] * 2, np.arange(3)[None], [n],
                                       inv_freq=f.numpy())
    assert ks.max() == 247 and ks.min() == 63
    for x, ref in ((Kc.view(torch.uint8), kc), (Vc.view(torch.uint8), vc), (Ks, ks), (Vs, vs)):
        assert np.array_equal(x.cpu().numpy(), ref)


def test_append_in_place_and_strided():
    B, Z, Zkv, T, A = 3, 4, 2, 5, 64
    x = torch.randn(B, T, Z + 2 * Zkv, A, generator=torch.Generator().manual_seed(2)).bfloat16().cuda().permute(0, 2, 1, 3)
    Q, K, V = x[:, :Z], x[:, Z:Z + Zkv], x[:, Z + Zkv:]
    lengths, counts = i32([5, 9, 4]), i32([5, 2, 0])
    table = i32(np.arange(9).reshape(3, 3))
    for R in (64, 20):
        f = frequencies(R).cuda()
        a, b = pools(table, Zkv, 4, A, 9), pools(table, Zkv, 4, A, 9)
        ref = rsa.cache_append(rsa.make_cache_desc(a[0], table, Z), K.contiguous(), V.contiguous(), *a[:2], table, lengths, counts, None, f,
                               Q=Q.contiguous(), Ks=a[2], Vs=a[3])
        assert (ref[1, :, 2:] == 0).all() and (ref[2] == 0).all() and (ref[0] != 0).any()
        y = x.permute(0, 2, 1, 3).clone().permute(0, 2, 1, 3)
        q, k, v = y[:, :Z], y[:, Z:Z + Zkv], y[:, Z + Zkv:]
        d = rsa.make_cache_desc(b[0], table, Z, Q=q, K=k)
        rsa.cache_append(d, k, v, *b[:2], table, lengths, counts, None, f, Q=q, Qr=q, Ks=b[2], Vs=b[3])
        assert all(torch.equal(p.view(torch.uint8), r.view(torch.uint8)) for p, r in zip(a, b))
        there = torch.arange(T, device="cuda")[None] < counts[:, None]
        assert torch.equal(q, torch.where(there[:, None, :, None], ref, Q)) and torch.equal(y[:, Z:], x[:, Z:])
        assert rsa.cache_append(d, k, v, *b[:2], table, lengths, counts, None, f, Ks=b[2], Vs=b[3]) is None


@pytest.mark.parametrize("B,T", [(4096, 9), (4097, 9), (5000, 1)])
def test_append_for_many_sequences(B, T):
    """... against calls for a few of them at a time."""
    Zkv, A, page, W, count = 1, 64, 8, 3, 3 * 5000
    g = torch.Generator(device="cuda").manual_seed(23)
    rng = np.random.default_rng(24)
    Q, K, V = (torch.randn(B, Zkv, T, A, generator=g, device="cuda").bfloat16() for _ in range(3))
    table = torch.randperm(count, generator=g, device="cuda")[:B * W].reshape(B, W).int()
    n, c = i32(rng.integers(0, W * page + 3, B)), i32(np.where(rng.random(B) < 0.7, 0, rng.integers(-1, T + 2, B)))
    f = frequencies(A).cuda()

    def run(step):
        Kc, Vc, Ks, Vs = pools(table, Zkv, page, A, count)
        Qr = torch.full_like(Q, 3.0)
        for b in range(0, B, step):
            s = slice(b, b + step)
            rsa.cache_append(rsa.make_cache_desc(Kc, table[s], Zkv), K[s], V[s], Kc, Vc, table[s], n[s], c[s], None, f, Q=Q[s], Qr=Qr[s], Ks=Ks, Vs=Vs)
        return Kc.view(torch.uint8), Vc.view(torch.uint8), Ks, Vs, Qr
    for x, y in zip(run(B), run(61)):
        assert torch.equal(x, y) and (x != x.flatten()[0]).any()


# ------------------------------------------------------------------ read ----
READ = [  # dtype, Zkv, A, page, T, lengths, counts
    ("bf16", 2, 64, 16, 1, [1, 17, 0], None), ("bf16", 3, 128, 5, 30, [100, 30, 12], [30, 7, 40]), ("bf16", 1, 192, 24, 11, [50, 3], None),
    ("bf16", 5, 256, 1, 9, [9, 30], [0, -4]), ("f32", 2, 64, 16, 20, [33, 20], [20, 3]), ("f32", 3, 192, 7, 6, [6, 20, -3], None),
    ("f32", 1, 128, 16, 70, [100, 65], [70, 70]), ("f32", 2, 256, 16, 13, [40, 13], None),
]


@pytest.mark.parametrize("case", READ)
@pytest.mark.parametrize("eight", [False, True])
def test_read(case, eight):
    dtype, Zkv, A, page, T, lengths, counts = case
    if eight and dtype == "f32":
        return
    rng = np.random.default_rng(52)
    width = -(-max(lengths) // page) + 1
    c = (Cache8 if eight else Cache)(rng, lengths, Zkv, A, page, width, dtype)
    c.table[0, 0] = -1                                         # a page that is no longer held
    Kc, Vc, table, n = c.gpu()
    d = rsa.make_cache_desc(Kc, table, Zkv)
    s = c.scales() if eight else {}
    B = len(lengths)
    K, V = (torch.full((B, Zkv, T, A), 5.0, dtype=DTYPES[dtype], device="cuda") for _ in range(2))
    dev = None if counts is None else i32(counts)
    got = rsa.cache_read(d, T, Kc, Vc, table, n, dev, K, V, **s)
    assert got[0].data_ptr() == K.data_ptr()
    for x, pool in ((K, c.Kc), (V, c.Vc)):
        assert np.array_equal(f64(x), oracle.read(f64(pool), c.table, lengths, T, counts, np.full(K.shape, 5.0)))
    half = rsa.cache_read(d, T, Kc, Vc, table, n, dev, V=torch.full_like(V, 5.0), **s)
    assert np.array_equal(f64(half[0]), oracle.read(f64(c.Kc), c.table, lengths, T, counts)) and torch.equal(half[1], V)
    for x, pool in zip(rsa.cache_read(d, T, Kc, Vc, table, n, dev, **s), (c.Kc, c.Vc)):
        assert np.array_equal(f64(x), oracle.read(f64(pool), c.table, lengths, T, counts))
    # heads side by side
    wide = torch.zeros(B, T, 2 * Zkv, A, dtype=DTYPES[dtype], device="cuda").permute(0, 2, 1, 3)
    k, v = wide[:, :Zkv], wide[:, Zkv:]
    d = rsa.make_cache_desc(Kc, table, Zkv, K=k)
    rsa.cache_read(d, T, Kc, Vc, table, n, dev, k, v, **s)
    assert np.array_equal(f64(wide[:, :Zkv]), oracle.read(f64(c.Kc), c.table, lengths, T, counts))
    assert np.array_equal(f64(wide[:, Zkv:]), oracle.read(f64(c.Vc), c.table, lengths, T, counts))


def test_every_byte_and_exponent_is_read_as_what_it_stands_for():
    Kc = torch.arange(256, dtype=torch.uint8, device="cuda").reshape(1, 1, 1, 256).repeat(254, 1, 1, 1).view(torch.float8_e4m3fn)
    Ks = torch.arange(254, dtype=torch.uint8, device="cuda").reshape(254, 1, 1)
    table = torch.arange(254, dtype=torch.int32, device="cuda")[None]
    K, V = rsa.cache_read(rsa.make_cache_desc(Kc, table, 1), 254, Kc, Kc.view(torch.uint8).clone().view(torch.float8_e4m3fn), table, i32([254]), Ks=Ks, Vs=Ks.clone())
    v = oracle.from_e4m3(np.arange(256))[None] * 2.0 ** (np.arange(254) - 127.0)[:, None]
    want = torch.from_numpy(v).float().bfloat16()
    normal_power = slice(63, 248)                              # what is ever written: exact
    for x in (K, V):
        got = x[0, 0].cpu()
        assert torch.equal(got[normal_power].nan_to_num(7.0), want[normal_power].nan_to_num(7.0))
        assert torch.equal(got.isnan(), want.isnan())


# ---------------------------------------------------------------- attend ----
ATTEND = [  # Z, Zkv, A, page, lengths
    (4, 4, 64, 16, [1, 2, 15, 16, 17, 0]), (8, 2, 128, 16, [300, 0, 31, 32, 33, 700]), (2, 2, 64, 1, [70, 129]), (6, 2, 64, 24, [127, 128, 129, 25]),
    (17, 1, 64, 16, [200, 64]), (33, 1, 128, 64, [400]), (48, 2, 64, 16, [90, 0, 260]), (3, 3, 192, 32, [65, 190]), (10, 2, 256, 16, [33, 600]),
    (20, 1, 256, 7, [333]), (12, 12, 64, 256, [1025]),
]


@pytest.mark.parametrize("case", ATTEND)
@pytest.mark.parametrize("spread", [1.0, 30.0])
def test_attend(case, spread):
    """NaN and exponents of 255 wherever no sequence has a token; rows of keys of powers of their own."""
    Z, Zkv, A, page, lengths = case
    rng = np.random.default_rng(53)
    c = Cache8(rng, lengths, Zkv, A, page, -(-max(lengths) // page) + 1)
    for e in c.exps:
        e[...] = np.where(e == 255, 255, e + np.round(rng.uniform(-1, 1, e.shape) * np.log2(spread)).astype(int))
    Q = normal(rng, (len(lengths), Z, 1, A), "bf16", 1 / spread)
    Kc, Vc, table, n = c.gpu()
    d = rsa.make_cache_desc(Kc, table, Z)
    got = rsa.cache_attend(d, Q.cuda(), Kc, Vc, table, n, **c.scales())
    k, v = f64(c.Kc), f64(c.Vc)
    O, LSE = oracle.attend(f64(Q), k, v, c.table, c.lengths)
    bO, bL = attend_bounds(f64(Q), k, v, c.table, c.lengths, O, LSE, "bf16")
    within(got[0], O, bO, "O")
    within(got[1], LSE, bL, "LSE")


@pytest.mark.parametrize("Z,Zkv,A,page,lengths", [(8, 2, 128, 64, [20000]), (4, 4, 64, 16, [9000, 1, 5000, 33]), (20, 4, 128, 48, [3000 + 61 * b for b in range(40)]),
                                                  (6, 2, 256, 32, [7000, 8192, 12]), (5, 5, 192, 16, [6001, 2]), (16, 1, 256, 16, [9000])])
def test_long_and_many_sequences(Z, Zkv, A, page, lengths):
    """The same kernels' bf16 form on what the pools stand for sums alike: results agree to the last rounding."""
    g = torch.Generator(device="cuda").manual_seed(54)
    B, W = len(lengths), -(-max(lengths) // page)
    Kc, Vc = (torch.randn(B * W, Zkv, page, A, generator=g, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    Ks, Vs = (torch.randint(125, 130, (B * W, Zkv, page), generator=g, device="cuda").to(torch.uint8) for _ in range(2))
    two = torch.tensor([2.0 ** k for k in range(-2, 3)], device="cuda")
    table = torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).to(torch.int32)
    Q = (torch.randn(B, Z, 1, A, generator=g, device="cuda") / 2).bfloat16()
    d = rsa.make_cache_desc(Kc, table, Z)
    ws = torch.full((max(16, rsa.cache_workspace_bytes(d)),), 0xFF, dtype=torch.uint8, device="cuda")
    O, LSE = rsa.cache_attend(d, Q, Kc, Vc, table, i32(lengths), ws=ws, Ks=Ks, Vs=Vs)
    k, v = ((x.float() * two[s.long() - 125][..., None]).bfloat16() for x, s in ((Kc, Ks), (Vc, Vs)))
    rO, rLSE = rsa.cache_attend(d, Q, k, v, table, i32(lengths))
    # both are within a rounding and 2^-15 of sum p |v| (below 10 here) of the exact result
    assert (O.float() - rO.float()).abs().max() <= 2 * (2.0 ** -8 * rO.float().abs().max() + 2.0 ** -15 * 10)
    assert (LSE - rLSE).abs().max() <= 2.0 ** -15 * rLSE.abs().max()
    again = rsa.cache_attend(d, Q, Kc, Vc, table, i32(lengths), Ks=Ks, Vs=Vs)
    assert torch.equal(again[0], O) and torch.equal(again[1], LSE)


@pytest.mark.parametrize("shape", [(8, 2, 128, 100), (4, 4, 64, 8)])
def test_captured_and_replayed_with_other_lengths(shape):
    """A step of an answer: a token stored, attention to it, the row read back."""
    Z, Zkv, A, width = shape
    rng = np.random.default_rng(55)
    B, page = 3, 16
    table = i32(rng.permutation(B * width).reshape(B, width))
    Kc, Vc, Ks, Vs = pools(table, Zkv, page, A, B * width)
    d = rsa.make_cache_desc(Kc, table, Z)
    n = i32([1, 1, 1])
    q, k, v = (normal(rng, (B, z, 1, A), "bf16").cuda() for z in (Z, Zkv, Zkv))
    f = frequencies(A).cuda()
    qr, O, LSE = torch.empty_like(q), torch.empty_like(q), torch.empty(B, Z, 1, device="cuda")
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    ws = torch.zeros(max(16, rsa.cache_workspace_bytes(d)), dtype=torch.uint8, device="cuda")

    def step():
        rsa.cache_append(d, k, v, Kc, Vc, table, n, inv_freq=f, Q=q, Qr=qr, Ks=Ks, Vs=Vs)
        rsa.cache_attend(d, qr, Kc, Vc, table, n, O, LSE, ws, Ks, Vs)
        rsa.cache_read(d, 1, Kc, Vc, table, n, K=rk, V=rv, Ks=Ks, Vs=Vs)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths in ([1, 2, 3], [40, 0, 7], [100, 101, 102], [width * page, 5, width * page + 3]):
        n.copy_(i32(lengths))
        for x in (q, k, v):
            x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (qr, O, LSE, rk, rv)]
        step()
        assert all(torch.equal(x, y) for x, y in zip(got, (qr, O, LSE, rk, rv)))


@pytest.mark.parametrize("eight", [False, True])
def test_appended_slices_and_new_dense_results_by_one_descriptor(eight):
    """Keys and values as slices of one projection output, appended and read back by the same descriptor: results that are given have its
    strides, new ones are dense."""
    rng = np.random.default_rng(51)
    B, Z, Zkv, T, A, page = 2, 4, 2, 33, 64, 16
    x = normal(rng, (B, T, Z + 2 * Zkv, A), "bf16").cuda().permute(0, 2, 1, 3)
    Q, K, V = x[:, :Z], x[:, Z:Z + Zkv], x[:, Z + Zkv:]
    table = torch.arange(6, dtype=torch.int32, device="cuda").reshape(B, 3)
    dt = torch.float8_e4m3fn if eight else torch.bfloat16
    Kc, Vc = (torch.zeros(6, Zkv, page, A, dtype=torch.uint8 if eight else dt, device="cuda").view(dt) for _ in range(2))
    s = {k: torch.zeros(6, Zkv, page, dtype=torch.uint8, device="cuda") for k in ("Ks", "Vs")} if eight else {}
    n = torch.tensor([T, 20], dtype=torch.int32, device="cuda")
    d = rsa.make_cache_desc(Kc, table, Z, Q=Q, K=K)
    rsa.cache_append(d, K, V, Kc, Vc, table, n, n, **s)
    k, v = rsa.cache_read(d, T, Kc, Vc, table, n, n, **s)
    assert k.is_contiguous() and v.is_contiguous() and k.shape == (B, Zkv, T, A)
    ref = rsa.cache_read(rsa.make_cache_desc(Kc, table, Z), T, Kc, Vc, table, n, n, **s)
    assert torch.equal(k, ref[0]) and torch.equal(v, ref[1]) and (k[1, :, 20:] == 0).all()
    if not eight:
        assert torch.equal(k[0], K[0]) and torch.equal(v[1, :, :20], V[1, :, :20])
    y = torch.full_like(x, 7.0)
    rsa.cache_read(d, T, Kc, Vc, table, n, n, K=y[:, Z:Z + Zkv], V=y[:, Z + Zkv:], **s)
    assert torch.equal(y[0, Z:Z + Zkv], k[0]) and torch.equal(y[1, Z + Zkv:, :20], v[1, :, :20])
    assert (y[:, :Z] == 7).all() and (y[1, Z:, 20:] == 7).all()
