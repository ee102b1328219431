"""What the calls on a cache in e4m3, the one that reads tokens back and the one for several new tokens refuse on the host, before
anything is launched (CPU only)."""
import ctypes

import pytest
import torch

import launches
from paper_2105_13120_amd import rsa
from test_cache_refusals import BAD, cache

# tensors of the calls below, 16 MB apart
NAMES = ("Q", "K", "V", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "counts", "first", "inv_freq", "Qr", "O", "LSE", "ws")
AT = {n: (1 << 40) + (i << 24) for i, n in enumerate(NAMES)}
B, Z, ZKV, A, PAGE, PAGES, WIDTH, T = 2, 4, 2, 64, 16, 200, 1000, 3
ROWS = PAGES * ZKV * PAGE
SIZE = dict(Q=B * Z * T * A * 2, K=B * ZKV * T * A * 2, V=B * ZKV * T * A * 2, Kc=ROWS * A, Vc=ROWS * A, Ks=ROWS, Vs=ROWS, table=B * WIDTH * 4,
            lengths=B * 4, counts=B * 4, first=B * 4, inv_freq=A // 2 * 4, Qr=B * Z * T * A * 2, O=B * Z * T * A * 2, LSE=B * Z * T * 4)


def desc(**kw):
    return cache(**{**dict(B=B, Z=Z, Zkv=ZKV, A=A, page=PAGE, pages=PAGES, width=WIDTH), **kw})


def append8(d=None, T=T, R=A, lib=None, **at):
    a = {**AT, **at}
    front = [a[n] for n in ("Q", "K", "V", "table", "lengths", "counts", "first")]
    return (lib or rsa.lib()).rsa_cache_append8(ctypes.byref(d or desc()), T, *front, R, 0, *(a[n] for n in ("inv_freq", "Qr", "Kc", "Vc", "Ks", "Vs")), None)


def attend8(d=None, n=1 << 30, lib=None, **at):
    a = {**AT, **at}
    return (lib or rsa.lib()).rsa_cache_attend8(ctypes.byref(d or desc()), *(a[n] for n in ("Q", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "O", "LSE", "ws")), n, None)


def read(d=None, T=T, pad=3, lib=None, **at):
    a = {**AT, **at}
    return (lib or rsa.lib()).rsa_cache_read(ctypes.byref(d or desc()), T, pad, *(a[n] for n in ("Kc", "Vc", "Ks", "Vs", "table", "lengths", "counts", "K", "V")), None)


def chunk(d=None, T=T, causal=1, pad=3, n=1 << 30, lib=None, **at):
    a = {**AT, **at}
    return (lib or rsa.lib()).rsa_cache_attend_chunk(ctypes.byref(d or desc()), T, causal, pad,
                                                     *(a[n] for n in ("Q", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "counts", "O", "LSE", "ws")), n, None)


CALLS = {  # call: tensors that have to be there, aligned to 16 bytes, to 4
    append8: (("K", "V", "table", "lengths", "Kc", "Vc", "Ks", "Vs", "Q", "Qr"), ("Q", "K", "V", "Qr", "Kc", "Vc"), ("table", "lengths", "counts", "first", "inv_freq")),
    attend8: (("Q", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "O", "LSE"), ("Q", "Kc", "Vc", "O", "ws"), ("table", "lengths", "LSE")),
    read: (("Kc", "Vc", "Ks", "Vs", "table", "lengths", "K", "V"), ("Kc", "Vc", "K", "V"), ("table", "lengths", "counts")),
    chunk: (("Q", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "O", "LSE"), ("Q", "Kc", "Vc", "O", "ws"), ("table", "lengths", "counts", "LSE")),
}


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__)
def test_pointers(call):
    there, by_16, by_4 = CALLS[call]
    for k in there:
        assert call(**{k: None}) == -1, k
    for k in by_16:
        assert call(**{k: AT[k] + 8}) == -3, k
    for k in by_4:
        assert call(**{k: AT[k] + 2}) == -3, k


@pytest.mark.parametrize("kw,status", BAD)
def test_descriptors(kw, status):
    d = cache(**kw)
    assert append8(d) == attend8(d) == read(d) == chunk(d) == status
    assert rsa.cache_chunk_workspace_bytes(d, 4) == 0
    none = [None] * 16
    L = rsa.lib()
    assert L.rsa_cache_append8(None, 1, *none[:7], 64, 0, *none[:7]) == L.rsa_cache_attend8(None, *none[:10], 0, None) == -1
    assert L.rsa_cache_read(None, 1, 0, *none[:10]) == L.rsa_cache_attend_chunk(None, 1, 1, 0, *none[:11], 0, None) == -1


def test_types_and_numbers():
    f32 = desc(dtype=rsa.RSA_F32)
    assert append8(f32) == attend8(f32) == read(f32) == chunk(f32) == -3              # pools in e4m3 for calls in bf16
    for call in (append8, read, chunk):
        assert call(T=0) == call(T=-1) == -2 and call(T=1 << 30) == -3                # B T = 2^31
    for R in (0, -2, 66, 65):
        assert append8(R=R) == -2
    assert append8(R=9) == -3
    for t in (0, -5):
        assert rsa.cache_chunk_workspace_bytes(desc(), t) == 0
    # T Z = 2^31, and B Z T A beyond 2^34
    for kw, t in ((dict(B=1, Z=1 << 20, Zkv=1 << 20, pages=8), 1 << 11), (dict(B=1, Z=8, Zkv=8, A=256), (1 << 23) + 1), (dict(B=1, Z=4, Zkv=2), (1 << 26) + 1)):
        assert chunk(desc(**kw), t) == -3 and rsa.cache_chunk_workspace_bytes(desc(**kw), t) == 0


def test_workspaces():
    few, many = desc(), desc(Z=32, Zkv=2)
    for d, t, part in ((few, 3, 0), (many, 100, 0)):
        need = rsa.cache_chunk_workspace_bytes(d, t)
        assert need > 0
        assert chunk(d, t, n=need - 1) == chunk(d, t, ws=None) == -4
    need = rsa.cache_workspace_bytes(few)
    assert need > 0 and attend8(few, n=need - 1) == attend8(few, ws=None) == -4
    assert rsa.cache_chunk_workspace_bytes(desc(width=2), 100) == 0                   # 32 slots: nothing to divide


@pytest.fixture(scope="module")
def rec(tmp_path_factory):
    return launches.Recorder(str(tmp_path_factory.mktemp("recorder")))


def test_results_over_other_tensors(rec):
    """Each result at the place of another tensor, over its end and over its start, is refused; right behind it, taken."""
    chunk_ins, ws = ("Q", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "counts"), rsa.cache_chunk_workspace_bytes(desc(), T)
    pairs = [(append8, out, ("K", "V", "table", "lengths", "counts", "first", "inv_freq") + more) for out, more in (
        ("Kc", ("Vc", "Q", "Qr", "Ks", "Vs")), ("Vc", ("Kc", "Q", "Qr", "Ks", "Vs")), ("Qr", ("Ks", "Vs")), ("Ks", ("Vs", "Kc", "Vc", "Q", "Qr")), ("Vs", ("Ks", "Kc", "Vc", "Q", "Qr")))]
    pairs += [(read, "K", ("V", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "counts")), (read, "V", ("K", "Kc", "Vc", "Ks", "Vs", "table", "lengths", "counts"))]
    pairs += [(chunk, "O", chunk_ins + ("LSE", "ws")), (chunk, "LSE", chunk_ins + ("ws",)), (chunk, "ws", chunk_ins)]
    assert 0 < ws < 1 << 24
    size = {**SIZE, "ws": ws}
    for call, out, others in pairs:
        assert call(lib=rec.lib) == 0
        for x in others:
            for at in (AT[x], AT[x] + size[x] - 16 if size[x] > 16 else AT[x], AT[x] - size[out] + 16 if size[out] > 16 else AT[x]):
                if at % 16 == 0:
                    assert call(lib=rec.lib, **{out: at}) == -3, (call, out, x)
            assert call(lib=rec.lib, **{out: AT[x] + -(-size[x] // 16) * 16}) == 0, (call, out, x)
    assert append8(lib=rec.lib, Qr=AT["Q"]) == 0                                      # in place
    assert append8(lib=rec.lib, Qr=AT["Q"] + 16) == -3
    # results between each other's rows
    every = (2 * ZKV * T * A, 2 * T * A, A)
    assert read(desc(kv_stride=every), lib=rec.lib, V=AT["K"] + T * A * 2) == 0 and read(desc(kv_stride=every), lib=rec.lib, V=AT["K"]) == -3


def tensors(T=3, eight=True, dtype=torch.bfloat16, B=2, Z=4, Zkv=2, A=64, page=16, pages=8, width=4):
    e = lambda *s, t=dtype: torch.zeros(*s, dtype=t)
    pool = torch.float8_e4m3fn if eight else dtype
    x = dict(Kc=e(pages, Zkv, page, A, t=pool), Vc=e(pages, Zkv, page, A, t=pool), table=e(B, width, t=torch.int32), lengths=e(B, t=torch.int32),
             counts=e(B, t=torch.int32), K=e(B, Zkv, T, A), V=e(B, Zkv, T, A), Q=e(B, Z, T, A), O=e(B, Z, T, A), LSE=e(B, Z, T, t=torch.float32))
    x["Ks"], x["Vs"] = (e(pages, Zkv, page, t=torch.uint8) if eight else None for _ in range(2))
    return rsa.make_cache_desc(x["Kc"], x["table"], Z), x


def calls(d, x, T=3):
    """Each of the four on these tensors: its name, what it takes of them, the call."""
    s = dict(Ks=x["Ks"], Vs=x["Vs"])
    pools = x["Kc"], x["Vc"], x["table"], x["lengths"]
    common = {"Kc", "Vc", "Ks", "Vs", "table", "lengths"}
    return [("append", common | {"K", "V", "counts"}, lambda: rsa.cache_append(d, x["K"], x["V"], *pools, x["counts"], **s)),
            ("read", common | {"K", "V", "counts"}, lambda: rsa.cache_read(d, T, *pools, x["counts"], x["K"], x["V"], **s)),
            ("attend", common, lambda: rsa.cache_attend(d, x["Q"][:, :, :1].contiguous(), *pools, **s)),
            ("chunk", common | {"Q", "O", "LSE", "counts"}, lambda: rsa.cache_attend_chunk(d, x["Q"], *pools, x["counts"], True, x["O"], x["LSE"], **s))]


E4, BF = torch.float8_e4m3fn, torch.bfloat16


@pytest.mark.parametrize("name,bad", [
    ("Kc", torch.zeros(8, 2, 16, 64, dtype=BF)), ("Vc", torch.zeros(8, 2, 16, 64, dtype=BF)), ("Kc", torch.zeros(8, 2, 16, 64).to(torch.float8_e5m2)),
    ("Vc", torch.zeros(7, 2, 16, 64).to(E4)), ("Vc", torch.zeros(8, 16, 2, 64).to(E4).transpose(1, 2)),
    ("Ks", None), ("Vs", None), ("Ks", torch.zeros(8, 2, 16)), ("Vs", torch.zeros(8, 2, 16, dtype=torch.int8)), ("Ks", torch.zeros(8, 2, 15, dtype=torch.uint8)),
    ("Vs", torch.zeros(8, 16, 2, dtype=torch.uint8).transpose(1, 2)), ("Ks", torch.zeros(8, 2, 16, 1, dtype=torch.uint8)),
    ("table", torch.zeros(2, 4, dtype=torch.int64)), ("table", torch.zeros(2, 5, dtype=torch.int32)), ("table", None), ("lengths", None),
    ("lengths", torch.zeros(3, dtype=torch.int32)), ("counts", torch.zeros(2)), ("counts", torch.zeros(2, 1, dtype=torch.int32)),
    ("K", torch.zeros(2, 2, 3, 64)), ("V", torch.zeros(2, 2, 2, 64, dtype=BF)), ("K", torch.zeros(2, 2, 3, 128, dtype=BF)[..., :64]),
    ("Q", torch.zeros(2, 4, 3, 64)), ("Q", torch.zeros(2, 2, 3, 64, dtype=BF)), ("Q", torch.zeros(2, 3, 4, 64, dtype=BF).transpose(1, 2)),
    ("O", torch.zeros(2, 4, 2, 64, dtype=BF)), ("O", torch.zeros(2, 4, 3, 64)), ("LSE", torch.zeros(2, 4, 3, dtype=BF)), ("LSE", torch.zeros(2, 4))])
def test_tensors_that_do_not_fit_the_descriptor(name, bad):
    d, x = tensors()
    x[name] = bad
    reached = [c for c in calls(d, x) if name in c[1]]
    assert reached
    for what, _, call in reached:
        with pytest.raises((ValueError, TypeError)) as said:
            call()
        assert "argument" in str(said.value) or bad is None, what


@pytest.mark.parametrize("name", ["Ks", "Vs"])
def test_exponents_without_a_pool_in_8_bits(name):
    d, x = tensors(eight=False)
    x[name] = torch.zeros(8, 2, 16, dtype=torch.uint8)
    for what, _, call in calls(d, x):
        with pytest.raises(ValueError, match="argument"):
            call()


def test_pools_in_8_bits_with_queries_in_32():
    d, x = tensors()
    for k in ("Q", "K", "V", "O"):
        x[k] = x[k].float()
    for what, _, call in calls(d, x):
        with pytest.raises(ValueError, match="argument"):
            call()
    d.dtype = rsa.RSA_F32
    for what, _, call in calls(d, x):
        with pytest.raises((ValueError, rsa.RSAError, AssertionError, RuntimeError)):
            call()


def test_numbers_of_tokens_and_strides():
    d, x = tensors()
    pools, s = (x["Kc"], x["Vc"], x["table"], x["lengths"]), dict(Ks=x["Ks"], Vs=x["Vs"])
    for T in (0, -1, 1 << 31, 1 << 62):
        with pytest.raises(ValueError, match="argument"):
            rsa.cache_read(d, T, *pools, **s)
    for T in (1.5, "1", None):
        with pytest.raises((TypeError, ValueError)):
            rsa.cache_read(d, T, *pools, **s)
    with pytest.raises(ValueError, match="argument"):
        rsa.cache_attend_chunk(d, x["Q"][:, :, :0], *pools, **s)
    with pytest.raises(ValueError, match="argument"):
        rsa.cache_attend_chunk(d, x["Q"][:, :, 0], *pools, **s)
    wide = torch.zeros(2, 3, 2, 64, dtype=BF).transpose(1, 2)                         # tokens with their heads side by side
    d = rsa.make_cache_desc(x["Kc"], x["table"], 4, K=wide)
    for kw in (dict(K=wide), dict(V=wide), dict(K=wide, V=x["V"])):                   # a new tensor would not have these strides
        with pytest.raises(ValueError, match="argument"):
            rsa.cache_read(d, 3, *pools, **kw, **s)
    d, _ = tensors()
    with pytest.raises(ValueError, match="argument"):
        rsa.cache_read(d, 3, *pools, K=wide, V=wide, **s)                             # ... or the descriptor's
    with pytest.raises(TypeError):
        rsa.cache_attend_chunk(rsa.make_desc(torch.zeros(1, 2, 256, 64, dtype=BF), 4), x["Q"], *pools, **s)


@pytest.mark.skipif(torch.cuda.is_available(), reason="without a GPU")
def test_tensors_on_the_cpu_are_refused_last():
    for eight in (False, True):
        d, x = tensors(eight=eight)
        for what, _, call in calls(d, x):
            with pytest.raises((AssertionError, RuntimeError)):
                call()
