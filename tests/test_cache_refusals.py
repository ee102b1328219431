"""What the rotation and the cache's entry points refuse on the host, before anything is launched (CPU only)."""
import ctypes

import pytest
import torch

from paper_2105_13120_amd import rsa

p = ctypes.c_void_p(0x10000)
far = ctypes.c_void_p(1 << 45)
odd, word = ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10002)


def ring(**kw):
    d = dict(B=1, Z=2, A=64, L=256, N=4, rank_begin=0, rank_end=4, causal=0, dtype=rsa.RSA_BF16, scale=0.0, flags=rsa.MODE_FUSED)
    d.update(kw)
    return rsa.RSADesc(**d)


def cache(**kw):
    d = dict(B=2, Z=4, Zkv=2, A=64, page=16, pages=8, width=4, dtype=rsa.RSA_BF16, scale=0.0, flags=0)
    d.update(kw)
    for k in ("q_stride", "kv_stride", "o_stride"):
        if k in d:
            d[k] = (ctypes.c_int64 * 3)(*d[k])
    return rsa.CacheDesc(**d)


def rotate(d=None, R=64, freq=p, Q=p, K=p, Qr=p, Kr=p):
    d = ctypes.byref(d or ring())
    status = {f(d, R, 0, freq, Q, K, Qr, Kr, None) for f in (rsa.lib().rsa_rotate, rsa.lib().rsa_rotate_bwd)}
    assert len(status) == 1
    return status.pop()


def test_rotate():
    assert rotate(ring(N=3)) == -2 and rotate(ring(A=96)) == -3
    assert rsa.lib().rsa_rotate(None, 64, 0, p, p, p, p, p, None) == rsa.lib().rsa_rotate_bwd(None, 64, 0, p, p, p, p, p, None) == -1
    for R in (0, -2, 66, 65):
        assert rotate(R=R) == -2
    assert rotate(R=7) == -3
    assert rotate(freq=None) == -1 and rotate(freq=word) == -3
    assert rotate(Q=None, K=None, Qr=None, Kr=None) == -1
    assert rotate(Qr=None) == rotate(Q=None) == rotate(K=None) == rotate(Kr=None) == -1
    for k in ("Q", "K", "Qr", "Kr"):
        assert rotate(**{k: odd}) == -3
    assert rotate(ring(B=1 << 14, Z=1, L=1 << 17, N=1, rank_end=1)) == -3            # B L = 2^31


def append(d=None, T=1, Q=p, K=p, V=p, table=p, lengths=p, counts=p, first=p, R=64, freq=p, Qr=p, Kc=p, Vc=far):
    return rsa.lib().rsa_cache_append(ctypes.byref(d or cache()), T, Q, K, V, table, lengths, counts, first, R, 0, freq, Qr, Kc, Vc, None)


def attend(d=None, Q=p, Kc=p, Vc=far, table=p, lengths=p, O=p, LSE=p, ws=p, n=1 << 40):
    return rsa.lib().rsa_cache_attend(ctypes.byref(d or cache()), Q, Kc, Vc, table, lengths, O, LSE, ws, n, None)


def join(d=None, N=2, Op=p, LSEp=p, O=far, LSE=ctypes.c_void_p(1 << 46)):
    return rsa.lib().rsa_cache_join(ctypes.byref(d or cache()), N, Op, LSEp, O, LSE, None)


BAD = [(dict(**{k: v}), -2) for k in ("B", "Z", "Zkv", "A", "page", "pages", "width") for v in (0, -1)] + [
    (dict(Z=5), -2), (dict(scale=-1.0), -2), (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2),
    (dict(A=96), -3), (dict(A=320), -3), (dict(dtype=2), -3), (dict(flags=1), -3), (dict(B=65536), -3),
    (dict(width=1 << 27), -3),                                                       # 2^31 slots
    (dict(pages=1 << 28, page=8, Zkv=2), -3),                                        # 2^32 rows
    (dict(B=65535, Z=512, Zkv=1), -3),
    (dict(q_stride=(256, 0, 64)), -2), (dict(kv_stride=(-64, 64, 64)), -2), (dict(o_stride=(256, 64, 0)), -2),
    (dict(q_stride=(260, 64, 64)), -3), (dict(kv_stride=(1 << 41, 64, 64)), -3), (dict(o_stride=(256, 66, 64)), -3),
]


@pytest.mark.parametrize("kw,status", BAD)
def test_descriptors(kw, status):
    d = cache(**kw)
    assert append(d) == attend(d) == join(d) == status
    assert rsa.cache_workspace_bytes(d) == 0


def test_append():
    assert rsa.lib().rsa_cache_append(None, 1, p, p, p, p, p, p, p, 64, 0, p, p, p, p, None) == -1
    for k in ("K", "V", "table", "lengths", "Kc", "Vc", "Q", "Qr"):
        assert append(**{k: None}) == -1
    for k in ("Q", "K", "V", "Qr", "Kc", "Vc"):
        assert append(**{k: odd}) == -3
    for k in ("table", "lengths", "counts", "first", "freq"):
        assert append(**{k: word}) == -3
    assert append(T=0) == -2 and append(T=1 << 30) == -3
    for R in (0, 66, 65, -2):
        assert append(R=R) == -2
    assert append(R=9) == -3
    assert append(Vc=p) == -3 and append(Vc=ctypes.c_void_p(0x10000 + 8 * 2 * 16 * 128 - 16)) == -3       # one pool over the other


def test_attend():
    assert rsa.lib().rsa_cache_attend(None, p, p, p, p, p, p, p, p, 0, None) == -1
    for k in ("Q", "Kc", "Vc", "table", "lengths", "O", "LSE"):
        assert attend(**{k: None}) == -1
    for k in ("Q", "Kc", "Vc", "O", "ws"):
        assert attend(**{k: odd}) == -3
    for k in ("table", "lengths", "LSE"):
        assert attend(**{k: word}) == -3


def test_join():
    assert rsa.lib().rsa_cache_join(None, 1, p, p, p, p, None) == -1
    for k in ("Op", "LSEp", "O", "LSE"):
        assert join(**{k: None}) == -1
    assert join(Op=odd) == join(O=odd) == join(LSE=word) == join(LSEp=word) == -3
    assert join(N=0) == -2
    assert join(LSE=p) == -3


def tensors(T=1, B=2, Z=4, Zkv=2, A=64, page=16, pages=8, width=4, dtype=torch.bfloat16):
    e = lambda *s, t=dtype: torch.zeros(*s, dtype=t)
    x = dict(Kc=e(pages, Zkv, page, A), Vc=e(pages, Zkv, page, A), table=e(B, width, t=torch.int32), lengths=e(B, t=torch.int32),
             K=e(B, Zkv, T, A), V=e(B, Zkv, T, A), Q=e(B, Z, T, A), f=e(A // 2, t=torch.float32))
    return rsa.make_cache_desc(x["Kc"], x["table"], Z), x


def call_append(d, x, **kw):
    return rsa.cache_append(d, x["K"], x["V"], x["Kc"], x["Vc"], x["table"], x["lengths"], inv_freq=x["f"], Q=x["Q"], **kw)


def call_attend(d, x, **kw):
    return rsa.cache_attend(d, x["Q"], x["Kc"], x["Vc"], x["table"], x["lengths"], **kw)


@pytest.mark.parametrize("name,bad", [
    ("K", torch.zeros(2, 2, 1, 64)), ("K", torch.zeros(2, 4, 1, 64).bfloat16()), ("V", torch.zeros(2, 2, 2, 64).bfloat16()),
    ("K", torch.zeros(2, 2, 1, 128).bfloat16()[..., :64]), ("K", torch.zeros(2, 2, 64).bfloat16()), ("Kc", torch.zeros(7, 2, 16, 64).bfloat16()),
    ("Vc", torch.zeros(8, 16, 2, 64).bfloat16().transpose(1, 2)), ("table", torch.zeros(2, 4, dtype=torch.int64)),
    ("table", torch.zeros(2, 5, dtype=torch.int32)), ("lengths", torch.zeros(3, dtype=torch.int32)), ("lengths", torch.zeros(2)),
    ("f", torch.zeros(32).double()), ("f", torch.zeros(4, 8)), ("f", torch.zeros(0)), ("f", torch.zeros(129)),
    ("Q", torch.zeros(2, 4, 2, 64).bfloat16()), ("Q", torch.zeros(4, 2, 1, 64).bfloat16().transpose(0, 1))])
def test_tensors_that_do_not_fit_the_descriptor(name, bad):
    d, x = tensors()
    x[name] = bad
    with pytest.raises(ValueError, match="argument"):
        call_append(d, x)
    if name not in ("K", "V", "f"):
        with pytest.raises(ValueError, match="argument"):
            call_attend(d, x)


def test_results_that_do_not_fit():
    d, x = tensors(T=3)
    for kw in (dict(Qr=torch.zeros(2, 4, 1, 64).bfloat16()), dict(counts=torch.zeros(2, dtype=torch.int64)), dict(first=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError, match="argument"):
            call_append(d, x, **kw)
    d, x = tensors()
    for kw in (dict(O=torch.zeros(2, 4, 64).bfloat16()), dict(LSE=torch.zeros(2, 4)), dict(LSE=torch.zeros(2, 4, 1).bfloat16())):
        with pytest.raises(ValueError, match="argument"):
            call_attend(d, x, **kw)
    with pytest.raises(ValueError, match="argument"):
        rsa.cache_join(d, torch.zeros(3, 2, 4, 1, 64).bfloat16(), torch.zeros(2, 2, 4, 1))
    with pytest.raises(ValueError, match="argument"):
        rsa.cache_join(d, torch.zeros(3, 2, 4, 64).bfloat16(), torch.zeros(3, 2, 4, 1))
    with pytest.raises(ValueError, match="argument"):
        rsa.cache_append(d, x["K"], x["V"], x["Kc"], x["Vc"], x["table"], x["lengths"], Qr=x["Q"])
    with pytest.raises((ValueError, TypeError)):
        rsa.cache_append(d, x["K"], x["V"], x["Kc"], x["Vc"], None, x["lengths"])
    none = x["K"][:, :, :0]
    with pytest.raises(ValueError, match="argument"):
        rsa.cache_append(d, none, none, x["Kc"], x["Vc"], x["table"], x["lengths"])
    K = torch.zeros(1, 2, 256, 64).bfloat16()
    d = rsa.make_desc(K, 4, rank_end=1)
    for bad in (dict(Q=K), dict(Q=K[:, :, :64].float()), dict(K=K[:, :, :64]), dict(K=K, Kr=K[:, :, :64]), dict(Qr=K)):
        with pytest.raises(ValueError, match="argument"):
            rsa.rotate(d, torch.zeros(32), **bad)
    with pytest.raises(TypeError):
        rsa.cache_join(d, K, K)                                                      # another kind of descriptor
    with pytest.raises(TypeError):
        rsa.rotate(tensors()[0], torch.zeros(32), K=K)


@pytest.mark.parametrize("N", [0, -1])
def test_rotate_with_descriptors_that_divide_by_nothing(N):
    K = torch.zeros(1, 2, 256, 64).bfloat16()
    d = rsa.make_desc(K, 4)
    d.N = N
    with pytest.raises((ZeroDivisionError, ValueError, rsa.RSAError)):
        rsa.rotate(d, torch.zeros(32), Q=K)


@pytest.mark.skipif(torch.cuda.is_available(), reason="without a GPU")
def test_tensors_on_the_cpu_are_refused_last():
    d, x = tensors()
    for call in (call_append, call_attend):
        with pytest.raises((AssertionError, RuntimeError)):
            call(d, x)
    K = torch.zeros(1, 2, 256, 64).bfloat16()
    with pytest.raises((AssertionError, RuntimeError)):
        rsa.rotate(rsa.make_desc(K, 4), torch.zeros(32), K=K)
