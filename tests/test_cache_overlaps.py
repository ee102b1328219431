"""Results over other tensors of a call on the cache: refused on the host, before anything is launched (CPU only)."""
import ctypes

import pytest

import launches
from paper_2105_13120_amd import rsa

# tensors of the calls below, 16 MB apart
AT = {n: (1 << 40) + (i << 24) for i, n in enumerate(
    ("Q", "K", "V", "Kc", "Vc", "table", "lengths", "counts", "first", "inv_freq", "Qr", "O", "LSE", "ws", "Op", "LSEp"))}
B, Z, ZKV, A, PAGE, PAGES, WIDTH, T, N = 2, 4, 2, 64, 16, 200, 1000, 3, 5
# bytes of a dense one, bf16
SIZE = dict(Q=B * Z * T * A * 2, K=B * ZKV * T * A * 2, V=B * ZKV * T * A * 2, Kc=PAGES * ZKV * PAGE * A * 2, Vc=PAGES * ZKV * PAGE * A * 2,
            table=B * WIDTH * 4, lengths=B * 4, counts=B * 4, first=B * 4, inv_freq=A // 2 * 4, Qr=B * Z * T * A * 2,
            O=B * Z * A * 2, LSE=B * Z * 4, Op=N * B * Z * A * 2, LSEp=N * B * Z * 4)


@pytest.fixture(scope="module")
def rec(tmp_path_factory):
    return launches.Recorder(str(tmp_path_factory.mktemp("recorder")))


def desc(**kw):
    d = rsa.CacheDesc(B=B, Z=Z, Zkv=ZKV, A=A, page=PAGE, pages=PAGES, width=WIDTH, dtype=rsa.RSA_BF16, scale=0.0, flags=0)
    for k, st in kw.items():
        setattr(d, k, (ctypes.c_int64 * 3)(*st))
    return d


def append(rec, at, d=None):
    a = [at[n] for n in ("Q", "K", "V", "table", "lengths", "counts", "first")]
    return rec.lib.rsa_cache_append(ctypes.byref(d or desc()), T, *a, A, 0, at["inv_freq"], at["Qr"], at["Kc"], at["Vc"], None)


def attend(rec, at, d=None):
    d = d or desc()
    a = [at[n] for n in ("Q", "Kc", "Vc", "table", "lengths", "O", "LSE", "ws")]
    return rec.lib.rsa_cache_attend(ctypes.byref(d), *a, 1 << 30, None)


def join(rec, at, d=None):
    return rec.lib.rsa_cache_join(ctypes.byref(d or desc()), N, *(at[n] for n in ("Op", "LSEp", "O", "LSE")), None)


def check(rec, call, out, others, size=SIZE):
    assert call(rec, AT) == 0
    for x in others:
        for at in (AT[x], AT[x] + size[x] - 16 if size[x] > 16 else AT[x], AT[x] - size[out] + 16 if size[out] > 16 else AT[x]):
            if at % 16 == 0:
                assert call(rec, {**AT, out: at}) == -3, (out, x)
        behind = AT[x] + -(-size[x] // 16) * 16
        assert call(rec, {**AT, out: behind}) == 0, (out, x)


def test_append(rec):
    ins = ("K", "V", "table", "lengths", "counts", "first", "inv_freq")
    check(rec, append, "Kc", ins + ("Vc", "Q", "Qr"))
    check(rec, append, "Vc", ins + ("Kc", "Q", "Qr"))
    check(rec, append, "Qr", ins)
    assert append(rec, {**AT, "Qr": AT["Q"]}) == 0                                   # in place
    assert append(rec, {**AT, "Qr": AT["Q"] + 16}) == append(rec, {**AT, "Qr": AT["Q"] - 16}) == -3
    assert append(rec, {**AT, "Q": None, "Qr": None, "counts": None, "first": None, "inv_freq": None}) == 0


def test_attend(rec):
    size = {**SIZE, "Q": B * Z * A * 2, "ws": rsa.cache_workspace_bytes(desc())}
    ins = ("Q", "Kc", "Vc", "table", "lengths")
    assert 0 < size["ws"] < 1 << 20
    for out, others in (("O", ins + ("LSE", "ws")), ("LSE", ins + ("ws",)), ("ws", ins)):
        check(rec, attend, out, others, size)


def test_join(rec):
    check(rec, join, "O", ("Op", "LSEp", "LSE"))
    check(rec, join, "LSE", ("Op", "LSEp"))


def test_slices_of_one_projection_may_lie_between_each_other(rec):
    """Tensors with gaps: Qr over the rows of Q among those of K and V, and O in the gaps of another."""
    row = (Z + 2 * ZKV) * A
    packed = (T * row, A, row)
    x = AT["Q"]
    at = {**AT, "Q": x, "Qr": x, "K": x + Z * A * 2, "V": x + (Z + ZKV) * A * 2}
    assert append(rec, at, desc(q_stride=packed, kv_stride=packed)) == 0
    every = (2 * Z * A, 2 * A, A)
    assert attend(rec, {**AT, "O": AT["Q"] + A * 2}, desc(q_stride=every, o_stride=every)) == 0


def test_what_a_refusal_says():
    """One text for all calls: it names what the cache's and the rotation's need, not the ring's limits alone."""
    said = rsa.strerror(-3)
    for word in ("even R", "calls on the cache", "strides", "flags", "over another tensor", "calls of the ring", "head size of 64 or 128"):
        assert word in said, word
    odd = desc()
    odd.flags = 1
    assert rsa.lib().rsa_cache_join(ctypes.byref(odd), 1, None, None, None, None, None) == -3
