"""Which kernels the calls on a cache in e4m3, the one that reads tokens back and the one for several new tokens take, and that
their grids cover the work, on the CPU."""
import re

import pytest

import launches
from paper_2105_13120_amd import rsa
from test_cache_launches import cache


@pytest.fixture(scope="module")
def rec(tmp_path_factory):
    return launches.Recorder(str(tmp_path_factory.mktemp("recorder")))


def chunk(rec, d, T, eight=False, causal=1, pad=0, counts="counts"):
    s = ("Ks", "Vs") if eight else (None, None)
    return rec("cache_attend_chunk", d, T, causal, pad, "Q", "Kc", "Vc", *s, "table", "lengths", counts, "O", "LSE", "ws")


def numbers(name):
    """A template's whole numbers and truths, in a plain name or one that was left mangled."""
    if "<" in name:
        return [int(x) if x.isdigit() else int(x == "true") for x in re.search(r"<(.*)>", name).group(1).split(", ") if x.isdigit() or x in ("true", "false")]
    return [int(x) for x in re.findall(r"L[ib](\d+)E", name)]


@pytest.mark.parametrize("kw,T,few", [
    (dict(Z=8, Zkv=2), 4, True), (dict(Z=8, Zkv=2), 5, False), (dict(Z=2, Zkv=2, A=192), 16, True), (dict(Z=2, Zkv=2, A=192), 17, False),
    (dict(Z=2, Zkv=2, A=128), 32, True), (dict(Z=2, Zkv=2, A=128), 33, False), (dict(Z=2, Zkv=2, A=256), 16, True), (dict(Z=2, Zkv=2, A=256), 32, None),
    (dict(Z=64, Zkv=1), 1, False), (dict(Z=8, Zkv=2, dtype=rsa.RSA_F32), 500, True), (dict(Z=8, Zkv=2, A=256), 9, False)])
@pytest.mark.parametrize("eight", [False, True])
def test_few_rows_and_many(rec, kw, T, few, eight):
    d = cache(**kw)
    if eight and d.dtype == rsa.RSA_F32:
        pytest.skip("pools in e4m3 for calls in bf16")
    few = eight if few is None else few                                              # (heads of 256, 17 to 32 rows)
    names = [k.name for k in chunk(rec, d, T, eight)]
    assert all(("attend_" in n) == few and ("chunk_" in n) != few for n in names), names
    form = numbers(names[0])
    if few:
        assert form[0] == d.A and form[-1] == (2 | eight)                            # several tokens, e4m3
    else:
        assert form[0] == d.A // 64 and form[-1] == eight


# (A, heads, rows of a key head) and the table's slots: 32-row blocks of a wave, waves of different rows, divided or not
@pytest.mark.parametrize("A,B,Zkv,group,T,slots,qb,rw,divided", [
    (64, 1, 2, 1, 33, 64, 1, 2, False), (128, 1, 2, 1, 64, 64, 1, 2, False), (128, 1, 2, 1, 65, 65, 1, 4, False),
    (64, 1, 2, 1, 64, 1024, 1, 2, True), (64, 8, 8, 4, 512, 512, 2, 4, False),
    (64, 1, 8, 4, 480, 480, 1, 4, False), (128, 1, 8, 4, 2048, 2048, 1, 4, False), (128, 1, 8, 4, 2048, 8192, 1, 8, False),
    (128, 8, 8, 4, 512, 512, 1, 8, False), (128, 1, 8, 4, 500, 65536, 1, 4, True), (192, 1, 2, 1, 128, 128, 1, 4, False),
    (192, 1, 2, 1, 129, 129, 1, 8, False), (192, 1, 2, 1, 129, 4096, 1, 8, True), (256, 1, 2, 1, 500, 500, 1, 8, False), (256, 1, 2, 1, 128, 500, 1, 4, False),
    (256, 1, 2, 1, 33, 8192, 1, 2, True), (256, 1, 2, 1, 65, 8192, 1, 4, True), (192, 1, 2, 1, 64, 100, 1, 2, False), (128, 65, 2, 1, 65, 8192, 1, 4, False), (128, 64, 2, 1, 65, 8192, 1, 4, True)])
@pytest.mark.parametrize("eight", [False, True])
def test_work_groups_and_parts(rec, A, B, Zkv, group, T, slots, qb, rw, divided, eight):
    d = cache(A=A, B=B, Z=Zkv * group, Zkv=Zkv, page=1, width=slots, pages=B * slots)
    k = chunk(rec, d, T, eight)
    shares = 2 if rw == 2 or (rw == 4 and (A == 192 or (A == 256 and eight))) else 1                            # waves of the same rows
    assert numbers(k[0].name) == [A // 64, qb, rw * shares, shares, eight] and k[0].threads == 64 * rw * shares
    tiles = -(-T * group // (32 * qb * rw))
    heads = B * Zkv
    need = rsa.cache_chunk_workspace_bytes(d, T)
    if not divided:
        assert k[0].grid == (heads * tiles, 1, 1) and len(k) == 1 and need == 0
        return
    parts, rest = divmod(k[0].grid[0], heads * tiles)
    assert rest == 0 and 2 <= parts <= 32 and parts * 8 <= -(-slots // 64)
    assert len(k) == 2 and k[1].grid == (heads * tiles * qb * rw, 1, 1) and k[1].threads == 256       # 32 rows a work-group
    rows = heads * tiles * 32 * qb * rw
    assert need == 64 * 4 + parts * rows * (A + 2) * 4 and parts * rows * (A + 2) * 4 <= 512 << 20


def test_largest_calls_fit_a_grid(rec):
    for kw, T in ((dict(B=1, Z=1, Zkv=1), 1 << 28), (dict(B=4096, Z=1984, Zkv=1984), 33), (dict(B=4096, Z=1984, Zkv=1984, dtype=rsa.RSA_F32), 33),
                  (dict(B=4096, Z=2048, Zkv=2048, dtype=rsa.RSA_F32), 8), (dict(B=65535, Z=255, Zkv=255, pages=1), 1)):
        d = cache(**kw)
        for k in chunk(rec, d, T):
            assert k.grid[0] * k.threads < 1 << 32 and k.grid[0] > 0


@pytest.mark.parametrize("B,T,counts,work_groups", [(1, 1, False, None), (64, 1, False, None), (8, 2048, True, 1024), (5000, 20, True, None), (1, 1 << 20, False, None)])
@pytest.mark.parametrize("R,adjacent,form", [(0, 0, 0), (64, 1, 1), (8, 1, 1), (64, 0, 2), (16, 0, 2), (8, 0, 3), (6, 1, 3), (20, 0, 3), (2, 0, 3)])
def test_append8(rec, R, adjacent, form, B, T, counts, work_groups):
    d = cache(B=B, width=200)
    (k,) = rec("cache_append8", d, T, "Q", "K", "V", "table", "lengths", "counts" if counts else None, None, R, adjacent, "f" if R else None, "Qr",
               "Kc", "Vc", "Ks", "Vs")
    assert k.threads == 256 and k.grid[1:] == (1, 1) and numbers(k.name) == [64, form]
    assert 1 <= k.grid[0] <= 1 << 20 and (work_groups is None or k.grid[0] == work_groups)


@pytest.mark.parametrize("dtype,eight", [("bf16", False), ("bf16", True), ("f32", False)])
@pytest.mark.parametrize("A", [64, 128, 192, 256])
@pytest.mark.parametrize("B,T,counts,pad", [(1, 1, False, 0), (64, 1, True, 0), (8, 2048, True, 3), (8, 2048, True, 0), (5000, 20, True, 1), (1, 1 << 20, False, 0)])
def test_read(rec, dtype, eight, A, B, T, counts, pad):
    d = cache(B=B, A=A, width=200, dtype=rsa.RSA_BF16 if dtype == "bf16" else rsa.RSA_F32)
    s = ("Ks", "Vs") if eight else (None, None)
    (k,) = rec("cache_read", d, T, pad, "Kc", "Vc", *s, "table", "lengths", "counts" if counts else None, "K", "V")
    assert "read_kernel" in k.name and k.threads == 256 and 1 <= k.grid[0] <= 1 << 20 and numbers(k.name)[-1] == A
