"""Which kernels the calls on the cache and the rotation take, and that their grids cover the work, on the CPU."""
import ctypes
import re

import pytest

import launches
from paper_2105_13120_amd import rsa


@pytest.fixture(scope="module")
def rec(tmp_path_factory):
    return launches.Recorder(str(tmp_path_factory.mktemp("recorder")))


def cache(**kw):
    d = dict(B=2, Z=8, Zkv=2, A=64, page=16, pages=8, width=4, dtype=rsa.RSA_BF16, scale=0.0, flags=0)
    d.update(kw)
    return rsa.CacheDesc(**d)


def attend(rec, d):
    return rec("cache_attend", d, "Q", "Kc", "Vc", "table", "lengths", "O", "LSE", "ws")


@pytest.mark.parametrize("kw,whole,queries", [
    (dict(width=48), True, 1), (dict(width=49), False, 1), (dict(width=3, page=256), True, 1), (dict(width=769, page=1), False, 1),
    (dict(width=24, dtype=rsa.RSA_F32), True, 1), (dict(width=25, dtype=rsa.RSA_F32), False, 1), (dict(width=12, A=256), True, 1),
    (dict(width=100, Z=32), False, 1), (dict(width=100, Z=34), False, 2), (dict(width=100, Z=80, A=128), False, 2),
    (dict(width=100, Z=80, A=192), False, 1), (dict(width=100, B=4096), False, 1), (dict(width=100, B=4097), True, 1),
    (dict(width=1 << 20, page=2047, Zkv=8, B=4), False, 1), (dict(width=1 << 20, page=2047, Zkv=8, B=9), True, 1)])
def test_whole_segments_or_shares(rec, kw, whole, queries):
    d = cache(**kw)
    group = d.Z // d.Zkv
    tiles = -(-group // (16 * queries))
    k = attend(rec, d)
    # (bf16 in a template's arguments stays as the compiler writes it: ..kernelI<type>Li<A>ELi<queries>E..)
    forms = [re.search(r"attend_(\w+?)_kernel(?:I\w+?Li|<float, )(\d+)(?:ELi|, )(\d)", x.name).groups() for x in k]
    assert forms == [(f, str(d.A), str(queries)) for f in (["whole"] if whole else ["shares", "join"])]
    segments = d.B * d.Zkv * tiles
    if whole:
        assert k[0].grid == (segments, 1, 1) and rsa.cache_workspace_bytes(d) == 0
    else:
        shares, rows = k[0].grid[0], min(group, 16 * queries)
        assert k[1].grid[:2] == (segments if segments <= shares else shares, rows)      # a work-group a note and row
        assert rsa.cache_workspace_bytes(d) >= 16 * shares + 2 * shares * rows * (d.A + 4) * 4


@pytest.mark.parametrize("kw,blocks", [(dict(B=1, Z=4, Zkv=1, A=128, width=4096), 4), (dict(B=1, Z=4, Zkv=1, A=128, width=400), 1), (dict(B=2, Z=4, Zkv=2, A=128, width=4096), 4),
                                       (dict(B=5, Z=4, Zkv=1, A=128, width=4096), 1), (dict(B=1, Z=40, Zkv=1, A=256, width=4096), 1), (dict(B=1, Z=30, Zkv=1, A=256, width=4096), 8)])
def test_segments_of_many_parts_are_joined_by_columns(rec, kw, blocks):
    assert attend(rec, cache(**kw))[1].grid[2] == blocks


def test_one_byte_less_of_workspace_is_refused():
    d = cache(width=100)
    p, need = ctypes.c_void_p(0x10000), rsa.cache_workspace_bytes(d)
    assert need > 0
    for ws, n in ((p, need - 1), (None, 1 << 40)):
        assert rsa.lib().rsa_cache_attend(ctypes.byref(d), p, p, p, p, p, p, p, ws, n, None) == -4


@pytest.mark.parametrize("A,R,dtype,rows", [(64, 64, "bf16", 8), (128, 128, "bf16", 8), (64, 8, "bf16", 8), (64, 20, "bf16", 8),
                                            (128, 6, "bf16", 8), (64, 64, "f32", 8), (192, 192, "f32", 4), (256, 256, "f32", 4), (256, 6, "f32", 4)])
@pytest.mark.parametrize("L,B", [(64, 1), (4096, 3), (1 << 20, 1), (1 << 30, 1)])
def test_rotation_covers_all_rows(rec, A, R, dtype, rows, L, B):
    code = rsa.RSA_BF16 if dtype == "bf16" else rsa.RSA_F32
    d = launches.descriptor(B, 2, L, 1, A, dtype=code, mode=rsa.MODE_FUSED if dtype == "bf16" else rsa.MODE_STAGED)
    for tensors, sides in ((("Q", "K", "Qr", "Kr"), 2), (("Q", None, "Qr", None), 1), ((None, "K", None, "Kr"), 1)):
        (k,) = rec("rotate", d, R, 0, "f", *tensors)
        x, y, z = k.grid
        assert k.threads == 256 and x * z >= sides * -(-L // rows) and x * (z - 1) < sides * -(-L // rows)
        assert x * 256 < 1 << 32 and 1 <= y <= B


@pytest.mark.parametrize("T,B,counts,work_groups", [(1, 1, False, 3), (1, 64, False, 24), (2048, 8, False, 2048), (2048, 8, True, 1024), (1, 9, True, 6)])
def test_append(rec, T, B, counts, work_groups):
    d = cache(B=B, width=200)                   # 8 rows a tile, 12 heads in two passes of eight
    (k,) = rec("cache_append", d, T, "Q", "K", "V", "table", "lengths", "counts" if counts else None, None, 64, 0, "f", "Qr", "Kc", "Vc")
    assert k.threads == 256 and k.grid[1:] == (1, 1)
    tiles = -(-B * T // 8)
    assert k.grid[0] == (1024 if counts and T > 8 else tiles * min(2, -(-512 // tiles)))


def test_join_covers_all_rows(rec):
    d = cache(B=300, Z=7, Zkv=7, A=192)
    (k,) = rec("cache_join", d, 5, "Op", "Lp", "O", "L")
    assert k.grid[0] * 256 >= 300 * 7 * 192 // 8 > (k.grid[0] - 1) * 256
