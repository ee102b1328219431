"""Few new tokens of many sequences, on the CPU: the kernel that is launched, its grid, the join's and the workspace go by the same
number of rows of a work-group."""
import pytest

from paper_2105_13120_amd import rsa
from test_cache_chunk_launches import chunk, numbers, rec  # noqa: F401  (rec: a fixture)
from test_cache_launches import cache


# A, sequences, key heads, query heads of one, tokens, slots
@pytest.mark.parametrize("A,B,Zkv,group,T,slots", [
    (64, 64, 8, 4, 8, 16384), (64, 64, 8, 4, 8, 8192), (64, 64, 8, 4, 16, 8192), (64, 40, 14, 1, 58, 7136), (64, 64, 8, 1, 17, 4096),
    (64, 32, 16, 2, 32, 8192), (64, 64, 8, 4, 17, 8192), (64, 64, 8, 4, 32, 8192), (64, 64, 8, 4, 33, 8192), (64, 64, 16, 4, 512, 8192),
    (64, 64, 8, 4, 16, 64), (64, 65, 8, 4, 16, 8192), (64, 128, 8, 4, 100, 8192),
    (128, 32, 8, 4, 16, 4096), (128, 64, 8, 4, 16, 4096), (128, 64, 8, 4, 9, 16384), (128, 64, 8, 4, 20, 4096), (128, 64, 8, 4, 64, 4096),
    (192, 64, 8, 4, 8, 8192), (192, 64, 8, 4, 20, 8192), (192, 64, 8, 4, 64, 8192), (256, 64, 8, 4, 16, 8192), (256, 64, 8, 4, 20, 8192),
    (256, 64, 8, 4, 64, 8192)])
@pytest.mark.parametrize("eight", [False, True])
def test_a_work_groups_rows(rec, A, B, Zkv, group, T, slots, eight):  # noqa: F811
    d = cache(A=A, B=B, Z=Zkv * group, Zkv=Zkv, page=1, width=slots, pages=B * slots)
    k = chunk(rec, d, T, eight)
    _, qb, waves, shares, _ = numbers(k[0].name)
    rows = 32 * qb * waves // shares
    tiles, heads = -(-T * group // rows), B * Zkv
    parts, rest = divmod(k[0].grid[0], heads * tiles)
    assert rest == 0 and k[0].grid[1:] == (1, 1) and k[0].threads == 64 * waves
    need = rsa.cache_chunk_workspace_bytes(d, T)
    if parts == 1:
        assert len(k) == 1 and need == 0
        return
    assert len(k) == 2 and k[1].grid == (heads * tiles * rows // 32, 1, 1)
    assert need >= 64 * 4 + parts * heads * tiles * rows * (A + 2) * 4


@pytest.mark.parametrize("A", [64, 128])
@pytest.mark.parametrize("B,Zkv", [(1, 2), (32, 8), (64, 8), (64, 16), (128, 16)])
@pytest.mark.parametrize("slots", [128, 8192])
@pytest.mark.parametrize("eight", [False, True])
def test_few_rows_have_no_larger_work_groups_however_many_heads_there_are(rec, A, B, Zkv, slots, eight):  # noqa: F811
    d = cache(A=A, B=B, Z=Zkv * 4, Zkv=Zkv, page=1, width=slots, pages=B * slots)
    for T in (9, 16):
        assert numbers(chunk(rec, d, T, eight)[0].name) == [A // 64, 1, 4, 2, eight]
    for T in (17, 32):
        assert numbers(chunk(rec, d, T, eight)[0].name) == [A // 64, 1, 4, 1, eight]
