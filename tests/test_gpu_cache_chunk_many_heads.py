"""A few new tokens of each of many sequences of uneven lengths, whose walks are divided, against the definition in 64 bits."""
import pytest

from chunk_checks import check

pytestmark = pytest.mark.gpu

UNEVEN = [3 + 131 * b for b in range(63)] + [8192]
ONE_LONG = [20 + 3 * b for b in range(63)] + [30000]


@pytest.mark.parametrize("A,Z,Zkv,T,lengths", [
    (64, 32, 8, 8, UNEVEN), (64, 32, 8, 8, ONE_LONG), (64, 32, 8, 16, UNEVEN), (64, 14, 14, 58, UNEVEN[-40:]), (64, 8, 8, 17, ONE_LONG),
    (128, 32, 8, 16, UNEVEN[-32:]), (128, 32, 8, 16, ONE_LONG)])
@pytest.mark.parametrize("eight", [False, True])
def test_few_rows_of_many_heads(A, Z, Zkv, T, lengths, eight):
    check("bf16", Z, Zkv, A, 16, T, lengths, eight=eight, seed=len(lengths) + T)
