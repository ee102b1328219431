"""How exactly up to 32 rows of a key head attend, where a lost bit of a probability shows."""
import numpy as np
import pytest
import torch

from cache8_helpers import i32
from cache_helpers import F32, STEP, within
from chunk_checks import check
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu

ROOM = 128       # slots of a page


def cancelling(n, first, second, B, Z, T, A, eight):
    """Two slots of n count: probabilities 1 and p of each row before they are divided by their sum, and in a
    column or more of each row values that cancel to 2^-15 of themselves.  Values have four bits (as e4m3 has), their ratios do not, and
    scores are sums of two products, of 16 bits (k = 0, -1 and, for slots that do not count, -32768)."""
    rng = np.random.default_rng(60 + n + A)
    dt = torch.float8_e4m3fn if eight else torch.bfloat16
    scale = 0.125
    v0, v1 = (torch.from_numpy(rng.integers(lo, lo + 8, (B, A)) / 8.0).double() for lo in (8, 8))
    v1 = v1 * torch.from_numpy(2.0 ** rng.integers(1, 3, (B, A)))
    ratio = v0 / v1                                           # from 0.13 to 0.94
    want = ratio[:, torch.arange(Z * T) % A].reshape(B, Z, T).log() / -scale
    Q = torch.zeros(B, Z, T, A, dtype=torch.bfloat16)
    Q[..., 0] = want.bfloat16()
    Q[..., 1] = (want - Q[..., 0].double()).bfloat16()
    K, V = (torch.zeros(B, 1, ROOM, A, dtype=torch.float64) for _ in range(2))
    K[:, 0, :n, 0] = -1.0 if eight else -32768.0
    K[:, 0, first, 0] = 0.0
    K[:, 0, second, :2] = -1.0
    V[:, 0, :n] = 1.0
    V[:, 0, first], V[:, 0, second] = v0, -v1
    s = {k: torch.full((B, 1, ROOM), 127, dtype=torch.uint8) for k in ("Ks", "Vs")}
    s["Ks"][:, 0, :n] = 127 + 15
    s["Ks"][:, 0, second] = 127
    pools = [x.to(dt) for x in (K, V)]
    p = torch.exp(-(Q[..., 0].double() + Q[..., 1].double()) * scale)[..., None]
    v0, v1 = v0[:, None, None], v1[:, None, None]
    O, PV = (v0 - p * v1) / (1 + p), (v0 + p * v1) / (1 + p)
    return Q, pools, s if eight else {}, O.numpy(), PV.numpy(), scale


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("A", [64, 128, 192, 256])
@pytest.mark.parametrize("Z,T", [(4, 4), (1, 17), (3, 8), (4, 8), (1, 32)])
@pytest.mark.parametrize("n,first,second,width", [(2, 0, 1, 1), (40, 0, 20, 1), (64, 3, 60, 1), (128, 70, 90, 1), (60, 40, 35, 200)])
def test_probabilities_are_held_to_32_bits(n, first, second, width, Z, T, A, eight):
    """A score is off by the rounding of its sum, the exponent by three more (scale log2(e) and their product), 4 2^-24 of at most 2.1, exp by 2^-22:
    p by less than 2^-20.  Sums are of two slots' three parts of p, of two waves' or more parts of a walk, and divided: 12 roundings; the result is rounded
    once."""
    B = 24
    Q, pools, s, O, PV, scale = cancelling(n, first, second, B, Z, T, A, eight)
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(B)
    Kc, Vc = (x.cuda() for x in pools)
    d = rsa.make_cache_desc(Kc, table, Z, scale=scale)
    got, _ = rsa.cache_attend_chunk(d, Q.cuda(), Kc, Vc, table.cuda(), i32([n] * B), causal=False, **{k: x.cuda() for k, x in s.items()})
    assert (np.abs(O) < 2.0 ** -13 * PV).sum() >= B * Z * T    # (some of each row cancel)
    within(got, O, (2.0 ** -20 + 12 * F32) * PV + STEP["bf16"] * np.abs(O), "O")


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("A,Z,Zkv,T,lengths", [
    (64, 4, 1, 5, [700, 33, 5]), (64, 2, 2, 32, [90, 1000]), (64, 8, 2, 8, [5000, 16]), (128, 2, 2, 17, [60, 700]), (128, 4, 1, 8, [3000, 9]), (128, 8, 2, 8, [130] * 40),
    (192, 3, 1, 9, [200, 64]), (192, 1, 1, 32, [2000]), (256, 4, 2, 10, [300, 41]), (256, 2, 2, 32, [1500, 32]), (256, 1, 1, 20, [64, 65])])
def test_up_to_32_rows(A, Z, Zkv, T, lengths, eight):
    check("bf16", Z, Zkv, A, 16, T, lengths, eight=eight, all_bits=True, seed=T)
