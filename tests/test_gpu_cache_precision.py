"""How exactly a new token attends and shares are joined, where a lost bit shows."""
import numpy as np
import pytest
import torch

from cache_helpers import DTYPES, F32, STEP, f64, within
from oracle import cache as oracle
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu


def one_page(keys, values, width, room=64):
    """Pools, table and lengths of sequences (B, Zkv, n, A), a page of `room` slots each, in tables of `width` entries."""
    B, Zkv, n, A = keys.shape
    Kc, Vc = (torch.full((B, Zkv, room, A), float("nan"), dtype=keys.dtype) for _ in range(2))
    Kc[:, :, :n], Vc[:, :, :n] = keys, values
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(B)
    return Kc.cuda(), Vc.cuda(), table.cuda(), torch.full((B,), n, dtype=torch.int32).cuda()


def cancelling(n, B=64, Z=16, A=64):
    """Two slots of n count, the first and the last: probabilities 1 and p of each query before they are divided by their sum,
    and in each column values that cancel for one of the queries.  Scores are single products (k = 0, -1 and, for slots that do
    not count, -30000)."""
    rng = np.random.default_rng(30 + n)
    Q, K, V = torch.zeros(B, Z, 1, A).bfloat16(), torch.zeros(B, 1, n, A).bfloat16(), torch.ones(B, 1, n, A).bfloat16()
    Q[..., 0, 0] = torch.from_numpy(rng.uniform(1, 16, (B, Z))).bfloat16()
    K[:, 0, 1:n - 1, 0], K[:, 0, n - 1, 0] = -30000.0, -1.0
    p = torch.exp(-Q[..., 0, 0].double() / 8)
    V[:, 0, 0] = torch.from_numpy(rng.uniform(0.5, 2, (B, A))).bfloat16()
    V[:, 0, n - 1] = (-V[:, 0, 0].double() / p[:, torch.arange(A) % Z]).bfloat16()
    P = torch.stack([torch.ones_like(p), p], -1)
    v = V[:, 0, [0, n - 1]].double()
    total = P.sum(-1, keepdim=True)
    return Q, K, V, (P @ v / total)[:, :, None].numpy(), (P @ v.abs() / total)[:, :, None].numpy()


@pytest.mark.parametrize("width", [1, 1000])            # whole segments; shares
@pytest.mark.parametrize("n", [2, 30, 40])
def test_probabilities_are_held_to_32_bits(n, width):
    """Scores (below 2) are exact, their products by the scale and log2(e) off by 4 roundings, exp by 2^-22: p is off by 2^-20 at
    most, and the sums of two that count by a rounding each; the result is rounded once."""
    Q, K, V, O, PV = cancelling(n)
    Kc, Vc, table, lengths = one_page(K, V, width)
    d = rsa.make_cache_desc(Kc, table, Q.shape[1])
    assert (rsa.cache_workspace_bytes(d) > 0) == (width == 1000)
    got, _ = rsa.cache_attend(d, Q.cuda(), Kc, Vc, table, lengths)
    assert (np.abs(O) < 2.0 ** -11 * PV).sum() > 500    # (many cancel)
    within(got, O, (2.0 ** -20 + 6 * F32) * PV + STEP["bf16"] * np.abs(O), "O")


@pytest.mark.parametrize("width", [1, 1000])
@pytest.mark.parametrize("sign", [1, -1])
def test_an_infinite_value_under_a_small_probability(width, sign):
    """Probabilities of 2^-125 to 2^-87 of the row's largest: fp32 holds them, so an infinite value is the result."""
    B, Z, A = 64, 16, 64
    rng = np.random.default_rng(33)
    Q, K, V = torch.zeros(B, Z, 1, A).bfloat16(), torch.zeros(B, 1, 30, A).bfloat16(), torch.ones(B, 1, 30, A).bfloat16()
    Q[..., 0, 0] = torch.from_numpy(rng.uniform(60, 87, (B, Z))).bfloat16()
    K[:, 0, 1, 0], K[:, 0, 2:, 0] = -1.0, -30000.0
    V[:, 0, 1, 5] = sign * float("inf")
    Kc, Vc, table, lengths = one_page(K, V, width)
    got, LSE = rsa.cache_attend(rsa.make_cache_desc(Kc, table, Z, scale=1.0), Q.cuda(), Kc, Vc, table, lengths)
    want = torch.ones(B, Z, 1, A).bfloat16()
    want[..., 5] = sign * float("inf")
    assert torch.equal(got.cpu(), want) and (LSE == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("level", [0.0, 12.0, -100.0, 1000.0, -30000.0])
def test_joined_weights_go_by_the_differences_alone(dtype, level):
    """Shares whose LSE lie around any level.  A weight exp(l - l') of a difference below D: the difference and its product by log2(e) are
    off by a rounding each, 2 D 2^-24 relative, exp by 2^-22; the running maximum moves three times at most, each another such
    factor of D and 2^-22.  The sums have N terms; LSE is rounded once more, and log adds 2^-22."""
    N, B, Z, A = 16, 40, 8, 64
    rng = np.random.default_rng(34)
    Op = torch.from_numpy(rng.standard_normal((N, B, Z, 1, A))).to(DTYPES[dtype])
    LSEp = torch.from_numpy(rng.standard_normal((N, B, Z, 1)) * 2 + level).float()
    O, LSE = oracle.join(f64(Op), f64(LSEp))
    D = float(LSEp.max(0).values.sub(LSEp.min(0).values).max())
    assert D < 16
    rel = 2 * 4 * (2 * D * F32 + 2.0 ** -22) + 2 * N * F32             # (of the weights and of their sum)
    w = np.exp(f64(LSEp) - LSE)
    size = (w[..., None] * np.abs(f64(Op))).sum(0)
    pool, table = torch.zeros(1, Z, 16, A, dtype=DTYPES[dtype], device="cuda"), torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    got = rsa.cache_join(rsa.make_cache_desc(pool, table, Z), Op.cuda(), LSEp.cuda())
    within(got[0], O, rel * size + STEP[dtype] * np.abs(O), "O")
    within(got[1], LSE, rel + 2.0 ** -22 + F32 * np.abs(LSE), "LSE")


@pytest.mark.parametrize("width", [1, 1000])
def test_a_large_value_under_a_small_probability(width):
    """Values of 2^120 under probabilities p of 2^-125 to 2^-87 of the row's largest, where they decide.  A score is a single product; p is off by
    4 roundings of its exponent and exp's 2^-22; its parts are multiples of 2^-133, one cut off and two that may be raised to it."""
    B, Z, A = 64, 16, 64
    rng = np.random.default_rng(35)
    Q, K, V = torch.zeros(B, Z, 1, A).bfloat16(), torch.zeros(B, 1, 30, A).bfloat16(), torch.ones(B, 1, 30, A).bfloat16()
    Q[..., 0, 0] = torch.from_numpy(rng.uniform(60, 87, (B, Z))).bfloat16()
    K[:, 0, 1, 0], K[:, 0, 2:, 0] = -1.0, -30000.0
    V[:, 0, 1, :8], V[:, 0, 1, 8:16] = 2.0 ** 120, -1.75 * 2.0 ** 120
    V[:, 0, 2:, 16:] = 2.0 ** 127                               # (under probabilities of 0: no part of any result)
    Kc, Vc, table, lengths = one_page(K, V, width)
    got, _ = rsa.cache_attend(rsa.make_cache_desc(Kc, table, Z, scale=1.0), Q.cuda(), Kc, Vc, table, lengths)
    p = torch.exp(-Q[..., 0].double())
    O = 1.0 + p[..., None] * (V[:, :1, 1:2].double() - 1)
    off = (4 * F32 * 87 + 2.0 ** -22) * p[..., None] + 3 * 2.0 ** -133
    bound = off * V[:, :1, 1:2].double().abs() + 8 * F32
    within(got, O.numpy(), bound.numpy() + STEP["bf16"] * O.abs().numpy(), "O")
