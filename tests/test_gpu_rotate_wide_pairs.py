"""Rotation of heads of 192, which leave lanes of every wave without a row, in pairs that are no whole 16 bytes."""
import numpy as np
import pytest
import torch

from cache_helpers import f64, frequencies, normal, rotated_bound, within
from oracle import cache as oracle
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,adjacent", [(66, False), (130, False), (182, False), (190, False), (130, True), (190, True)])
@pytest.mark.parametrize("back", [False, True])
def test_heads_of_192(dtype, R, adjacent, back):
    rng = np.random.default_rng(40)
    B, Z, L, A = 2, 3, 128, 192
    X, f = normal(rng, (B, Z, L, A), dtype), frequencies(R)
    d = rsa.make_desc(X, 2, mode=rsa.MODE_STAGED)
    turn = rsa.rotate_bwd if back else rsa.rotate
    Y = turn(d, f.cuda(), X.cuda(), adjacent=adjacent)[0]
    ref = oracle.rotate(f64(X), np.arange(L), f.numpy(), adjacent, back)
    within(Y, ref, rotated_bound(f64(X), ref, R, adjacent, dtype), "Y")
    assert torch.equal(Y.cpu()[..., R:], X[..., R:])
    into = X.cuda()
    turn(d, f.cuda(), into, None, into, adjacent=adjacent)
    assert torch.equal(into, Y)
