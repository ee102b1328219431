"""Angles next to where a cosine or a sine is 0: pairs (1, 0) and (0, 1) turned, which are the cosine and the sine themselves."""
import numpy as np
import pytest
import torch

from cache_helpers import F32, f64
from oracle import cache as oracle
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", ["rows", "cache"])
def test_cosines_and_sines_to_their_last_bits(path):
    """Frequencies of quarter turns and a little, so that positions lie around multiples of them: every cosine and sine is right relative to its own
    size, 4 units of the last place (the functions' bound, 2^-21 of the value), and 2^-23 of it for the rounded angle's rest; 2^-48 where it
    is 0 to fp64."""
    A, L = 64, 1024
    quarter = np.arctan2(1.0, 0.0)
    f = torch.from_numpy(np.concatenate([quarter * (1 + np.arange(16)), quarter + 10.0 ** -np.arange(4.0, 12.0), quarter / (1 + np.arange(8))])).float()
    X = torch.zeros(1, 2, L, A)
    X[:, 0, :, :A // 2] = 1.0
    X[:, 1, :, A // 2:] = 1.0
    if path == "rows":
        Y = rsa.rotate(rsa.make_desc(X, 1, mode=rsa.MODE_STAGED), f.cuda(), K=X.cuda())[1]
    else:
        pool = torch.zeros(1, 2, L, A, device="cuda")
        one = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
        Y = torch.zeros_like(pool)
        rsa.cache_append(rsa.make_cache_desc(pool, one, 2), X.cuda(), X.cuda(), Y, pool, one, one[0] + L, inv_freq=f.cuda())
    ref = oracle.rotate(f64(X), np.arange(L), f.numpy())
    err = np.abs(f64(Y) - ref)
    assert (np.abs(ref) < 1e-6).sum() > 100
    bad = err > (2.0 ** -21 + 2 * F32) * np.abs(ref) + 2.0 ** -48
    assert not bad.any(), (bad.sum(), f64(Y)[bad][:4], ref[bad][:4])
