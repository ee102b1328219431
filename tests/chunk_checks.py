"""A call on several new tokens against its definition in 64 bits, for caches that are too long for loops."""
import torch

from cache8_helpers import i32, vectorised_chunk
from cache_helpers import DTYPES, F32, STEP, f64, within
from paper_2105_13120_amd import rsa

BEHIND = 1 << 16      # bytes behind a workspace


def check(dtype, Z, Zkv, A, page, T, lengths, counts=None, causal=True, eight=False, all_bits=False, seed=0):
    """all_bits: whether probabilities weigh values with all their 24 bits (off by 2^-15 as a sum of two bf16 numbers would be, which
    leaves room for the three that there are), or rounded to bf16 once (2^-8).  The rest is as in attend_bounds, with |q| |k| of these
    inputs for the sum of products (powers up to 4 in 8 bits)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, W = len(lengths), -(-max(lengths) // page)
    Kc, Vc = (torch.randn(B * W, Zkv, page, A, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    table = torch.randperm(B * W, generator=g, device="cuda").reshape(B, W).to(torch.int32)
    Q = torch.randn(B, Z, T, A, generator=g, device="cuda").to(DTYPES[dtype])
    pools, kw = (Kc, Vc), {}
    if eight:                     # powers of two of their own per row, the numbers e4m3's
        e = torch.randint(-3, 3, (2, B * W, Zkv, page), generator=g, device="cuda")
        pools = [x.to(torch.float8_e4m3fn) for x in pools]
        kw = dict(zip(("Ks", "Vs"), (e + 127).to(torch.uint8)))
        two = torch.tensor([2.0 ** k for k in range(-3, 3)], device="cuda")
        Kc, Vc = (x.float() * two[k + 3][..., None] for x, k in zip(pools, e))
    d = rsa.make_cache_desc(pools[0], table, Z)
    need = rsa.cache_chunk_workspace_bytes(d, T)
    memory = torch.full((need + BEHIND,), 0xFF, dtype=torch.uint8, device="cuda")
    O, LSE = rsa.cache_attend_chunk(d, Q, *pools, table, i32(lengths), None if counts is None else i32(counts), causal, ws=memory[:need] if need else None, **kw)
    assert (memory[need:] == 0xFF).all()
    rO, rLSE, PV = vectorised_chunk(Q, Kc, Vc, table, lengths, counts, causal)
    rel = 2 * (A + 4) * F32 * A ** 0.5 * (24 if eight else 6) + 2.0 ** -21 + 2 * max(lengths) * F32
    bound = (rel + (0.0 if dtype == "f32" else 2.0 ** -15 if all_bits else 2.0 ** -8)) * PV + STEP[dtype] * rO.abs()
    within(O, f64(rO), f64(bound), "O")
    finite = f64(rLSE)
    within(LSE, finite, rel + 4 * F32 * abs(finite), "LSE")
