"""Caches in 8 bits and bounds of several new tokens at a time, shared by their tests."""
import numpy as np
import torch

from cache_helpers import DTYPES, Cache, attend_bounds, f64, within
from oracle import cache as oracle
from paper_2105_13120_amd import rsa


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Cache8:
    """A Cache's values in e4m3.  Where no sequence has a token the bytes are NaN and the exponents 255."""

    def __init__(self, rng, lengths, Zkv, A, page, width, dtype="bf16", scale=1.0, spare=2):
        c = Cache(rng, lengths, Zkv, A, page, width, dtype, scale, spare)
        self.page, self.width, self.lengths, self.table = page, width, c.lengths, c.table
        self.bytes, self.exps = [], []
        for pool in (c.Kc, c.Vc):
            x = f64(pool)
            held = np.isfinite(x).all(-1)
            byte, e = oracle.to_e4m3(np.where(held[..., None], x, 0.0))
            self.bytes.append(np.where(held[..., None], byte, 255))
            self.exps.append(np.where(held, e, 255))

    def value(self, i):
        return torch.from_numpy(oracle.from_e4m3(self.bytes[i]) * 2.0 ** (np.where(self.exps[i] == 255, 127, self.exps[i]) - 127.0)[..., None])

    @property
    def Kc(self):
        return self.value(0)

    @property
    def Vc(self):
        return self.value(1)

    def gpu(self):
        pools = [torch.from_numpy(b.astype(np.uint8)).cuda().view(torch.float8_e4m3fn) for b in self.bytes]
        return *pools, torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lengths).cuda()

    def scales(self):
        return dict(zip(("Ks", "Vs"), (torch.from_numpy(e.astype(np.uint8)).cuda() for e in self.exps)))


def scales_of(c):
    return c.scales() if isinstance(c, Cache8) else {}


def chunk(c, Q, counts=None, causal=True, scale=0.0, **kw):
    Kc, Vc, table, n = c.gpu()
    d = rsa.make_cache_desc(Kc, table, Q.shape[1], scale=scale)
    return rsa.cache_attend_chunk(d, Q.cuda(), Kc, Vc, table, n, None if counts is None else i32(counts), causal, **scales_of(c), **kw)


def chunk_bounds(Q, Kc, Vc, table, lengths, counts, causal, O, LSE, dtype, few, scale=None):
    """attend_bounds row by row.  Beyond 16 rows of a key head in bf16, probabilities are rounded to bf16 once: off by 2^-8 at most."""
    bO, bL = np.zeros(O.shape), np.zeros(LSE.shape)
    n = oracle.seen_by(table, lengths, Q.shape[2], counts, causal, Kc.shape[2])
    for t in range(Q.shape[2]):
        s = slice(t, t + 1)
        bO[:, :, s], bL[:, :, s] = attend_bounds(Q[:, :, s], Kc, Vc, table, n[:, t], O[:, :, s], LSE[:, :, s], dtype, scale)
        if dtype == "bf16" and not few:
            # sum p |v|: the attention with |v| for v
            bO[:, :, s] += 2.0 ** -8 * oracle.attend(Q[:, :, s], Kc, np.abs(Vc), table, n[:, t], scale)[0]
    return bO, bL


def compare_chunk(c, Q, got, dtype, counts=None, causal=True, scale=None):
    Kc, Vc = f64(c.Kc), f64(c.Vc)
    few = dtype == "f32" or Q.shape[1] // Kc.shape[1] * Q.shape[2] <= 16
    O, LSE = oracle.attend_chunk(f64(Q), Kc, Vc, c.table, c.lengths, counts, causal, scale)
    bO, bL = chunk_bounds(f64(Q), Kc, Vc, c.table, c.lengths, counts, causal, O, LSE, dtype, few, scale)
    within(got[0], O, bO, "O")
    within(got[1], LSE, bL, "LSE")


def vectorised_chunk(Q, Kc, Vc, table, lengths, counts, causal):
    """The definition in fp64 on the GPU, for caches that are too long for loops: O, LSE and sum p |v|.  Kc, Vc: values."""
    B, Z, T, A = Q.shape
    Zkv, page = Kc.shape[1:3]
    O, PV = (torch.zeros(Q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    LSE = torch.full((B, Z, T), -float("inf"), dtype=torch.float64, device="cuda")
    for b in range(B):
        n, k = int(lengths[b]), T if counts is None else int(counts[b])
        if n < 1 or k < 1:
            continue
        rows = table[b, :-(-n // page)].long()
        K, V = (x[rows].transpose(0, 1).reshape(Zkv, -1, A)[:, :n].double() for x in (Kc, Vc))
        hidden = torch.arange(n, device="cuda")[None] > torch.arange(n - k, n, device="cuda")[:, None] if causal else torch.zeros(k, n, dtype=torch.bool, device="cuda")
        for z in range(Z):
            S = (Q[b, z, :k].double() @ K[z * Zkv // Z].T / A ** 0.5).masked_fill(hidden, -float("inf"))
            P = S.softmax(-1).nan_to_num(0.0)
            LSE[b, z, :k], O[b, z, :k], PV[b, z, :k] = S.logsumexp(-1), P @ V[z * Zkv // Z], P @ V[z * Zkv // Z].abs()
    return O, LSE, PV
