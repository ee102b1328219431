"""Inputs and bounds shared by the tests of rotation by position and of the paged cache."""
import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# a rounding: half a step relative to the value
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
F32 = 2.0 ** -24


def frequencies(R, base=10000.0):
    return torch.tensor(base ** (-2.0 * np.arange(R // 2) / R), dtype=torch.float32)


def normal(rng, shape, dtype, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(DTYPES[dtype])


def f64(t):
    return t.detach().cpu().double().numpy()


def rotated_bound(x, ref, R, adjacent, dtype):
    """The stored value's rounding, and fp32 before it: cosine and sine err by at most 2^-22 (the angle's fraction of a turn is
    rounded once, the functions themselves by two units), products and their sum by 2^-23, together 2^-21 of |x0| + |x1|.
    Elements from R on are copies."""
    a = np.abs(x)
    y = np.zeros_like(a)
    if adjacent:
        s = a[..., 0:R:2] + a[..., 1:R:2]
        y[..., 0:R:2] = y[..., 1:R:2] = s
    else:
        s = a[..., :R // 2] + a[..., R // 2:R]
        y[..., :R // 2] = y[..., R // 2:R] = s
    out = STEP[dtype] * np.abs(ref) + 2.0 ** -21 * y
    out[..., R:] = 0.0
    return out


def attend_bounds(Q, Kc, Vc, table, lengths, O, LSE, dtype, scale=None):
    """Bounds of |O| and |LSE| errors against fp64, from the definition.  A score is a sum of A products in fp32, off by at most
    dS = (A + 4) 2^-24 s sum|q k| (the scale and the exponent's argument are the 4); exp adds 2^-22, so probabilities are off by
    2 dS + 2^-21 relative to their normalised value, and n terms' sum by n 2^-24 at most.  In bf16 the probabilities that
    weigh V may be two bf16 numbers each, eight bits and what they leave, rounded: off by 2^-15.  The stored O is rounded once."""
    B, Z, _, A = Q.shape
    pages, Zkv, page, _ = Kc.shape
    s = 1.0 / np.sqrt(A) if scale is None else scale
    bO, bL = np.zeros(O.shape), np.zeros(LSE.shape)
    for b in range(B):
        at = [(int(table[b, j // page]), j % page) for j in range(max(0, min(int(lengths[b]), table.shape[1] * page)))]
        at = [p for p in at if 0 <= p[0] < pages]
        if not at:
            continue
        rows = [p[0] for p in at], [p[1] for p in at]
        n = len(at)
        for z in range(Z):
            h = z * Zkv // Z
            k, v = Kc[rows[0], h, rows[1]], Vc[rows[0], h, rows[1]]
            P = np.exp(k @ Q[b, z, 0] * s - LSE[b, z, 0])
            dS = (A + 4) * F32 * s * (np.abs(k) @ np.abs(Q[b, z, 0]))
            rel = 2 * dS.max() + 2.0 ** -21 + 2 * n * F32
            bL[b, z, 0] = rel + 4 * F32 * np.abs(LSE[b, z, 0])
            bO[b, z, 0] = rel * (P @ np.abs(v)) + STEP[dtype] * np.abs(O[b, z, 0])
            if dtype == "bf16":
                bO[b, z, 0] += 2.0 ** -15 * (P @ np.abs(v))
    return bO, bL


def within(got, ref, bound, what):
    with np.errstate(invalid="ignore"):              # (-inf for -inf)
        err = np.abs(f64(got) - ref)
    same = np.isneginf(ref) & np.isneginf(f64(got))
    bad = ~(same | (err <= bound))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} elements off, the first at {tuple(np.argwhere(bad)[0])}: " \
        f"{f64(got)[bad][0]} for {ref[bad][0]}, allowed {np.broadcast_to(bound, bad.shape)[bad][0]}"


class Cache:
    """Pools full of NaN, a table of random pages for sequences of the given lengths, and values in the slots."""

    def __init__(self, rng, lengths, Zkv, A, page, width, dtype, scale=1.0, spare=2, junk=float("nan")):
        B = len(lengths)
        self.page, self.width, self.lengths = page, width, np.array(lengths, np.int32)
        held = [-(-max(0, min(int(n), width * page)) // page) for n in lengths]
        pages = sum(held) + spare
        order = list(rng.permutation(pages))
        self.table = np.full((B, width), -1, np.int32)
        self.Kc = torch.full((pages, Zkv, page, A), junk, dtype=DTYPES[dtype])
        self.Vc = self.Kc.clone()
        for b, n in enumerate(lengths):
            n = max(0, min(int(n), width * page))
            for i in range(held[b]):
                p = self.table[b, i] = order.pop()
                fill = min(page, n - i * page)
                self.Kc[p, :, :fill] = normal(rng, (Zkv, fill, A), dtype, scale)
                self.Vc[p, :, :fill] = normal(rng, (Zkv, fill, A), dtype)

    def gpu(self):
        return self.Kc.cuda(), self.Vc.cuda(), torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lengths).cuda()
