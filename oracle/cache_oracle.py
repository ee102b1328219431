"""fp64 oracle of rotation by position and of the paged cache.  Test infrastructure only.

Rotation: the pairs of a head's first R elements are complex numbers, times exp(i angle); angle = position * inv_freq,
in longdouble before its cosine and sine are taken.  Cache: slot s of sequence b is place s % page of page table[b][s / page];
written and read token by token.  Nothing here is shared with the HIP path.
"""
import numpy as np

TWO_PI = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))


def rotate(x, pos, inv_freq, adjacent=False, back=False):
    """x (..., rows, A), pos (rows,)."""
    x = np.asarray(x, dtype=np.float64)
    R = 2 * len(inv_freq)
    angle = np.asarray(pos, np.longdouble)[:, None] * np.asarray(inv_freq, np.float32).astype(np.longdouble)[None]
    angle = np.remainder(angle, TWO_PI).astype(np.float64)
    turn = np.exp((-1j if back else 1j) * angle)
    y = x.copy()
    re, im = (slice(0, R, 2), slice(1, R, 2)) if adjacent else (slice(0, R // 2), slice(R // 2, R))
    z = (x[..., re] + 1j * x[..., im]) * turn
    y[..., re], y[..., im] = z.real, z.imag
    return y


def tokens(L, N, begin, end, zigzag=False):
    """The tokens of the rows that ranks [begin, end) own, in the order of the rows."""
    c = L // N
    if not zigzag:
        return np.arange(begin * c, end * c)
    h = c // 2
    return np.concatenate([np.arange(k * h, (k + 1) * h) for n in range(begin, end) for k in (n, 2 * N - 1 - n)])


def place(table, b, slot, pages, page):
    """(page, place) of a slot, None where it is not held."""
    if slot < 0 or slot >= table.shape[1] * page:
        return None
    p = int(table[b, slot // page])
    return (p, slot % page) if 0 <= p < pages else None


def append(K, V, Kc, Vc, table, lengths, counts=None, first=None, inv_freq=None, adjacent=False, Q=None, Qr=None):
    """Returns (Qr, Kc, Vc); Qr starts from the given one."""
    Kc, Vc = np.array(Kc, np.float64), np.array(Vc, np.float64)
    pages, _, page, _ = Kc.shape
    B, _, T, _ = K.shape
    Qr = None if Q is None else np.array(Q if Qr is None else Qr, np.float64)
    for b in range(B):
        count = T if counts is None else min(T, int(counts[b]))
        for t in range(count):
            slot = int(lengths[b]) - count + t
            pos = np.array([slot + (0 if first is None else int(first[b]))])

            def turned(x):
                x = np.asarray(x[b, :, t], np.float64)[:, None]
                return (x if inv_freq is None else rotate(x, pos, inv_freq, adjacent))[:, 0]
            if Q is not None:
                Qr[b, :, t] = turned(Q)
            at = place(table, b, slot, pages, page)
            if at is not None:
                Kc[at[0], :, at[1]] = turned(K)
                Vc[at[0], :, at[1]] = V[b, :, t]
    return Qr, Kc, Vc


def attend(Q, Kc, Vc, table, lengths, scale=None):
    """Q (B, Z, 1, A) -> O (B, Z, 1, A), LSE (B, Z, 1)."""
    Q = np.asarray(Q, np.float64)
    B, Z, _, A = Q.shape
    pages, Zkv, page, _ = Kc.shape
    s = 1.0 / np.sqrt(A) if scale is None else scale
    O, LSE = np.zeros(Q.shape), np.full((B, Z, 1), -np.inf)
    for b in range(B):
        at = [place(table, b, j, pages, page) for j in range(min(int(lengths[b]), table.shape[1] * page))]
        at = [p for p in at if p is not None]
        if not at:
            continue
        rows = [p[0] for p in at], [p[1] for p in at]
        for z in range(Z):
            h = z * Zkv // Z
            k, v = (np.asarray(c[rows[0], h, rows[1]], np.float64) for c in (Kc, Vc))
            S = k @ Q[b, z, 0] * s
            p = np.exp(S - S.max())
            O[b, z, 0] = p @ v / p.sum()
            LSE[b, z, 0] = np.log(p.sum()) + S.max()
    return O, LSE


def join(Op, LSEp):
    """(N, ...) shares -> O, LSE."""
    Op, LSEp = np.asarray(Op, np.float64), np.asarray(LSEp, np.float64)
    m = LSEp.max(0)
    ref = np.where(np.isneginf(m), 0.0, m)
    w = np.exp(LSEp - ref)
    total = w.sum(0)
    with np.errstate(divide="ignore"):
        LSE = np.log(total) + ref
    part = np.where(w[..., None] > 0, Op, 0.0) * w[..., None]
    return part.sum(0) / np.where(total > 0, total, 1.0)[..., None], LSE


# ---- the cache in 8 bits ----
# What the 127 bytes from 0 up to the largest number of e4m3 stand for, in ascending order: four bits of an exponent, three of a fraction.
E4M3 = np.array([(b & 7) * 2.0 ** -9 if b < 8 else (8 + (b & 7)) * 2.0 ** ((b >> 3) - 10) for b in range(127)])


def from_e4m3(byte):
    byte = np.asarray(byte, np.int64)
    v = np.append(E4M3, np.nan)[byte & 127]
    return np.where(byte & 128, -v, v)


def to_e4m3(x):
    """Rows (..., A) -> bytes, and the rows' exponents + 127: the least power of two, from 2^-64 on, under which no finite element
    passes 448, and the nearest number, of two the one with an even byte."""
    x = np.asarray(x, np.float64)
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(top.shape, -64)
    while (top > 448.0 * 2.0 ** e).any():
        e += top > 448.0 * 2.0 ** e
    y = np.abs(x) / 2.0 ** e[..., None]
    hi = np.clip(np.searchsorted(E4M3, np.nan_to_num(y)), 1, 126)
    below, above = y - E4M3[hi - 1], E4M3[hi] - y
    byte = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, hi - 1)
    byte = np.where(np.isfinite(x), byte, 127)
    return np.where(np.signbit(x) & np.isfinite(x), byte + 128, byte), e + 127


def append8(K, V, Kc, Vc, Ks, Vs, table, lengths, counts=None, first=None, inv_freq=None, adjacent=False, Q=None, Qr=None):
    """... to pools of bytes with exponents.  Returns (Qr, Kc, Vc, Ks, Vs)."""
    Kc, Vc, Ks, Vs = (np.array(x, np.int64) for x in (Kc, Vc, Ks, Vs))
    pages, _, page, _ = Kc.shape
    T = K.shape[2]
    mark = np.full(Kc.shape, np.nan)
    Qr, turned, moved = append(K, V, mark, mark, table, lengths, counts, first, inv_freq, adjacent, Q, Qr)
    for b in range(len(lengths)):
        count = T if counts is None else min(T, int(counts[b]))
        for slot in range(int(lengths[b]) - count, int(lengths[b])):
            at = place(table, b, slot, pages, page)
            if at is not None:
                Kc[at[0], :, at[1]], Ks[at[0], :, at[1]] = to_e4m3(turned[at[0], :, at[1]])
                Vc[at[0], :, at[1]], Vs[at[0], :, at[1]] = to_e4m3(moved[at[0], :, at[1]])
    return Qr, Kc, Vc, Ks, Vs


def read(pool, table, lengths, T, counts=None, start=None):
    """The last tokens of every sequence, (B, Zkv, T, A); rows of no token from the given ones (zero)."""
    pages, Zkv, page, A = pool.shape
    out = np.zeros((len(lengths), Zkv, T, A)) if start is None else np.array(start, np.float64)
    for b in range(len(lengths)):
        count = T if counts is None else min(T, int(counts[b]))
        for t in range(count):
            at = place(table, b, int(lengths[b]) - count + t, pages, page)
            out[b, :, t] = 0.0 if at is None else pool[at[0], :, at[1]]
    return out


# ---- several new tokens at a time ----
def seen_by(table, lengths, T, counts, causal, page):
    """Slots that token t of sequence b sees (from 0 on, those that are not held among them), -1 for a token that is not there."""
    n = np.full((len(lengths), T), -1)
    for b in range(len(lengths)):
        count = T if counts is None else max(0, min(T, int(counts[b])))
        most = max(0, min(int(lengths[b]), table.shape[1] * page))
        for t in range(count):
            n[b, t] = most if not causal else max(0, min(int(lengths[b]) - count + t + 1, most))
    return n


def attend_chunk(Q, Kc, Vc, table, lengths, counts=None, causal=True, scale=None):
    """Q (B, Z, T, A) -> O, LSE (B, Z, T), token by token; 0 and -inf for tokens that are not there."""
    Q = np.asarray(Q, np.float64)
    O, LSE = np.zeros(Q.shape), np.full(Q.shape[:3], -np.inf)
    n = seen_by(table, lengths, Q.shape[2], counts, causal, Kc.shape[2])
    for t in range(Q.shape[2]):
        O[:, :, t:t + 1], LSE[:, :, t:t + 1] = attend(Q[:, :, t:t + 1], Kc, Vc, table, n[:, t], scale)
    return O, LSE
