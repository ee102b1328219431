"""Serving in chunks and in 8 bits as timed cases: a paged cache in e4m3, reading it back, attention of several new tokens at a time.

A case is a dict of plain values; `prepare` makes what a user's program holds before the call, `run` is one pass: the
operators written out in elementary torch operations or, where `own` is true, the calls of `paper_2105_13120_amd.rsa`.

Kinds:
  store   keys and values of new tokens into their pages in e4m3, a power of two per row, then read back
  read    the last tokens of every sequence out of their pages, as dense tensors
  attend  one new token per sequence over the pages of its sequence, in e4m3
  chunk   several new tokens per sequence over the pages of its sequence, in the queries' type or in e4m3
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST_POOL = 64 * 8192 * 8 * 128      # elements of a cache's keys: no more than the largest listed one
MOST_SCORES = 1 << 32                # of the plain form, padding among them
E4M3_MOST, LEAST_SCALE, MOST_SCALE = 448.0, -64, 120


def case(name, kind, **kw):
    c = dict(name=name, kind=kind, dtype="bf16", e4m3=True, B=1, Z=16, Zkv=16, A=64, page=16, length=512, T=1, ragged=True, order=0)
    if kind == "store":
        c.update(R=64, adjacent=False, rank_share=False)
    if kind in ("store", "chunk"):
        c["packed"] = False
    if kind in ("attend", "chunk"):
        c.update(std=1.0, empty=False)
    if kind != "store":
        c["holes"] = False
    if kind == "chunk":
        c["causal"] = True
    c.update(kw)
    return c


def listed():
    return [
        # one token of each of 64 sequences, as a decoding step writes it
        case("store_decode_64", "store", B=64, Z=32, Zkv=8, A=128, R=128, length=1024),
        # prompts of uneven lengths, read back for whoever works on them next
        case("store_prompts_8x2k", "store", B=8, Z=32, Zkv=8, A=128, R=128, length=2048, T=2048, page=64),
        # one sequence's last tokens in 32 bits, odd pages
        case("read_f32_500", "read", dtype="f32", e4m3=False, B=3, Z=12, Zkv=12, length=700, T=500, page=24),
        # whole caches handed on to another rank or another layout
        case("read_handover_4x32k", "read", B=4, Z=32, Zkv=8, A=128, length=32768, T=32768, page=64),
        # one short sequence, all heads their own keys
        case("attend_e4m3_small_300", "attend", length=300),
        # a batch of chats of uneven lengths, four queries a key head
        case("attend_e4m3_serving_64", "attend", B=64, Z=32, Zkv=8, A=128, length=8192),
        # one document, split over its length
        case("attend_e4m3_long_128k", "attend", Z=32, Zkv=8, A=128, length=131072, ragged=False, page=64),
        # four guessed tokens of each of 16 sequences, checked at once
        case("chunk_guesses_16x4", "chunk", e4m3=False, B=16, Z=32, Zkv=8, A=128, length=4096, T=4),
        # prompts of uneven lengths, queries as slices of one projection output
        case("chunk_prompts_8x2k", "chunk", e4m3=False, B=8, Z=32, Zkv=8, A=128, length=2048, T=2048, page=64, packed=True),
        # the next piece of one long prompt
        case("chunk_2k_of_64k", "chunk", e4m3=False, Z=32, Zkv=8, A=128, length=65536, T=2048, ragged=False, page=64),
        # pieces of prompts over caches in 8 bits
        case("chunk_e4m3_512_of_16k", "chunk", B=8, Z=32, Zkv=8, A=128, length=16384, T=512),
        # in 32 bits, odd pages, an odd number of tokens
        case("chunk_f32_37_of_1k", "chunk", dtype="f32", e4m3=False, B=4, Z=12, Zkv=12, length=1000, T=37, page=24),
    ]


def spread(rng, lo, hi):
    """A size between lo and hi, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choices(["store", "read", "attend", "chunk"], [3, 1, 3, 5])[0]
        dtype = "f32" if kind in ("read", "chunk") and rng.random() < 0.25 else "bf16"
        e4m3 = dtype == "bf16" and (kind in ("store", "attend") or rng.random() < 0.5)
        Zkv, A, length = rng.randint(1, 16), rng.choice([64, 64, 128, 128, 192, 256]), spread(rng, 1, 131072)
        c = case("", kind, dtype=dtype, e4m3=e4m3, B=spread(rng, 1, 128), Z=Zkv * rng.choice([1, 1, 2, 3, 4, 5, 8, 16, 24]), Zkv=Zkv, A=A,
                 page=rng.choice([1, 16, 16, 24, 32, 64, 64, 100, 128, 256]), length=length, ragged=rng.random() < 0.7,
                 order=rng.randrange(1 << 30))
        if kind == "store":
            c.update(T=1 if rng.random() < 0.5 else spread(rng, 1, min(4096, length)), R=rng.choice([0, A, A, A // 2, 20]),
                     adjacent=rng.random() < 0.4, rank_share=rng.random() < 0.2, packed=rng.random() < 0.3)
        elif kind == "read":
            c.update(T=spread(rng, 1, length), holes=rng.random() < 0.2)
        else:
            c.update(holes=rng.random() < 0.2, empty=rng.random() < 0.2, std=rng.choice([0.5, 1.0, 2.0]))
            if kind == "chunk":
                c.update(T=spread(rng, 1, min(4096, length)), causal=rng.random() < 0.8, packed=rng.random() < 0.3)
        c.pop("name")
        if affordable(c):
            return c


def affordable(c):
    """Not the work of more than any listed case, and plain forms that fit the memory."""
    pool = c["B"] * padded(c) * c["Zkv"] * c["A"]
    if c["Z"] > 64 or pool > MOST_POOL // (2 if c["dtype"] == "f32" else 1) or (c["kind"] == "store" and pool > MOST_POOL // 8):
        return False
    if c["kind"] == "chunk" and c["B"] * c["Z"] * c["T"] * padded(c) > MOST_SCORES:
        return False
    return all(work(c)[k] <= max(work(x)[k] for x in listed()) for k in ("bytes", "flops"))


# --------------------------------------------------------------------------- sizes and work
def width(c):
    return -(-c["length"] // c["page"])


def padded(c):
    return width(c) * c["page"]


def lengths_of(c):
    """Tokens of each sequence, the new ones among them: part of the case, not of its inputs."""
    r = random.Random(c["order"])
    n = [c["length"]] * c["B"]
    if c["ragged"]:
        n = [c["length"] if b == 0 else spread(r, max(1, c["length"] // 16), c["length"]) for b in range(c["B"])]
    if c.get("empty"):
        n = [0 if r.random() < 0.3 else x for x in n]
    return n


def counts_of(c):
    """New tokens of each sequence: pieces of prompts are uneven too."""
    return [min(c["T"], n) for n in lengths_of(c)]


def missing_of(c):
    """Pages at the front of each sequence that are no longer held."""
    if not c.get("holes"):
        return [0] * c["B"]
    return [(n // c["page"]) // 2 for n in lengths_of(c)]


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    lengths, counts, gone = lengths_of(c), counts_of(c), [m * c["page"] for m in missing_of(c)]
    row = c["A"] + 1 if c["e4m3"] else c["A"] * es      # a stored row of keys or values, its scale among it
    new = sum(counts)
    if c["kind"] == "store":
        data = (2 * c["Z"] + 2 * c["Zkv"]) * c["A"] * es + 2 * c["Zkv"] * row           # queries in and out, keys and values in, and stored
        back = 2 * c["Zkv"] * (row + c["A"] * es)
        return {"bytes": new * (data + back), "flops": 3 * new * (c["Z"] + c["Zkv"]) * c["R"]}
    if c["kind"] == "read":
        held = sum(min(k, max(0, n - m)) for k, n, m in zip(counts, lengths, gone))
        return {"bytes": 2 * c["Zkv"] * (held * row + new * c["A"] * es), "flops": held * 2 * c["Zkv"] * c["A"]}
    seen = sum(max(0, n - m) for n, m in zip(lengths, gone))
    if c["kind"] == "attend":
        rows, pairs = c["B"] * c["Z"], seen * c["Z"]
    else:
        rows, pairs = new * c["Z"], 0
        for k, n, m in zip(counts, lengths, gone):      # token t sees slots m .. n - k + t, or all from m on
            first = max(n - k, m)
            pairs += c["Z"] * ((n - first) * (n - first + 1) // 2 + (n - first) * (first - m) if c["causal"] else k * max(0, n - m))
    return {"bytes": 2 * seen * c["Zkv"] * row + rows * (2 * c["A"] * es + 4), "flops": 4 * pairs * c["A"]}


# --------------------------------------------------------------------------- inputs
def frequencies(R, device="cuda"):
    i = torch.arange(R // 2, device=device, dtype=torch.float64)
    return (10000.0 ** (-2.0 * i / max(R, 1))).float()


def power(e, dtype=torch.float64):
    """2^e by its bits (functions of the GPU round powers of two)."""
    if dtype == torch.float64:
        return ((e.long() + 1023) << 52).view(torch.float64)
    return ((e.int() + 127) << 23).view(torch.float32)


def filled(x):
    """A pool's values in e4m3 and the exponents of its rows, as an earlier call has left them."""
    e = torch.frexp(x.float().abs().amax(-1) / E4M3_MOST).exponent
    q = x.float() * power(-e, torch.float32)[..., None]
    return q.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPES[c["dtype"]]

    def normal(*shape, std=1.0):
        x = torch.empty(shape, device="cuda", dtype=dt).normal_(generator=g)
        return x.mul_(std) if std != 1.0 else x

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    B, Z, Zkv, A, W, T = (c["B"], c["Z"], c["Zkv"], c["A"], width(c), c["T"])
    pages = B * W + 3
    s = dict(case=c, Kc=normal(pages, Zkv, c["page"], A), Vc=normal(pages, Zkv, c["page"], A), Ks=None, Vs=None, O=None,
             table=torch.randperm(pages, generator=g, device="cuda")[:B * W].reshape(B, W).to(torch.int32),
             lengths=ints(lengths_of(c)), counts=None if T == 1 else ints(counts_of(c)))
    if c["e4m3"]:
        s["Kc"], s["Ks"] = filled(s["Kc"])
        s["Vc"], s["Vs"] = filled(s["Vc"])
    if c["kind"] == "store":
        if c["packed"]:      # slices of one projection output
            x = normal(B, T, Z + 2 * Zkv, A).permute(0, 2, 1, 3)
            s["Q"], s["K"], s["V"] = x[:, :Z], x[:, Z:Z + Zkv], x[:, Z + Zkv:]
            s["Qr"] = torch.zeros(B, T, Z + 2 * Zkv, A, dtype=dt, device="cuda").permute(0, 2, 1, 3)[:, :Z]
        else:
            s["Q"], s["K"], s["V"] = normal(B, Z, T, A), normal(B, Zkv, T, A), normal(B, Zkv, T, A)
            s["Qr"] = torch.zeros_like(s["Q"])       # (rows of no token stay as they are)
        s["first"] = ints([1000 * b for b in range(B)]) if c["rank_share"] else None
        s["inv_freq"] = frequencies(c["R"]) if c["R"] else None
    else:
        s["table"][torch.arange(W, device="cuda")[None] < ints(missing_of(c))[:, None]] = -1
    if c["kind"] == "attend":
        s["Q"] = normal(B, Z, 1, A, std=c["std"])
    if c["kind"] == "chunk":
        if c["packed"]:
            s["Q"] = normal(B, T, Z + 2 * Zkv, A, std=c["std"]).permute(0, 2, 1, 3)[:, :Z]
            s["O"] = torch.zeros(B, T, Z, A, dtype=dt, device="cuda").permute(0, 2, 1, 3)
        else:
            s["Q"] = normal(B, Z, T, A, std=c["std"])
    if own:
        from paper_2105_13120_amd import rsa
        s["desc"] = rsa.make_cache_desc(s["Kc"], s["table"], Z, Q=s.get("Q"), K=s.get("K"), O=s["O"])
    return s


# --------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return run_own(state)
    return {"store": plain_store, "read": plain_read, "attend": plain_attend, "chunk": plain_attend}[state["case"]["kind"]](state)


def run_own(s):
    from paper_2105_13120_amd import rsa
    c, d = s["case"], s["desc"]
    pools, scales = (s["Kc"], s["Vc"], s["table"], s["lengths"]), dict(Ks=s["Ks"], Vs=s["Vs"])
    if c["kind"] == "store":
        Qr = rsa.cache_append(d, s["K"], s["V"], *pools, counts=s["counts"], first=s["first"], inv_freq=s["inv_freq"],
                              adjacent=c["adjacent"], Q=s["Q"], Qr=s["Qr"], **scales)
        return [Qr, *rsa.cache_read(d, c["T"], *pools, counts=s["counts"], **scales)]
    if c["kind"] == "read":
        return rsa.cache_read(d, c["T"], *pools, counts=s["counts"], **scales)
    if c["kind"] == "attend":
        return rsa.cache_attend(d, s["Q"], *pools, **scales)
    return rsa.cache_attend_chunk(d, s["Q"], *pools, counts=s["counts"], causal=c["causal"], O=s["O"], **scales)


def turned(x, pos, inv_freq, adjacent):
    """x (..., rows, A), rotated by the rows' positions in 64 bits: what is stored in e4m3 next to a border goes by them."""
    y = x.double()
    if inv_freq is None:
        return y
    R = 2 * inv_freq.numel()
    angle = pos.double()[..., None] * inv_freq.double()
    cos, sin = angle.cos(), angle.sin()
    y = y.clone()
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if adjacent else (y[..., :R // 2], y[..., R // 2:R])
    p, q = a * cos - b * sin, b * cos + a * sin
    a.copy_(p)
    b.copy_(q)
    return y


def quantised(x):
    """e4m3 times the least power of two under which no element passes 448; ties go to the even neighbour."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.frexp(top / E4M3_MOST).exponent
    e = torch.where(top <= E4M3_MOST * power(e - 1), e - 1, e).clamp(LEAST_SCALE, MOST_SCALE)
    y = x * power(-e)
    step = torch.clamp(torch.frexp(y).exponent - 1, min=-6) - 3
    q = torch.round(y * power(-step)) * power(step)
    return q.to(torch.float8_e4m3fn), (e[..., 0] + 127).to(torch.uint8)


def values(pool, scale):
    """What a pool's rows stand for, in 32 bits."""
    return pool.float() if scale is None else pool.float() * power(scale.int() - 127, torch.float32)[..., None]


def new_slots(s):
    """Slots of the call's tokens (B, T), and which of them are there."""
    c = s["case"]
    lengths = s["lengths"].long()
    counts = torch.full_like(lengths, c["T"]) if s["counts"] is None else s["counts"].long()
    t = torch.arange(c["T"], device="cuda")[None]
    return (lengths - counts)[:, None] + t, t < counts[:, None]


def plain_store(s):
    c = s["case"]
    page = c["page"]
    slot, there = new_slots(s)
    pos = (slot if s["first"] is None else slot + s["first"].long()[:, None])[:, None]
    there = there & (slot >= 0) & (slot < s["table"].shape[1] * page)
    b, t = there.nonzero(as_tuple=True)
    at = slot[b, t]
    where = s["table"].long()[b, at // page]
    q, e = quantised(turned(s["K"], pos, s["inv_freq"], c["adjacent"]))
    s["Kc"].view(torch.uint8)[where, :, at % page] = q.view(torch.uint8)[b, :, t]
    s["Ks"][where, :, at % page] = e[b, :, t]
    q, e = quantised(s["V"].double())
    s["Vc"].view(torch.uint8)[where, :, at % page] = q.view(torch.uint8)[b, :, t]
    s["Vs"][where, :, at % page] = e[b, :, t]
    Q = turned(s["Q"], pos, s["inv_freq"], c["adjacent"])
    s["Qr"].copy_(torch.where(there[:, None, :, None], Q.to(s["Qr"].dtype), s["Qr"]))
    return [s["Qr"], *plain_read(s)]


def plain_read(s):
    c = s["case"]
    B, Zkv, A, page = c["B"], c["Zkv"], c["A"], c["page"]
    slot, there = new_slots(s)
    there = there & (slot >= 0) & (slot < s["table"].shape[1] * page)
    at = slot.clamp(0, s["table"].shape[1] * page - 1)
    where = s["table"].long().gather(1, at // page)
    there = there & (where >= 0) & (where < s["Kc"].shape[0])
    where = where.clamp(0, s["Kc"].shape[0] - 1)

    def rows(pool, scale):
        if scale is None:
            x = pool[where, :, at % page]
        else:
            x = values(pool.view(torch.uint8)[where, :, at % page].view(torch.float8_e4m3fn), scale[where, :, at % page])
        return torch.where(there[:, None, :, None], x.transpose(1, 2), 0).to(DTYPES[c["dtype"]])
    return [rows(s["Kc"], s["Ks"]), rows(s["Vc"], s["Vs"])]


def plain_attend(s):
    c = s["case"]
    B, Z, Zkv, A, T, page = (c[k] for k in ("B", "Z", "Zkv", "A", "T", "page"))
    pages = s["Kc"].shape[0]
    table = s["table"].long()
    W = table.shape[1]
    held = (table >= 0) & (table < pages)
    at = table.clamp(0, pages - 1)

    def rows(pool, scale):      # (B, Zkv, W page, A)
        x = pool[at] if scale is None else values(pool.view(torch.uint8)[at].view(torch.float8_e4m3fn), scale[at])
        return x.permute(0, 2, 1, 3, 4).reshape(B, Zkv, W * page, A).float()

    slot, there = new_slots(s)
    j = torch.arange(W * page, device="cuda")
    seen = (held.repeat_interleave(page, 1) & (j[None] < s["lengths"].long()[:, None]))[:, None]      # (B, T or 1, slots)
    if c["kind"] == "chunk" and c["causal"]:
        seen = seen & (j <= slot[:, :, None])
    group = Z // Zkv
    q = s["Q"].float().reshape(B, Zkv, group * T, A)
    S = torch.matmul(q, rows(s["Kc"], s["Ks"]).transpose(-1, -2)).mul_(1.0 / math.sqrt(A)).view(B, Zkv, group, T, W * page)
    S.masked_fill_(~seen[:, None, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = S.sub_(m).exp_()
    total = P.sum(-1, keepdim=True)
    V = rows(s["Vc"], s["Vs"]).masked_fill(~seen.any(1)[:, None, :, None], 0.0)
    O = torch.matmul(P.view(B, Zkv, group * T, W * page), V).view(B, Zkv, group, T, A) / torch.where(total == 0, torch.ones_like(total), total)
    LSE = (torch.log(total) + m).reshape(B, Z, T)
    O = O.reshape(B, Z, T, A).to(s["Q"].dtype)
    if s["counts"] is not None:      # rows of no token
        O = torch.where(there[:, None, :, None], O, 0)
        LSE = torch.where(there[:, None], LSE, -math.inf)
    return [O, LSE]


# --------------------------------------------------------------------------- the definition, in 64 bits
def numbers_of_e4m3(device="cuda"):
    """All that e4m3 has from 0 on, by their bits: three of a fraction, four of an exponent."""
    v = [(f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)) for e in range(16) for f in range(8)]
    return torch.tensor(v[:-1], dtype=torch.float64, device=device)      # (the last one is NaN)


def powers(e, device="cuda"):
    """... of two, out of a list."""
    return torch.tensor([2.0 ** k for k in range(-200, 201)], dtype=torch.float64, device=device)[e.long() + 200]


def exact_e4m3(x):
    """The nearest of all numbers, of two the one with an even last bit, under the row's power of two."""
    v = numbers_of_e4m3(x.device)
    e = torch.full_like(x[..., :1], LEAST_SCALE)
    top = x.abs().amax(-1, keepdim=True)
    for k in range(LEAST_SCALE + 1, 40):      # (no input here is larger)
        e = torch.where(top > E4M3_MOST * 2.0 ** (k - 1), float(k), e)
    e = powers(e, x.device)
    y = x.abs() / e
    hi = torch.searchsorted(v, y.contiguous()).clamp(1, len(v) - 1)
    lo = hi - 1
    below, above = y - v[lo], v[hi] - y
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return torch.sign(x) * v[torch.where(up, hi, lo)] * e


def exact_turn(x, pos, inv_freq, adjacent):
    """Pairs as complex numbers, times exp(i angle)."""
    x = x.double()
    if inv_freq is None:
        return x
    R = 2 * inv_freq.numel()
    angle = torch.outer(pos.double(), inv_freq.double())
    z = torch.polar(torch.ones_like(angle), angle)
    if adjacent:
        p = torch.view_as_complex(x[..., :R].reshape(*x.shape[:-1], R // 2, 2).contiguous()) * z
        first = torch.view_as_real(p).flatten(-2)
    else:
        p = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous()) * z
        first = torch.cat([p.real, p.imag], -1)
    return torch.cat([first, x[..., R:]], -1)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    B, Z, Zkv, A, T, page, pages = c["B"], c["Z"], c["Zkv"], c["A"], c["T"], c["page"], s["Kc"].shape[0]
    lengths, counts = lengths_of(c), counts_of(c) if T > 1 else [1] * B
    f64 = dict(dtype=torch.float64, device="cuda")
    if c["kind"] == "store":
        Qr, K, V = s["Qr"].double(), torch.zeros(B, Zkv, T, A, **f64), torch.zeros(B, Zkv, T, A, **f64)
        for b, (n, k) in enumerate(zip(lengths, counts)):
            base = 0 if s["first"] is None else int(s["first"][b])
            pos = torch.arange(base + n - k, base + n, device="cuda")
            Qr[b, :, :k] = exact_turn(s["Q"][b, :, :k], pos, s["inv_freq"], c["adjacent"])
            K[b, :, :k] = exact_e4m3(exact_turn(s["K"][b, :, :k], pos, s["inv_freq"], c["adjacent"]))
            V[b, :, :k] = exact_e4m3(s["V"][b, :, :k].double())
        return [Qr, K, V]

    def stored(pool, scale, where, h, place):
        if scale is None:
            return pool[where, h, place].double()
        x = pool.view(torch.uint8)[where, h, place].view(torch.float8_e4m3fn).double()
        return x * powers(scale[where, h, place].long() - 127)[..., None]

    def held(b, first, last):      # slots, their pages and their places
        slots = torch.arange(max(first, 0), max(first, last, 0), device="cuda")
        where = s["table"][b].long()[slots // page]
        keep = (where >= 0) & (where < pages)
        return slots[keep], where[keep], slots[keep] % page
    if c["kind"] == "read":
        K, V = torch.zeros(B, Zkv, T, A, **f64), torch.zeros(B, Zkv, T, A, **f64)
        for b, (n, k) in enumerate(zip(lengths, counts)):
            slots, where, place = held(b, n - k, n)
            for h in range(Zkv):
                K[b, h, slots - (n - k)] = stored(s["Kc"], s["Ks"], where, h, place)
                V[b, h, slots - (n - k)] = stored(s["Vc"], s["Vs"], where, h, place)
        return [K, V]
    O = torch.zeros(B, Z, T, A, **f64)
    LSE = torch.full((B, Z, T), -math.inf, **f64)
    for b, (n, k) in enumerate(zip(lengths, counts)):
        slots, where, place = held(b, 0, n)
        if slots.numel() == 0:
            continue
        token = torch.arange(n - k, n, device="cuda")
        hidden = (slots[None] > token[:, None]) if c["kind"] == "chunk" and c["causal"] else torch.zeros(k, len(slots), dtype=torch.bool, device="cuda")
        for h in range(Zkv):
            K, V = stored(s["Kc"], s["Ks"], where, h, place), stored(s["Vc"], s["Vs"], where, h, place)
            for z in range(h * (Z // Zkv), (h + 1) * (Z // Zkv)):
                S = (s["Q"][b, z, :k].double() @ K.T / math.sqrt(A)).masked_fill(hidden, -math.inf)
                LSE[b, z, :k] = torch.logsumexp(S, -1)
                O[b, z, :k] = torch.softmax(S, -1).nan_to_num(0.0) @ V      # (a row that sees nothing is 0)
    return [O, LSE]
