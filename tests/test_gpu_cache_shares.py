"""Attention of a new token where its work is divided into shares: every slot counts once, wherever shares begin and end."""
import numpy as np
import pytest
import torch

from cache_helpers import F32, STEP, f64, within
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def apart(lengths, B, where, A=128, page=16):
    """Sequences of these lengths at the given places among B, the others empty; queries of zeros, so that every slot has the same weight."""
    n = np.zeros(B, np.int32)
    n[where] = lengths
    width = -(-max(lengths) // page)
    g = torch.Generator(device="cuda").manual_seed(50)
    pages = 512
    Kc, Vc = (torch.randn(pages, 1, page, A, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(pages, (B, width), generator=g, device="cuda", dtype=torch.int32)
    return torch.zeros(B, 4, 1, A, dtype=torch.bfloat16, device="cuda"), Kc, Vc, table, i32(n)


def time_of(call):
    """The shortest of ten in us, captured."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            call()
    best = float("inf")
    for _ in range(10):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        best = min(best, begin.elapsed_time(end) * 100)
    return best


def test_empty_sequences_between_long_ones():
    """A share that begins in one sequence and ends in one 2000 rows of the table behind it, in at most three times the time that it takes
    with the empty rows at the table's end (about as long; each empty row looked at alone takes five times as long)."""
    lengths, where = [35001, 7777, 16500], [0, 2000, 4095]
    Q, Kc, Vc, table, n = apart(lengths, 4096, where)
    all_of = rsa.make_cache_desc(Kc, table, 4)
    O, LSE = rsa.cache_attend(all_of, Q, Kc, Vc, table, n)
    for b, count in zip(where, lengths):
        v = Vc[table[b].long(), 0].reshape(-1, Vc.shape[-1])[:count].double()
        # equal weights: exp(0) is 1, their sum exact, log and its product off by 2^-22 and a rounding; sums of values by 2^-24 of their size a step of
        # the walk, 64 at most, the waves and the shares
        within(LSE[b], np.full((4, 1), np.log(count)), 2.0 ** -22 + 2 * F32 * np.log(count), "LSE")
        mean = f64(v.mean(0)).reshape(1, 1, -1)
        within(O[b], np.broadcast_to(mean, O[b].shape), STEP["bf16"] * np.abs(mean) + 400 * F32 * f64(v.abs().mean(0)), "O")
    none = torch.ones(4096, dtype=torch.bool)
    none[where] = False
    assert (O[none.cuda()] == 0).all() and torch.isneginf(LSE[none.cuda()]).all()
    ws = torch.empty(rsa.cache_workspace_bytes(all_of), dtype=torch.uint8, device="cuda")
    together = apart(lengths, 4096, [0, 1, 2])[-1]
    long, short = (time_of(lambda: rsa.cache_attend(all_of, Q, Kc, Vc, table, m, O, LSE, ws)) for m in (n, together))
    assert long <= 3 * short, (long, short)
