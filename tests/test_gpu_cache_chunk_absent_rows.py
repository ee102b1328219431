"""Rows of tokens that are not there cost no walk over the cache."""
import pytest
import torch

from cache8_helpers import i32
from paper_2105_13120_amd import rsa

pytestmark = pytest.mark.gpu


def time_of(T, counts, n=8192, A=64, heads=4, page=64, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(61)
    B, W = len(counts), n // page
    K, V = (torch.randn(B * W, heads, page, A, generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.arange(B * W, device="cuda").reshape(B, W).int()
    Q = torch.randn(B, heads, T, A, generator=g, device="cuda").to(dtype)
    O, LSE = torch.empty_like(Q), torch.empty(B, heads, T, device="cuda")
    d, lengths, counts = rsa.make_cache_desc(K, table, heads), i32([n] * B), i32(counts)
    ws = torch.empty(max(16, rsa.cache_chunk_workspace_bytes(d, T)), dtype=torch.uint8, device="cuda")
    call = lambda: rsa.cache_attend_chunk(d, Q, K, V, table, lengths, counts, O=O, LSE=LSE, ws=ws)
    best = float("inf")
    for _ in range(5):
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        call()
        e[0].record()
        for _ in range(5):
            call()
        e[1].record()
        torch.cuda.synchronize()
        best = min(best, e[0].elapsed_time(e[1]) / 5)
    return best


@pytest.mark.parametrize("T,B,counts", [(1024, 8, [32] * 8), (512, 80, [32] * 80), (512, 80, [512] * 4 + [0] * 76), (512, 80, [512, 64, 16, 0] * 20)])
def test_few_tokens_in_a_call_for_many(T, B, counts):
    """Walks of whole segments, of more work-groups than there are places: less than half of the time of all T tokens of each sequence."""
    some, full = time_of(T, counts), time_of(T, [T] * B)
    print(f"T {T} B {B}: {sum(counts)} tokens {some * 1e3:.1f} us, {T * B} {full * 1e3:.1f}", flush=True)
    assert some < full / 2
