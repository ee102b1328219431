"""What the README's example of pieces of prompts in a cache of 8 bits gives."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_pieces_of_prompts():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    names = {}
    for b in re.findall(r"```python\n(.*?)```", text, re.S):
        exec(compile(b, "README.md", "exec"), names)
    torch.cuda.synchronize()
    there = torch.arange(names["T"], device="cuda")[None] < names["counts"][:, None]
    for x in (names["o8"], names["k_back"], names["v_back"]):
        assert x.isfinite().all() and (x[~there[:, None].expand(x.shape[:3])] == 0).all()
    assert (names["lse8"].isneginf() == ~there[:, None]).all()
    # a sequence's first token sees itself alone: its value, as the cache holds it (half a step of e4m3 off at most)
    first, v = names["o8"][:, :, 0], names["v_back"][:, :, 0].repeat_interleave(4, 1)
    assert torch.equal(first, v)
    v8 = names["v8"].float() * there[:, None, :, None]
    step = torch.maximum(v8.abs() * 2.0 ** -4, v8.abs().amax(-1, keepdim=True) * 2.0 ** -17)   # below 2^-6 448 / 2 of the row's power: 2^-10 of that
    assert ((names["v_back"].float() - v8).abs() <= step).all()
