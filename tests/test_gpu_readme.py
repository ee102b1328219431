"""The README's Python examples run, one after the other in one program."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_examples():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    blocks = re.findall(r"```python\n(.*?)```", text, re.S)
    assert len(blocks) == 2
    names = {}
    for b in blocks:
        exec(compile(b, "README.md", "exec"), names)
    torch.cuda.synchronize()
    assert names["dQ"].isfinite().all() and names["o"].isfinite().all()
    # one token in the cache: its value
    assert torch.equal(names["o"], names["v"].repeat_interleave(4, 1))
