"""Refusals of the operators around the attention calls, in the binding."""
from __future__ import annotations

import pytest
import torch

from paper_2606_13392_amd import msa


@pytest.mark.parametrize("absent", ["q", "k"])
@pytest.mark.parametrize("buffer", ["d_{}", "d_{}_weight"])
def test_gradient_buffers_need_their_upstream_gradient(absent, buffer):
    """They would be left as they are."""
    bf = torch.bfloat16
    seqs = msa.Seqs([4], [4], [0], 4, "cpu")
    x, w = torch.zeros((4, 2, 128), dtype=bf), torch.ones(128)
    g = {"q": x, "k": x, absent: None}
    kw = {buffer.format(absent): torch.zeros(128) if "weight" in buffer else torch.zeros_like(x)}
    with pytest.raises(ValueError, match=f"without d_{absent}_out"):
        msa.qk_norm_rope_backward(x, x, g["q"], g["k"], seqs, None, w, w, **kw)
