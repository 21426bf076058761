"""Weight gradients of msa_qk_norm_rope_backward where a tensor has no heads: a sum over nothing is written."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2606_13392_amd import msa
from tests.operators_util import padded_seqs

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("other_norm", [True, False], ids=["other_normed", "other_rotated"])
@pytest.mark.parametrize("rows", [5, 0])
@pytest.mark.parametrize("absent", ["q", "k"])
def test_weight_gradient_without_heads_is_zero(absent, rows, other_norm):
    seqs = padded_seqs([rows], [9])
    H = 2
    x, g, d = (torch.randn((rows, H, D), device="cuda").to(torch.bfloat16) for _ in range(3))
    w = torch.ones(D, device="cuda")
    dw = {n: torch.full((D,), 7.0, device="cuda") for n in ("q", "k")}
    size = msa.qk_norm_rope_backward_workspace_size(seqs, 0 if absent == "q" else H, 0 if absent == "k" else H, D)
    ws = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
    side = {n: (None, 0, None, w.data_ptr(), None, 0, dw[n].data_ptr(), 0) if n == absent else
            (x.data_ptr(), H * D, g.data_ptr(), w.data_ptr() if other_norm else None, d.data_ptr(), H * D,
             dw[n].data_ptr() if other_norm else None, H) for n in ("q", "k")}
    (xq, sq, gq, wq, dq, dsq, dwq, hq), (xk, sk, gk, wk, dk, dsk, dwk, hk) = side["q"], side["k"]
    st = msa.lib().msa_qk_norm_rope_backward(xq, sq, xk, sk, gq, gk, seqs.ref(), hq, hk, D, wq, wk, 1e-6, None, dq, dsq, dk, dsk,
                                             dwq, dwk, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == msa.MSA_OK
    assert bool((dw[absent] == 0).all())
    other = "k" if absent == "q" else "q"
    if other_norm:
        names = dict(q=None, k=None, d_q_out=None, d_k_out=None, q_weight=None, k_weight=None)
        names.update({other: x, f"d_{other}_out": g, f"{other}_weight": w})
        want = msa.qk_norm_rope_backward(seqs=seqs, rope=None, eps=1e-6, **names)
        assert torch.equal(dw[other], want[2 if other == "q" else 3])
        assert torch.equal(d, want[0 if other == "q" else 1])
