"""Every form of msa_latent_attn and of its gradients: which one a call takes, told from the kernel timer's names, and its
results against the float64 oracle."""
from __future__ import annotations

import pytest
import torch

from paper_2606_13392_amd import msa
from tests.latent_util import ExpandedBatch, some_rows
from tests.test_gpu_latent_backward import CASES as GRADIENT_CASES, check, make, run

pytestmark = pytest.mark.gpu
WIDE, NARROW, SHARES = {"latent_attn_kernel"}, {"latent_attn_narrow_kernel"}, {"latent_attn_kernel", "latent_join_kernel"}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


def launched(call):
    """(what the call returned, names of the kernels that it launched)."""
    msa.profile_enable(True)
    msa.profile_reset()
    try:
        out = call()
        torch.cuda.synchronize()
        return out, set(msa.profile_read())
    finally:
        msa.profile_enable(False)
        msa.profile_reset()


# name, kernels, q_rows, kv_lens, heads, rows behind the last sequence
CASES = [
    # a CTA of 8 waves for each tile: several tiles of a sequence behind a context, one, part of one, prompts
    ("wide_chunk", WIDE, [512], [1100], 128, 0),
    ("wide_chunks", WIDE, [512, 500], [1400, 1300], 64, 3),
    ("wide_tile_of_many_heads", WIDE, [200], [500], 256, 1),
    ("wide_few_rows_of_many_heads", WIDE, [32, 7, 1, 20], [600, 500, 70, 20], 129, 0),
    ("wide_prompts", WIDE, [2100, 900], [2100, 900], 128, 0),
    # of 4
    ("narrow_chunk", NARROW, [200], [2000], 128, 0),
    ("narrow_chunks", NARROW, [100, 120], [1000, 900], 100, 2),
    ("narrow_chunks_of_many_heads", NARROW, [128, 3], [1500, 64], 136, 0),
    ("narrow_prompt", NARROW, [777], [777], 20, 0),
    ("narrow_prompts", NARROW, [600, 1, 300], [600, 1, 300], 64, 0),
    # shares of the steps and their join; several tiles, one, heads that do not divide the CTAs
    ("shares_chunks", SHARES, [130, 20], [1500, 900], 8, 0),
    ("shares_few_rows", SHARES, [64], [9000], 8, 0),
    ("shares_twenty_heads", SHARES, [500, 300], [3000, 2500], 20, 1),
    ("shares_eighty_heads", SHARES, [200], [3000], 80, 0),
]


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_forms(case):
    name, kernels, q_rows, kv_lens, H, pad = case
    b = ExpandedBatch(name, q_rows, kv_lens, H, pad)
    T, n = b.n + pad, b.n
    o = torch.full((T, H, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), 7.0, device="cuda")
    size = msa.latent_attn_workspace_size(b.seqs, H)
    assert (size > 0) == (kernels is SHARES)
    ws = torch.full((max(1, size),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN where it is read unwritten
    _, names = launched(lambda: msa.latent_attn(b.dq, b.dq_rope, b.dkv, b.dk_rope, b.seqs, out=o, lse=lse, workspace=ws))
    assert names == kernels
    assert bool((o[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    b.check(o, lse, some_rows(b.rng, b.lay.q_offsets, n, 24), name)


@pytest.mark.parametrize("case,kernel", [(GRADIENT_CASES[4], "latent_backward_q_narrow_kernel"),
                                         (GRADIENT_CASES[10], "latent_backward_q_kernel")], ids=lambda c: c[0] if isinstance(c, tuple) else c)
def test_gradient_forms(case, kernel):
    b, o, lse = make(case)
    got, names = launched(lambda: run(b, o, lse))
    assert names == {kernel, "latent_backward_kv_kernel", "latent_sum_kernel"}
    check(b, o, lse, got)
