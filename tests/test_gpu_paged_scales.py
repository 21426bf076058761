"""msa_dense_attn_paged_fp8: the score scale is the product of three factors, none of which has to stay in fp32's range
with only one of the others."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2606_13392_amd import msa
from tests.operators_util import padded_seqs, page_table

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("softmax_scale,power", [(11.0, 126), (1e-3, -126)], ids=["overflow", "underflow"])
@pytest.mark.parametrize("q_rows", [[1, 3], [40, 2]], ids=["few_rows", "tiles"])
def test_scales_may_cancel(q_rows, softmax_scale, power):
    """(q, k) scales of (1.3 2^p, 2^-p) are those of (1.3, 1): the same bits."""
    rng = np.random.default_rng(7)
    kv_lens = [50, 90]
    table, total, _ = page_table(rng, kv_lens, 64)
    seqs = padded_seqs(q_rows, kv_lens, total_kv=total, table=torch.from_numpy(table).cuda(), page=64)
    draw = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, D)).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).cuda()  # noqa: E731,E501
    q, k, v = draw(sum(q_rows), 8), draw(total, 2), draw(total, 2)
    q_scale = float(np.float32(1.3))
    want = msa.dense_attn_paged_fp8(q, k, v, (q_scale, 1.0, 0.5), seqs, softmax_scale=softmax_scale)
    got = msa.dense_attn_paged_fp8(q, k, v, (q_scale * 2.0 ** power, 2.0 ** -power, 0.5), seqs, softmax_scale=softmax_scale)
    assert bool(torch.isfinite(want[1]).all())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
