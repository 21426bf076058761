"""msa_latent_attn_paged where a CTA's share of the steps goes on from tile to tile, against the float64 oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2606_13392_amd import msa
from tests.latent_util import PagedBatch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


def call(b):
    if b.fp8:
        return msa.latent_attn_paged_fp8(b.dq, b.dq_rope, b.cache, b.scale, b.seqs)
    return msa.latent_attn_paged(b.dq, b.dq_rope, b.cache, b.seqs)


def runs(q_rows, kv_lens, heads):
    """Steps (of 64 keys) of each tile that each CTA's share has, in order; the rule of the kernel's plan."""
    blocks = -(-heads // 64)
    rows = 64 // heads if blocks == 1 else 1
    shares = max(8, 256 // blocks // 8 * 8)
    tiles = []
    for q, m in zip(q_rows, kv_lens):
        tiles += [-(-min(m, max(m - q, 0) + (x + 1) * rows) // 64) for x in range(-(-q // rows))]
    per = max(2, -(-sum(tiles) // shares))
    out, cut, first = [[]], per, 0
    for t in tiles:
        while t:
            n = min(t, cut - first)
            out[-1].append(n)
            first, t = first + n, t - n
            if first == cut:
                out.append([])
                cut += per
    return out


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("R", [256, 512])
@pytest.mark.parametrize("heads,steps", [(64, 1), (64, 3), (32, 5)])
def test_shares_that_go_on_after_an_odd_number_of_steps(heads, steps, R, fp8):
    """Behind a tile's last step copies go into the buffer that the next step would have had; after an odd number of steps
    the next tile's queries go there.  Each row has queries of its own, and all are checked."""
    n = 300 if steps < 5 else 200
    kv_lens = [64 * steps - i % 64 for i in range(n)]
    q_rows = [1 + (heads < 64 and i % 2) for i in range(n)]
    q_rows = [min(q, m) for q, m in zip(q_rows, kv_lens)]
    crossing = [r for r in runs(q_rows, kv_lens, heads) if any(x % 2 for x in r[:-1])]
    assert len(crossing) >= 100
    b = PagedBatch(f"shares_{heads}_{steps}", q_rows, kv_lens, heads, R, 64, 0, fp8)
    o, lse = call(b)
    b.check(o, lse, np.arange(b.n), "shares")
    for _ in range(3):
        o2, l2 = call(b)
        assert torch.equal(o, o2) and torch.equal(lse, l2)


# name, q_rows, kv_lens, heads, latent, page
MANY_TILES = [
    ("three_rows_a_tile", [400, 250], [900, 260], 20, 256, 64),          # 134 and 84 tiles
    ("five_rows_a_tile", [700], [700], 12, 512, 16),                     # 140
    ("six_rows_a_tile", [3, 900], [300, 1500], 10, 256, 128),            # 150
    ("nine_rows_a_tile", [1200, 1, 600], [1300, 70, 600], 7, 256, 32),   # 134 and 67
]


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", MANY_TILES, ids=[c[0] for c in MANY_TILES])
def test_tiles_beyond_a_period(case, fp8):
    """Steps of tiles whose rows are no power of two repeat after 64 tiles; sequences of more tiles than that."""
    name, q_rows, kv_lens, H, R, page = case
    assert max(-(-q // (64 // H)) for q in q_rows) > 128
    b = PagedBatch(name, q_rows, kv_lens, H, R, page, 0, fp8)
    o, lse = call(b)
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all())
    b.check(o, lse, np.arange(0, b.n, 2), name)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("H,R", [(200, 512), (600, 512), (1000, 256), (1024, 512)])
def test_many_head_blocks(H, R, fp8):
    """4, 10 and 16 blocks of heads, the last of them smaller or not."""
    b = PagedBatch(f"blocks_{H}", [1, 2, 1], [700, 130, 1], H, R, 64, 0, fp8)
    o, lse = call(b)
    b.check(o, lse, np.arange(b.n), "blocks")
