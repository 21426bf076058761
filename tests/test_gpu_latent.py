"""msa_latent_attn against the float64 oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa
from tests.latent_util import ExpandedBatch, some_rows
from tests.operators_util import replay

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


# name, q_rows, kv_lens, heads, rows behind the last sequence
CASES = [
    ("first_token", [1], [1], 8, 0),
    ("one_row_each", [1, 1, 1, 1], [1, 63, 64, 1000], 5, 0),
    ("one_head", [300], [300], 1, 0),
    ("prompt", [333], [333], 20, 0),
    ("prompts", [65, 0, 256, 1, 257], [65, 7, 256, 1, 257], 8, 3),
    ("chunks", [130, 20], [1500, 900], 8, 0),
    ("chunk_on_long", [64], [9000], 8, 0),
    ("mixed", [1, 300, 1, 0, 40, 1], [2000, 900, 64, 128, 41, 777], 20, 2),
    ("many_heads", [70, 33], [70, 90], 256, 0),
    ("many_tiles", [2100, 900], [2100, 900], 128, 0),
    ("100_sequences", [1 + 3 * i % 50 for i in range(100)], [1 + 3 * i % 50 + i for i in range(100)], 8, 1),
]


def run(b, **kw):
    return msa.latent_attn(b.dq, b.dq_rope, b.dkv, b.dk_rope, b.seqs, **kw)


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_latent_attn(case):
    name, q_rows, kv_lens, H, pad = case
    b = ExpandedBatch(name, q_rows, kv_lens, H, pad)
    T, n = b.n + pad, b.n
    o = torch.full((T, H, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), 7.0, device="cuda")
    ws = torch.full((max(1, msa.latent_attn_workspace_size(b.seqs, H)),), 0xFF, dtype=torch.uint8, device="cuda")
    run(b, out=o, lse=lse, workspace=ws)                                      # NaN where it is read unwritten
    assert bool((o[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    assert bool(torch.isfinite(o[:n]).all()) and bool(torch.isfinite(lse[:n]).all())
    b.check(o, lse, some_rows(b.rng, b.lay.q_offsets, n), name)
    o2, l2 = run(b)                                                           # the same bits again
    assert torch.equal(o2[:n], o[:n]) and torch.equal(l2[:n], lse[:n])


@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-30, 0.2])
def test_softmax_scales(scale):
    b = ExpandedBatch("scales", [3, 80], [70, 130], 8)
    o, l = run(b, softmax_scale=scale)
    b.check(o, l, np.arange(b.n), "scale", scale=scale)


def test_strides():
    """Heads first, per-head [own, rotated] columns and contiguous queries give the same bits."""
    b = ExpandedBatch("strides", [2, 90], [200, 100], 20)
    o, l = run(b)
    both = torch.cat((b.dq, b.dq_rope), -1)
    first = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (b.dq, b.dq_rope)]
    for q, e in ((both[..., :128], both[..., 128:]), first, (b.dq.contiguous(), b.dq_rope.contiguous())):
        o2, l2 = msa.latent_attn(q, e, b.dkv, b.dk_rope.contiguous(), b.seqs)
        assert torch.equal(o, o2) and torch.equal(l, l2)


@pytest.mark.parametrize("heads", [8, 256])
def test_rows_without_keys(heads):
    """Lengths that fall behind the rows: rows without a key get zeros and -inf."""
    b = ExpandedBatch("empty", [1, 300, 3], [5, 300, 70], heads)
    b.seqs.kv_lens.copy_(torch.tensor([0, 20, 70], dtype=torch.int32))
    o, l = run(b)
    assert bool((o[:281] == 0).all()) and bool((l[:281] == -float("inf")).all())
    b.check(o, l, np.r_[270:304], "empty", lay=O.Layout([1, 300, 3], [0, 20, 70], b.lay.kv_starts))


@pytest.mark.parametrize("case", [CASES[3], CASES[5], CASES[9]], ids=lambda c: c[0])
def test_captured_with_lengths_that_grow(case):
    name, q_rows, kv_lens, H, pad = case
    b = ExpandedBatch(name, q_rows, kv_lens, H, pad)
    ws = torch.empty(max(1, msa.latent_attn_workspace_size(b.seqs, H)), dtype=torch.uint8, device="cuda")
    def step():
        return run(b, workspace=ws)
    replay(step, step)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    shorter = [max(q, 1, int(m * f)) for q, m, f in zip(q_rows, kv_lens, b.rng.uniform(0.1, 1.0, len(q_rows)))]
    for lens in (shorter, kv_lens):
        b.seqs.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        b.check(*got, some_rows(b.rng, b.lay.q_offsets, b.n, 12), name, lay=O.Layout(q_rows, lens, b.lay.kv_starts))


def test_two_calls_at_once():
    made = [ExpandedBatch(*CASES[i]) for i in (5, 7)]
    want = [run(b) for b in made]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for st, b in zip(streams, made):
            with torch.cuda.stream(st):
                got.append(run(b))
        torch.cuda.synchronize()
        for b, (o, l), (o2, l2) in zip(made, want, got):
            assert torch.equal(o[:b.n], o2[:b.n]) and torch.equal(l[:b.n], l2[:b.n])


def test_keys_past_4_gib():
    """Key rows whose bytes lie past 2^32 of the tensor."""
    H, rows = 64, 140000                                   # 32 KiB each: 4.6 GB
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB")
    b = ExpandedBatch("past", [100], [300], H)
    kv = torch.empty((rows, H, 256), dtype=torch.bfloat16, device="cuda")
    k_rope = torch.empty((rows, 64), dtype=torch.bfloat16, device="cuda")
    at = rows - 310
    kv[at:at + 300], k_rope[at:at + 300] = b.dkv[3:303], b.dk_rope[3:303]
    o, l = msa.latent_attn(b.dq, b.dq_rope, kv, k_rope, msa.Seqs([100], [300], [at], rows, "cuda"))
    b.check(o, l, np.arange(0, 100, 9), "past 4 GiB")
