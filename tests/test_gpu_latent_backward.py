"""msa_latent_attn_backward against the float64 oracle's formulas, and against differences of the forward."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa
from tests.latent_util import ROT, SCALE, ExpandedBatch, check_grad
from tests.operators_util import bf16, dev, host, replay

pytestmark = pytest.mark.gpu
NAMES = ("d_q", "d_q_rope", "d_k", "d_k_rope", "d_v")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


# name, q_rows, kv_lens, heads, rows behind the last sequence
CASES = [
    ("one_token", [1], [1], 8, 0),
    ("one_row_each", [1, 1, 1], [1, 64, 200], 5, 0),
    ("short", [17], [17], 1, 0),
    ("prompt", [333], [333], 2, 0),
    ("tile_edges", [64, 65, 128, 129, 127], [64, 65, 128, 129, 127], 3, 0),
    ("documents", [65, 0, 300, 1], [65, 9, 300, 1], 5, 3),
    ("chunks", [130, 20], [400, 190], 2, 0),
    ("few_on_many", [3], [700], 2, 0),
    ("many_heads", [20, 33], [20, 40], 64, 0),
    ("70_sequences", [1 + 3 * i % 20 for i in range(70)], [1 + 3 * i % 20 + i % 7 for i in range(70)], 2, 1),
    # so many tiles that a wave takes 64 queries, in one of them several tiles long
    ("long_among_many", [700, 300] + [2] * 385, [700, 500] + [2] * 385, 2, 0),
    # none, one and several tiles of keys each, some sequences without rows
    ("600_sequences", [i % 3 for i in range(600)], [i % 3 + (130 * (i % 17 == 0)) for i in range(600)], 2, 1),
]


def make(case):
    name, q_rows, kv_lens, H, pad = case
    b = ExpandedBatch(name, q_rows, kv_lens, H, pad)
    b.d_o = bf16(b.rng.standard_normal((b.n + pad, H, 128)))
    o, lse = msa.latent_attn(b.dq, b.dq_rope, b.dkv, b.dk_rope, b.seqs)
    o[b.n:], lse[b.n:] = float("nan"), float("nan")        # rows behind the last sequence take no part
    b.d_o_dev = dev(b.d_o)
    return b, o, lse


def run(b, o, lse, **kw):
    return msa.latent_attn_backward(b.dq, b.dq_rope, b.dkv, b.dk_rope, o, lse, b.d_o_dev, b.seqs, **kw)


def check(b, o, lse, got, scale=SCALE, lay=None):
    ref, size = O.latent_attention_backward(b.q, b.q_rope, b.kv[..., :128], b.k_rope, b.kv[..., 128:], host(o), host(lse), b.d_o,
                                            lay or b.lay, scale)
    dq, de, dkv, dr = (host(x) for x in got)
    for name, x, r, z in zip(NAMES, (dq[:b.n], de[:b.n], dkv[..., :128], dr, dkv[..., 128:]),
                             (ref[0][:b.n], ref[1][:b.n], *ref[2:]), (size[0][:b.n], size[1][:b.n], *size[2:])):
        check_grad(x, r, z, name)


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_latent_backward(case):
    name, q_rows, kv_lens, H, pad = case
    b, o, lse = make(case)
    T = b.n + pad
    joint = torch.full((T, H * (128 + ROT) + 4), 7.0, dtype=torch.bfloat16, device="cuda")
    d_q, d_e = joint[:, :H * 128].view(T, H, 128), joint[:, H * 128:H * (128 + ROT)].view(T, H, ROT)
    d_kv = torch.full((b.N, H, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    wide = torch.full((b.N, 16 + ROT), 7.0, dtype=torch.bfloat16, device="cuda")
    size = msa.latent_attn_backward_workspace_size(b.seqs, H)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")          # NaN where it is read unwritten
    got = run(b, o, lse, d_q=d_q, d_q_rope=d_e, d_kv=d_kv, d_k_rope=wide[:, 16:], workspace=ws)
    assert bool((joint[b.n:] == 7.0).all()) and bool((joint[:, -4:] == 7.0).all()) and bool((wide[:, :16] == 7.0).all())
    assert bool((d_kv[torch.from_numpy(~b.owned).cuda()] == 0).all()) and bool((wide[torch.from_numpy(~b.owned).cuda(), 16:] == 0).all())
    check(b, o, lse, got)
    for x, y in zip(got, run(b, o, lse)):                                     # the same bits again
        assert torch.equal(x[:b.n] if x is d_q or x is d_e else x, y[:b.n] if x is d_q or x is d_e else y)


@pytest.mark.parametrize("scale", [0.0, -0.1, 0.2])
def test_softmax_scales(scale):
    b, _, _ = make(("scales", [3, 80], [70, 130], 2, 0))
    o, lse = msa.latent_attn(b.dq, b.dq_rope, b.dkv, b.dk_rope, b.seqs, softmax_scale=scale)
    check(b, o, lse, run(b, o, lse, softmax_scale=scale), scale)


def test_against_differences():
    """The gradients of sum(d_o O) along random directions, against central differences of the forward in 64 bits."""
    b, o, lse = make(("differences", [40, 9], [60, 9], 2, 0))
    got = [host(x) for x in run(b, o, lse)]
    grads = (got[0], got[1], got[2][..., :128], got[3], got[2][..., 128:])
    x = [b.q, b.q_rope, b.kv[..., :128].copy(), b.k_rope, b.kv[..., 128:].copy()]
    for x_ in x[2:]:
        x_[~b.owned] = 0.0
    def loss(v):
        return (O.latent_attention(v[0], v[1], v[2], v[3], v[4], b.lay, SCALE)[0] * b.d_o).sum()
    eps = 1e-4
    for i, name in enumerate(NAMES):
        # along the gradient's signs every element counts, so errors cannot hide in a sum of both signs
        step = np.sign(grads[i])
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + eps * step, x[i] - eps * step
        want = (loss(up) - loss(down)) / (2 * eps)
        have = np.abs(grads[i]).sum()
        # roundings of bf16 in P or dS, in O (through D) and in the result, each at most 2^-8 of a term; terms of both signs
        # make a gradient smaller than its terms, so their relative part is allowed 4 times that
        assert abs(have - want) <= 4 * 2.0 ** -8 * abs(want), (name, have, want)


def test_rows_without_keys():
    b, _, _ = make(("empty", [1, 300, 3], [5, 300, 70], 2, 0))
    lens = [0, 20, 70]
    b.seqs.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    o, lse = msa.latent_attn(b.dq, b.dq_rope, b.dkv, b.dk_rope, b.seqs)
    got = run(b, o, lse)
    assert bool((got[0][:281] == 0).all()) and bool((got[1][:281] == 0).all())
    check(b, o, lse, got, lay=O.Layout([1, 300, 3], lens, b.lay.kv_starts))


def test_no_query_rows():
    """Keys that no query attends get zeros."""
    seqs = msa.Seqs([0, 0], [40, 5], [0, 50], 60, "cuda")
    z = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    d_kv, d_r = z(60, 4, 256), z(60, ROT)
    msa.latent_attn_backward(z(0, 4, 128), z(0, 4, ROT), z(60, 4, 256), z(60, ROT), z(0, 4, 128), torch.ones((0, 4), device="cuda"),
                             z(0, 4, 128), seqs, d_kv=d_kv, d_k_rope=d_r)
    assert bool((d_kv == 0).all()) and bool((d_r == 0).all())


def test_captured():
    b, o, lse = make(CASES[4])
    ws = torch.empty(msa.latent_attn_backward_workspace_size(b.seqs, b.H), dtype=torch.uint8, device="cuda")
    def step():
        return run(b, o, lse, workspace=ws)
    replay(step, step)


def test_two_calls_at_once():
    made = [make(CASES[i]) for i in (4, 6)]
    want = [run(*m) for m in made]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for st, m in zip(streams, made):
            with torch.cuda.stream(st):
                got.append(run(*m))
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
