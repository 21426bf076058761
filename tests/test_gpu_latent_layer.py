"""A layer's calls together, as serving and training make them: projections' columns through rotation, the latent cache and
both forms of the attention."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa
from tests.latent_util import ROT, SCALE, check_grad, check_lse, check_o
from tests.operators_util import amplitude, bf16, check_bf16, dev, host, page_table, replay

pytestmark = pytest.mark.gpu
H, R, EPS = 20, 256, 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


def _rope():
    f, by = msa.rope_frequencies(ROT, scaling="by_parts", factor=4.0, trained_len=4096)
    return f.numpy(), msa.Rope(f.cuda(), interleaved=True, scale=by), by


def test_serving():
    """Two prompts, then a captured step that serves token after token: rotation of the queries' part, append, absorbed
    attention, with lengths that grow on the device.  The cache's rows go through the oracle once written."""
    rng = np.random.default_rng(11)
    f, rope, by = _rope()
    prompts, steps, page = [70, 33], 4, 16
    final = [m + steps for m in prompts]
    table, total, rows = page_table(rng, final, page)
    tab = torch.from_numpy(table).cuda()
    x = [bf16(rng.standard_normal((m, R + ROT))) for m in final]              # a projection's rows: [latent, key part]
    w = (1 + 0.2 * rng.standard_normal(R)).astype(np.float32)
    q = [bf16(rng.standard_normal((m, H, R + ROT)) * np.sqrt(0.5)) for m in final]
    weight = torch.from_numpy(w).cuda()
    cache = torch.full((total, R + ROT), float("nan"), dtype=torch.bfloat16, device="cuda")

    def layer(xs, qs, seqs, ws):
        msa.latent_append(xs[:, :R], xs[:, R:], seqs, rope, cache, weight, EPS)
        q_rot, _ = msa.qk_norm_rope(qs[..., R:].contiguous(), None, seqs, rope)
        o, lse = msa.latent_attn_paged(qs[..., :R], q_rot, cache, seqs, workspace=ws)
        return o, lse, q_rot

    def check(got, lens, n_rows):
        """Rows of each sequence against the cache as it is."""
        o, lse, q_rot = (host(t) for t in got)
        at = 0
        for i, (m, n) in enumerate(zip(lens, n_rows)):
            kv = host(cache)[rows[i][:m]]
            assert np.isfinite(kv).all()
            c = kv[:, None, :R]
            ref = O.latent_attention(q[i][m - n:m, :, :R], q_rot[at:at + n], c, kv[:, R:], c, O.Layout([n], [m], [0]), SCALE)
            check_o(o[at:at + n], ref[0], ref[2], "o")
            check_lse(lse[at:at + n], ref[1], "lse")
            rot = O.norm_rope(q[i][m - n:m, :, R:], range(m - n, m), None, 0.0, f, True, by)
            check_bf16(q_rot[at:at + n], rot, amplitude(q[i][m - n:m, :, R:], ROT, True, by), "rotation")
            at += n

    seqs = msa.Seqs(prompts, prompts, [0, 0], total, "cuda", block_table=tab, page_size=page)
    ws = torch.empty(msa.latent_attn_paged_workspace_size(seqs, H, R), dtype=torch.uint8, device="cuda")
    cut = lambda a: dev(np.concatenate([t[:m] for t, m in zip(a, prompts)]))  # noqa: E731
    check(layer(cut(x), cut(q), seqs, ws), prompts, prompts)

    one = msa.Seqs([1, 1], final, [0, 0], total, "cuda", block_table=tab, page_size=page)
    xs, qs = dev(np.zeros((2, R + ROT))), dev(np.zeros((2, H, R + ROT)))
    one.kv_lens.copy_(torch.tensor([m + 1 for m in prompts], dtype=torch.int32))
    layer(xs, qs, one, ws)                                 # what a capture needs loaded
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = layer(xs, qs, one, ws)
    for k in range(steps):
        lens = [m + k + 1 for m in prompts]
        xs.copy_(dev(np.stack([t[m - 1] for t, m in zip(x, lens)])))
        qs.copy_(dev(np.stack([t[m - 1] for t, m in zip(q, lens)])))
        one.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        check(got, lens, [1, 1])
    want = O.norm_rope(np.concatenate(x)[:, None, :R], [0] * sum(final), w, EPS, np.zeros(0))[:, 0]
    check_bf16(host(cache)[np.concatenate(rows)][:, :R], want, np.abs(want), "latents")


def test_training_step():
    """Rotation, expanded attention, and back: every gradient against the oracle's at the values the step itself made, and a
    captured step against an eager one."""
    rng = np.random.default_rng(12)
    f, rope, by = _rope()
    q_rows = [100, 1, 77]
    T = sum(q_rows)
    starts = np.cumsum([0] + q_rows)[:-1].tolist()
    joint = dev(rng.standard_normal((T, H * (128 + ROT))))
    q, q_raw = joint[:, :H * 128].view(T, H, 128), joint[:, H * 128:].view(T, H, ROT)
    k_raw, kv, d_o = dev(rng.standard_normal((T, 1, ROT))), dev(rng.standard_normal((T, H, 256))), dev(rng.standard_normal((T, H, 128)))
    seqs = msa.Seqs(q_rows, q_rows, starts, T, "cuda")

    def step():
        e, r = msa.qk_norm_rope(q_raw, k_raw, seqs, rope)
        o, lse = msa.latent_attn(q, e, kv, r[:, 0], seqs)
        d_q, d_e, d_kv, d_r = msa.latent_attn_backward(q, e, kv, r[:, 0], o, lse, d_o, seqs)
        d_q_raw, d_k_raw, _, _ = msa.qk_norm_rope_backward(None, None, d_e, d_r[:, None], seqs, rope)
        return o, lse, d_q, d_kv, d_q_raw, d_k_raw, e, r, d_e, d_r

    o, lse, d_q, d_kv, d_q_raw, d_k_raw, e, r, d_e, d_r = (host(t) for t in step())
    lay = O.Layout(q_rows, q_rows, starts)
    k, v = host(kv)[..., :128], host(kv)[..., 128:]
    ref = O.latent_attention(host(q), e, k, r[:, 0], v, lay, SCALE)
    check_o(o, ref[0], ref[2], "o")
    check_lse(lse, ref[1], "lse")
    grads, sizes = O.latent_attention_backward(host(q), e, k, r[:, 0], v, o, lse, host(d_o), lay, SCALE)
    for got, want, size, name in zip((d_q, d_e, d_kv[..., :128], d_r, d_kv[..., 128:]), grads, sizes, ("q", "q_rope", "k", "k_rope", "v")):
        check_grad(got, want, size, name)
    pos = [t for n in q_rows for t in range(n)]
    for got, up, raw in ((d_q_raw, d_e, host(q_raw)), (d_k_raw, d_r[:, None], host(k_raw))):
        want = O.norm_rope_backward(raw, up, pos, None, 0.0, f, True, by)[0]
        check_bf16(got, want, amplitude(up, ROT, True, by), "rotation's gradient")
    replay(step, step)
