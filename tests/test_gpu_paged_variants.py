"""Every form of msa_dense_attn_paged (paged_cases.py) against the float64 oracle, long runs of page places, and LSE
where the scores are exact.

Bars as in test_gpu_dense_paged.py; the pools are NaN wherever no sequence's key lies.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa, synth
from tests.operators_util import padded_seqs, page_table
from tests.paged_cases import LONG, VARIANTS
from tests.test_gpu_dense_paged import LSE_TOL, SCALES, _make, _reference
from tests.util import check_outputs, from_dev_bits, to_dev

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _call(fp8, q, k, v, seqs, **kw):
    return msa.dense_attn_paged_fp8(q, k, v, SCALES, seqs, **kw) if fp8 else msa.dense_attn_paged(q, k, v, seqs, **kw)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", VARIANTS, ids=[c[0] for c in VARIANTS])
def test_forms(case, fp8):
    name, _, split, q_rows, kv_lens, H_q, H_kv, page, pad = case
    x, d, seqs, lay, _ = _make((name, q_rows, kv_lens, H_q, H_kv, page, pad), fp8)
    n, T = sum(q_rows), sum(q_rows) + pad
    o = torch.full((T, H_q, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H_q), 7.0, device="cuda")
    size = msa.dense_attn_paged_workspace_size(seqs, H_q, H_kv, D)
    assert (size > 0) == split
    ws = torch.full((max(1, size),), 0xFF, dtype=torch.uint8, device="cuda")   # NaN where it is read unwritten
    _call(fp8, *d, seqs, out=o, lse=lse, workspace=ws)
    assert bool((o[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    o_ref, l_ref = _reference(None, x, lay, fp8, np.arange(n))
    stats = check_outputs(o[:n].float().cpu().numpy(), lse[:n].cpu().numpy(), o_ref, l_ref, name)
    assert stats[2] <= LSE_TOL, stats


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", LONG, ids=[c[0] for c in LONG])
def test_long_runs(case, fp8):
    name, _, split, q_rows, kv_lens, H_q, H_kv, page, _ = case
    rng = np.random.default_rng(sum(map(ord, name)))
    gen = torch.Generator(device="cuda").manual_seed(len(name))
    table, total, rows = page_table(rng, kv_lens, page)
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    used[torch.from_numpy(np.concatenate(rows)).cuda()] = True

    def draw(n):
        t = torch.randn((n, H_kv if n == total else H_q, D), dtype=torch.bfloat16, device="cuda", generator=gen)
        return (t.float() * 16).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else t

    q, k, v = draw(sum(q_rows)), draw(total), draw(total)
    k[~used], v[~used] = (0x7F, 0x7F) if fp8 else (float("nan"), float("nan"))
    seqs = padded_seqs(q_rows, kv_lens, total_kv=total, table=torch.from_numpy(table).cuda(), page=page)
    o, lse = _call(fp8, q, k, v, seqs)
    oh, lh = o.float().cpu().numpy(), lse.cpu().numpy()
    assert np.isfinite(oh).all() and np.isfinite(lh).all()
    # a few groups' heads of the longest sequence's first, middle and last rows, and of two others' last
    lay = O.Layout(q_rows, kv_lens, np.cumsum([0] + kv_lens)[:-1])
    long = int(np.argmax(kv_lens))
    a, b = lay.q_offsets[long], lay.q_offsets[long + 1]
    others = [lay.q_offsets[s + 1] - 1 for s in (0, len(q_rows) - 1) if s != long]
    pick = np.unique([a, (a + b) // 2, b - 1] + others)
    G = H_q // H_kv
    for g in sorted({0, H_kv // 2, H_kv - 1}):
        at = torch.from_numpy(np.concatenate(rows)).cuda()
        if fp8:
            bits = lambda t, s: synth.bf16_bits_from_f32((O.decode_fp8_e4m3(t.cpu().numpy()) * s).astype(np.float32))  # noqa: E731
        else:
            bits = lambda t, s: from_dev_bits(t)  # noqa: E731
        qb, kb, vb = bits(q[:, g * G:(g + 1) * G], SCALES[0]), bits(k[at, g:g + 1], SCALES[1]), bits(v[at, g:g + 1], SCALES[2])
        o_ref, l_ref = O.dense_causal_attention(qb, kb, vb, lay, rows=pick)
        stats = check_outputs(oh[pick, g * G:(g + 1) * G], lh[pick, g * G:(g + 1) * G], o_ref, l_ref, f"{name} group {g}")
        assert stats[2] <= LSE_TOL, stats


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [4, 8, 16, 40], ids=["few_rows", "two_waves", "four_waves", "eight_waves"])
def test_lse_of_exact_scores(rows, fp8):
    """Scores that fp32 holds whatever the order of their sum: LSE is then as good as its own arithmetic.

    q and k hold +-2^-e and +-1.5 2^-e, e = 0 .. 6: products are multiples of 2^-14 of at most 2.25, sums of 128 of them
    at most 288 < 2^9 and so exact in 24 bits.  With S = the largest |score| * scale of a row of n keys, in units of
    2^-24: the scale's two roundings 2 S; the exponents' (their offset S, themselves 2 S); a weight's own 2; its place in
    a sum of n terms n; the logarithm's, the offset's and the result's roundings 4 S + 6 ln n: 9 S + n + 2 + 6 ln n.
    """
    rng = np.random.default_rng(rows)
    kv_lens = [rows, rows + 1, 31 + rows, 65]
    q_rows = [min(rows, n) for n in kv_lens]
    H_q, H_kv, page, scale = 16, 2, 32, 0.125
    one = lambda s: rng.choice([-1.0, 1.0], s) * rng.choice([1.0, 1.5], s) * 2.0 ** -rng.integers(0, 7, s)  # noqa: E731
    q, k, v = (one((sum(m), h, D)) for m, h in ((q_rows, H_q), (kv_lens, H_kv), (kv_lens, H_kv)))
    table, total, at = page_table(rng, kv_lens, page)
    pools = [np.zeros((total, H_kv, D)) for _ in range(2)]
    for pool, x in zip(pools, (k, v)):
        pool[np.concatenate(at)] = x
    seqs = padded_seqs(q_rows, kv_lens, total_kv=total, table=torch.from_numpy(table).cuda(), page=page)
    assert msa.dense_attn_paged_workspace_size(seqs, H_q, H_kv, D) == 0
    if fp8:
        codes = [torch.from_numpy(t.astype(np.float32)).to(torch.float8_e4m3fn) for t in (q, *pools)]
        assert all(np.array_equal(c.float().numpy(), t) for c, t in zip(codes, (q, *pools)))
        _, lse = msa.dense_attn_paged_fp8(*(c.view(torch.uint8).cuda() for c in codes), (1.0, 1.0, 1.0), seqs, softmax_scale=scale)
    else:
        _, lse = msa.dense_attn_paged(*(to_dev(synth.bf16_bits_from_f32(t.astype(np.float32))) for t in (q, *pools)), seqs,
                                      softmax_scale=scale)
    lse = lse.double().cpu().numpy()
    lay = O.Layout(q_rows, kv_lens, np.cumsum([0] + kv_lens)[:-1])
    for r in range(sum(q_rows)):
        s, p = lay.locate(r)
        keys = k[lay.kv_starts[s]:lay.kv_starts[s] + p + 1]
        for h in range(H_q):
            z = keys[:, h // (H_q // H_kv)] @ q[r, h] * scale
            top, n = z.max(), p + 1
            ref = top + np.log(np.exp(z - top).sum())
            tol = 2.0 ** -24 * (9 * np.abs(z).max() + n + 2 + 6 * np.log(n))
            assert abs(lse[r, h] - ref) <= tol, (r, h, n, lse[r, h] - ref, tol)
