"""Norms, rotation, cache append and paged attention without a GPU: refusals at the C ABI and in the binding, the
frequency helper, and the oracle's own functions against independent forms."""
from __future__ import annotations

import ctypes
import math

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa

INV, UNS, WS = msa.MSA_ERR_INVALID, msa.MSA_ERR_UNSUPPORTED, msa.MSA_ERR_WORKSPACE


def _seqs(**kw):
    base = dict(num_seqs=1, total_q_rows=100, total_kv_rows=128, max_q_rows=100, max_kv_len=100,
                q_offsets=8, kv_starts=8, kv_lens=8)   # fake non-null pointers, never dereferenced
    base.update(kw)
    return msa.MsaSeqsC(**base)


def _paged(**kw):
    return _seqs(**{**dict(block_table=8, block_table_stride=2, page_size=64), **kw})


def _rope(rot=64, inter=0, scale=1.0, freq=8):
    return msa.MsaRopeC(rot, inter, scale, freq)


# ------------------------------------------------------------------ norm and rotation
NORM_BAD = [
    (dict(d=96), UNS), (dict(d=0), INV), (dict(H=-1), INV), (dict(H=0, K=0), INV), (dict(H=1025), UNS),
    (dict(q=None), INV), (dict(k=None), INV), (dict(q_out=None), INV), (dict(k_out=None), INV),
    (dict(q_stride=8 * 128 - 4), INV), (dict(k_stride=2 * 128 + 2), UNS), (dict(q=12), UNS), (dict(k_out=20), UNS),
    (dict(eps=-1e-6), INV), (dict(eps=math.nan), INV), (dict(eps=math.inf), INV),
    (dict(rope=_rope(rot=136)), INV), (dict(rope=_rope(rot=-8)), INV), (dict(rope=_rope(rot=20)), UNS),
    (dict(rope=_rope(freq=0)), INV), (dict(rope=_rope(scale=math.inf)), INV), (dict(rope=_rope(scale=math.nan)), INV),
    (dict(seqs=_seqs(num_seqs=0)), INV), (dict(seqs=_seqs(q_offsets=0)), INV), (dict(seqs=_seqs(max_q_rows=101)), INV),
]


@pytest.mark.parametrize("kw,want", NORM_BAD)
def test_norm_rope_refuses(kw, want):
    a = dict(q=8, q_stride=8 * 128, k=8, k_stride=2 * 128, seqs=_seqs(), H=8, K=2, d=128, eps=1e-6, rope=_rope(), q_out=8,
             k_out=8)
    a.update(kw)
    L = msa.lib()
    s, r = ctypes.byref(a["seqs"]), ctypes.byref(a["rope"])
    tail = (s, a["H"], a["K"], a["d"], 8, 8, a["eps"], r, a["q_out"], a["k_out"], None)
    assert L.msa_qk_norm_rope(a["q"], a["q_stride"], a["k"], a["k_stride"], *tail) == want
    assert L.msa_qk_norm_rope_fp8(a["q"], a["q_stride"], a["k"], a["k_stride"], 1.0, 1.0, *tail) == want


@pytest.mark.parametrize("scale", [0.0, -1.0, math.inf, math.nan])
def test_code_scales_are_finite_and_positive(scale):
    L, s = msa.lib(), ctypes.byref(_seqs())
    p = ctypes.byref(_paged())
    for pair in ((scale, 1.0), (1.0, scale)):
        assert L.msa_qk_norm_rope_fp8(8, 1024, 8, 256, *pair, s, 8, 2, 128, None, None, 0.0, None, 8, 8, None) == INV
        assert L.msa_kv_append_fp8(8, 256, 8, 256, *pair, None, 0, s, 2, 128, 0, None, None, 0.0, None, None, 8, 8, None,
                                   None) == INV
        assert L.msa_dense_attn_paged_fp8(8, 8, 8, 1.0, *pair, p, 8, 2, 128, 0.1, 8, 8, 8, 1 << 30, None) == INV
    assert L.msa_dense_attn_paged_fp8(8, 8, 8, scale, 1.0, 1.0, p, 8, 2, 128, 0.1, 8, 8, 8, 1 << 30, None) == INV


@pytest.mark.parametrize("scale", [1e-40, 2.0 ** 127])
def test_code_scales_have_a_normal_reciprocal(scale):
    """1e-40 has an infinite one in fp32: a zero would become NaN."""
    L, s = msa.lib(), ctypes.byref(_seqs())
    for pair in ((scale, 1.0), (1.0, scale)):
        assert L.msa_qk_norm_rope_fp8(8, 1024, 8, 256, *pair, s, 8, 2, 128, None, None, 0.0, None, 8, 8, None) == INV
        assert L.msa_kv_append_fp8(8, 256, 8, 256, *pair, None, 0, s, 2, 128, 0, None, None, 0.0, None, None, 8, 8, None,
                                   None) == INV


def test_no_rows_need_no_tensors():
    L, s = msa.lib(), ctypes.byref(_seqs(total_q_rows=0, max_q_rows=0))
    assert L.msa_qk_norm_rope(None, 0, None, 0, s, 8, 2, 128, None, None, 0.0, None, None, None, None) == msa.MSA_OK
    assert L.msa_kv_append(None, 0, None, 0, None, 0, s, 2, 128, 0, None, None, 0.0, None, None, None, None, None,
                           None) == msa.MSA_OK
    p = ctypes.byref(_paged(total_q_rows=0, max_q_rows=0))
    assert L.msa_dense_attn_paged(None, None, None, p, 8, 2, 128, 0.1, None, None, None, 0, None) == msa.MSA_OK


BACK_BAD = [
    (dict(q=None), INV), (dict(g=None), INV), (dict(d_q=None), INV), (dict(d_stride=8 * 128 - 4), INV),
    (dict(d_stride=8 * 128 + 2), UNS), (dict(g=12), UNS), (dict(ws=None), WS), (dict(ws_bytes=64), WS),
    (dict(qw=None), INV),                                  # a weight's gradient without the weight
    (dict(d=32), UNS), (dict(rope=_rope(rot=12)), UNS), (dict(eps=-1.0), INV),
]


@pytest.mark.parametrize("kw,want", BACK_BAD)
def test_norm_rope_backward_refuses(kw, want):
    a = dict(q=8, g=8, d_q=8, d_stride=8 * 128, ws=8, ws_bytes=1 << 30, qw=8, d=128, rope=_rope(), eps=1e-6)
    a.update(kw)
    L, s = msa.lib(), ctypes.byref(_seqs())
    st = L.msa_qk_norm_rope_backward(a["q"], 8 * 128, 8, 2 * 128, a["g"], 8, s, 8, 2, a["d"], a["qw"], 8, a["eps"],
                                     ctypes.byref(a["rope"]), a["d_q"], a["d_stride"], 8, 2 * 128, 8, 8, a["ws"], a["ws_bytes"],
                                     None)
    assert st == want


def test_backward_workspace():
    L = msa.lib()
    n = L.msa_qk_norm_rope_backward_workspace_size(ctypes.byref(_seqs()), 8, 2, 128)
    assert n == 4 * 2 * 128 * 100                          # a partial for each of 100 rows
    big = _seqs(total_q_rows=1 << 20, max_q_rows=1 << 20, max_kv_len=1 << 20)
    assert L.msa_qk_norm_rope_backward_workspace_size(ctypes.byref(big), 8, 2, 64) == 4 * 2 * 64 * 1024
    assert L.msa_qk_norm_rope_backward_workspace_size(ctypes.byref(_seqs()), 8, 2, 100) == 0


# ------------------------------------------------------------------ append
APPEND_BAD = [
    (dict(d=64), UNS), (dict(H=65), UNS), (dict(H=0), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(kc=None), INV),
    (dict(vc=None), INV), (dict(ic=None), INV), (dict(i=None), INV), (dict(d_idx=96), UNS), (dict(vc=12), UNS),
    (dict(k_stride=128), INV), (dict(v_stride=2 * 128 + 1), UNS), (dict(i_stride=63), INV), (dict(eps=-1.0), INV),
    (dict(index_rope=_rope(rot=72)), INV), (dict(rope=_rope(rot=4)), UNS),
    (dict(seqs=_paged(page_size=48)), INV), (dict(seqs=_paged(page_size=8, block_table_stride=20)), INV),
    (dict(seqs=_paged(page_size=16384, total_kv_rows=1 << 20)), INV), (dict(seqs=_paged(block_table_stride=1)), INV),
]


@pytest.mark.parametrize("kw,want", APPEND_BAD)
def test_append_refuses(kw, want):
    a = dict(k=8, k_stride=256, v=8, v_stride=256, i=8, i_stride=64, seqs=_paged(), H=2, d=128, d_idx=64, eps=0.0, rope=_rope(),
             index_rope=_rope(32), kc=8, vc=8, ic=8)
    a.update(kw)
    L = msa.lib()
    tail = (a["i"], a["i_stride"], ctypes.byref(a["seqs"]), a["H"], a["d"], a["d_idx"], 8, 8, a["eps"],
            ctypes.byref(a["rope"]), ctypes.byref(a["index_rope"]), a["kc"], a["vc"], a["ic"], None)
    assert L.msa_kv_append(a["k"], a["k_stride"], a["v"], a["v_stride"], *tail) == want
    assert L.msa_kv_append_fp8(a["k"], a["k_stride"], a["v"], a["v_stride"], 1.0, 1.0, *tail) == want


# ------------------------------------------------------------------ paged attention
PAGED_BAD = [
    (dict(seqs=_seqs()), UNS),                             # contiguous
    (dict(seqs=_paged(page_size=96)), INV), (dict(seqs=_paged(page_size=8, block_table_stride=20)), INV),
    (dict(seqs=_paged(page_size=16384, total_kv_rows=1 << 20)), INV), (dict(seqs=_paged(block_table_stride=1)), INV),
    (dict(seqs=_paged(total_kv_rows=1 << 31)), UNS), (dict(d=64), UNS), (dict(H=6, K=4), INV), (dict(H=34, K=2), UNS),
    (dict(H=65, K=65), UNS), (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(o=None), INV),
    (dict(lse=None), INV), (dict(q=8), UNS), (dict(k=24), UNS), (dict(v=40), UNS), (dict(o=56), UNS),
]


@pytest.mark.parametrize("kw,want", PAGED_BAD)
def test_dense_paged_refuses(kw, want):
    a = dict(q=16, k=16, v=16, seqs=_paged(), H=8, K=2, d=128, o=16, lse=8)
    a.update(kw)
    L, s = msa.lib(), ctypes.byref(a["seqs"])
    tail = (s, a["H"], a["K"], a["d"], 0.1, a["o"], a["lse"], 8, 1 << 40, None)
    assert L.msa_dense_attn_paged(a["q"], a["k"], a["v"], *tail) == want
    assert L.msa_dense_attn_paged_fp8(a["q"], a["k"], a["v"], 1.0, 1.0, 1.0, *tail) == want
    if set(kw) <= {"seqs", "d", "H", "K"}:
        assert L.msa_dense_attn_paged_workspace_size(s, a["H"], a["K"], a["d"]) == 0


def test_dense_paged_workspace():
    """Parts of two tiles for every CTA of a split call; none where the keys are not split; too small a one is refused
    before anything is launched."""
    L = msa.lib()
    long = _paged(num_seqs=4, total_q_rows=4, max_q_rows=1, max_kv_len=65536, block_table_stride=1024, total_kv_rows=1 << 20)
    need = L.msa_dense_attn_paged_workspace_size(ctypes.byref(long), 64, 8, 128)
    assert need == 4 * 2 * 256 * 32 * 129
    call = lambda ws, n: L.msa_dense_attn_paged(16, 16, 16, ctypes.byref(long), 64, 8, 128, 0.1, 16, 16, ws, n, None)  # noqa: E731
    assert call(16, need - 1) == WS and call(None, need) == WS
    short = _paged(num_seqs=4, total_q_rows=4, max_q_rows=1, max_kv_len=128)
    assert L.msa_dense_attn_paged_workspace_size(ctypes.byref(short), 64, 8, 128) == 0
    many = _paged(num_seqs=300, total_q_rows=300, max_q_rows=1, max_kv_len=65536, block_table_stride=1024, total_kv_rows=1 << 20)
    assert L.msa_dense_attn_paged_workspace_size(ctypes.byref(many), 64, 8, 128) == 0


# ------------------------------------------------------------------ binding
def _cpu_seqs(rows=4):
    return msa.Seqs([rows], [rows], [0], rows, "cpu")


def test_binding_checks_shapes_and_types():
    s, bf = _cpu_seqs(), torch.bfloat16
    q, k = torch.zeros((4, 2, 128), dtype=bf), torch.zeros((4, 1, 128), dtype=bf)
    rope = msa.Rope(torch.ones(16, dtype=torch.float64))
    with pytest.raises(TypeError):
        msa.qk_norm_rope(q.float(), k, s, rope)
    with pytest.raises(ValueError):
        msa.qk_norm_rope(q[:3], k, s, rope)
    with pytest.raises(ValueError):
        msa.qk_norm_rope(q, k[..., :64], s, rope)
    with pytest.raises(ValueError):
        msa.qk_norm_rope(q.transpose(1, 2).contiguous().transpose(1, 2), None, s, rope)    # heads not contiguous
    with pytest.raises(TypeError):
        msa.qk_norm_rope(q, k, s, rope, torch.ones(128, dtype=bf))
    with pytest.raises(ValueError):
        msa.qk_norm_rope(q, k, s, rope, torch.ones(64))
    with pytest.raises(TypeError):
        msa.qk_norm_rope_fp8(q, k, (1.0, 1.0), s, rope, q_out=torch.zeros_like(q))
    with pytest.raises(TypeError):
        msa.Rope(torch.ones(16))
    with pytest.raises(ValueError):
        msa.Rope(torch.ones((2, 8), dtype=torch.float64))
    with pytest.raises(ValueError):
        msa.qk_norm_rope_backward(None, None, q, None, s, rope, torch.ones(128))           # the norm needs q
    with pytest.raises(ValueError):
        msa.qk_norm_rope_backward(q, None, None, None, s, rope)
    with pytest.raises(ValueError):
        msa.qk_norm_rope_backward(q, None, q, None, s, rope, d_q_weight=torch.ones(128))
    with pytest.raises(ValueError):
        msa.kv_append(k, q, s, rope, k, k)
    with pytest.raises(ValueError):
        msa.kv_append(k, k, s, rope, k, k, index_k=torch.zeros((4, 64), dtype=bf))
    with pytest.raises(TypeError):
        msa.kv_append_fp8(k, k, (1.0, 1.0), s, rope, k, k)
    with pytest.raises(TypeError):
        msa.dense_attn_paged_fp8(q, k, k, (1.0, 1.0, 1.0), s)
    with pytest.raises(ValueError):
        msa.dense_attn_paged(q, k[:3], k[:3], s)


def test_workspace_is_aligned_and_on_the_device():
    L = msa.lib()
    long = _paged(num_seqs=4, total_q_rows=4, max_q_rows=1, max_kv_len=65536, block_table_stride=1024, total_kv_rows=1 << 20)
    assert L.msa_dense_attn_paged(16, 16, 16, ctypes.byref(long), 64, 8, 128, 0.1, 16, 16, 24, 1 << 40, None) == UNS
    assert L.msa_qk_norm_rope_backward(8, 1024, 8, 256, 8, 8, ctypes.byref(_seqs()), 8, 2, 128, 8, 8, 0.0,
                                       ctypes.byref(_rope()), 8, 1024, 8, 256, 8, 8, 12, 1 << 30, None) == UNS
    s, q = _cpu_seqs(), torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    for ws in (torch.empty(1 << 20, dtype=torch.uint8, device="meta"), torch.zeros((4, 1 << 10), dtype=torch.uint8)[:, ::2]):
        with pytest.raises(ValueError, match="workspace"):
            msa.dense_attn_paged(q, q, q, s, workspace=ws)
        with pytest.raises(ValueError, match="workspace"):
            msa.qk_norm_rope_backward(q, None, q, None, s, None, torch.ones(128), workspace=ws)


def test_rope_frequencies():
    f, m = msa.rope_frequencies(64, 10000.0)
    assert f.dtype == torch.float64 and m == 1.0
    assert torch.allclose(f, torch.tensor([10000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64), rtol=1e-14)
    lin, m = msa.rope_frequencies(64, 10000.0, "linear", 4.0)
    assert m == 1.0 and torch.equal(lin * 4, f)
    ntk, m = msa.rope_frequencies(64, 10000.0, "ntk", 4.0)
    assert m == 1.0 and ntk[0] == 1 and abs(float(ntk[-1] * 4 / f[-1]) - 1) < 1e-12 and bool((ntk <= f).all())
    part, m = msa.rope_frequencies(64, 10000.0, "by_parts", 4.0, trained_len=4096)
    assert abs(m - (0.1 * math.log(4.0) + 1)) < 1e-15
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(part[turns > 32], f[turns > 32]) and torch.allclose(part[turns < 1] * 4, f[turns < 1], rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    keep = (turns[mid] - 1) / 31
    assert mid.any() and torch.allclose(part[mid], f[mid] * (keep + (1 - keep) / 4), rtol=1e-14)
    same, m = msa.rope_frequencies(64, 10000.0, "by_parts", 1.0, trained_len=4096)
    assert m == 1.0 and torch.allclose(same, f, rtol=1e-15)
    for bad in (dict(rot_dim=20), dict(rot_dim=0), dict(rot_dim=64, base=1.0), dict(rot_dim=64, factor=0.5),
                dict(rot_dim=64, scaling="cubic"), dict(rot_dim=64, scaling="by_parts", factor=2.0),
                dict(rot_dim=64, factor=math.inf, scaling="linear")):
        with pytest.raises(ValueError):
            msa.rope_frequencies(**bad)


# ------------------------------------------------------------------ the oracle's functions
@pytest.mark.parametrize("inter", [False, True])
def test_oracle_rotation_is_a_complex_product(inter):
    rng = np.random.default_rng(0)
    x, f, pos = rng.standard_normal((5, 2, 16)), rng.uniform(0, 1, 4), [0, 1, 7, 1000, 12345]
    y = O.norm_rope(x, pos, None, 0.0, f, inter, 1.3)
    a = np.arange(0, 8, 2) if inter else np.arange(4)
    b = a + (1 if inter else 4)
    z = (x[..., a] + 1j * x[..., b]) * 1.3 * np.exp(1j * np.outer(pos, f))[:, None]
    assert np.allclose(y[..., a], z.real, atol=1e-12) and np.allclose(y[..., b], z.imag, atol=1e-12)
    assert np.array_equal(y[..., 8:], x[..., 8:])


def test_oracle_rotation_keeps_distances():
    """Products of turned queries and keys depend on the difference of their positions alone."""
    rng = np.random.default_rng(1)
    q, k, f = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64)), rng.uniform(0, 1, 32)
    dot = lambda i, j: float((O.norm_rope(q, [i], None, 0, f) * O.norm_rope(k, [j], None, 0, f)).sum())  # noqa: E731
    assert abs(dot(5, 3) - dot(1005, 1003)) < 1e-9 and abs(dot(5, 3) - dot(5, 4)) > 1e-3


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_oracle_backward_matches_autograd(inter, norm):
    rng = np.random.default_rng(2)
    x, g, f, pos = rng.standard_normal((4, 3, 24)), rng.standard_normal((4, 3, 24)), rng.uniform(0, 1, 8), [3, 0, 50, 9]
    w = rng.standard_normal(24) if norm else None
    dx, dw = O.norm_rope_backward(x, g, pos, w, 1e-3, f, inter, 0.8)
    xt = torch.from_numpy(x).requires_grad_()
    n = xt
    if norm:
        wt = torch.from_numpy(w).requires_grad_()
        n = xt * torch.rsqrt((xt ** 2).mean(-1, keepdim=True) + 1e-3) * wt
    ang = torch.tensor(pos, dtype=torch.float64)[:, None, None] * torch.from_numpy(f)
    c, s = 0.8 * ang.cos(), 0.8 * ang.sin()
    u, v = (n[..., 0:16:2], n[..., 1:16:2]) if inter else (n[..., :8], n[..., 8:16])
    a, b = u * c - v * s, v * c + u * s
    y = torch.cat(((torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)), n[..., 16:]), -1)
    assert np.allclose(y.detach().numpy(), O.norm_rope(x, pos, w, 1e-3, f, inter, 0.8), atol=1e-12)
    y.backward(torch.from_numpy(g))
    assert np.allclose(dx, xt.grad.numpy(), atol=1e-12)
    assert (dw is None) == (not norm) and (dw is None or np.allclose(dw, wt.grad.numpy(), atol=1e-12))
