"""msa_qk_norm_rope, its E4M3 form and its backward against the float64 oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa
from tests.operators_util import (F32, BF16_HALF, amplitude, bf16, check_bf16, check_codes, dev, host, padded_seqs,
                                  positions, replay, rope_pair)

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


# name, dim, H, K, q_rows, kv_lens, rot, interleaved, norm, scale, rows behind the last sequence, columns of a wider tensor
CASES = [
    ("one_row", 128, 8, 2, [1], [1], 128, False, True, 1.0, 0, False),
    ("one_head", 64, 1, 0, [1], [70], 64, True, True, 1.0, 0, False),
    ("docs", 128, 6, 3, [33, 0, 1, 70], [33, 5, 1, 70], 64, False, True, 1.0, 0, True),
    ("pairs_in_part", 128, 5, 1, [17, 40], [400, 41], 24, True, True, 1.3, 3, True),
    ("half_in_part", 128, 4, 4, [50], [50], 24, False, True, 0.7, 7, False),
    ("index", 64, 8, 1, [129], [129], 32, False, True, 1.0, 0, False),
    ("index_rotation_only", 64, 4, 1, [65, 64], [3000, 64], 64, True, False, 1.1, 0, True),
    ("norm_only", 128, 16, 2, [31], [31], 0, False, True, 1.0, 2, False),
    ("smallest_part", 64, 3, 2, [9], [9], 8, False, False, 1.0, 0, False),
    ("far", 128, 2, 1, [40], [1048576], 128, False, True, 1.0, 0, False),
    ("far_pairs", 64, 2, 1, [3, 5], [2000000000, 999999], 64, True, False, 1.0, 0, False),
    ("decode_batch", 128, 64, 8, [1] * 70, [100 + 37 * i for i in range(70)], 64, False, True, 1.0, 2, True),
    ("many_rows", 128, 1, 1, [9000, 20000], [9000, 20000], 16, False, True, 1.0, 0, False),
    ("many_rows_index", 64, 1, 0, [70001], [70001], 16, True, True, 1.0, 5, False),
]


def _make(case):
    name, D, H, K, q_rows, kv_lens, rot, inter, norm, scale, pad, wide = case
    rng = np.random.default_rng(sum(map(ord, name)))
    T = sum(q_rows) + pad
    x = {"q": bf16(rng.standard_normal((T, H, D)) * 3), "k": bf16(rng.standard_normal((T, K, D)))}
    x["q"][0, 0] = 0.0                                     # a head of zeros
    w = {n: (1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if norm else None for n in ("q", "k")}
    seqs = padded_seqs(q_rows, kv_lens, pad)
    f, rope = rope_pair(rot, D, inter, scale)
    d = {}
    if wide:                                               # columns of one tensor, rows further apart than they are long
        joint = torch.zeros((T, (H + K) * D + 12), dtype=torch.bfloat16, device="cuda")
        d["q"], d["k"] = joint[:, 4:4 + H * D].view(T, H, D), joint[:, 4 + H * D:4 + (H + K) * D].view(T, K, D)
        for n in ("q", "k"):
            d[n].copy_(dev(x[n]))
    else:
        d = {n: dev(x[n]) for n in ("q", "k")}
    wd = {n: None if w[n] is None else torch.from_numpy(w[n]).cuda() for n in w}
    return x, w, d, wd, seqs, f, rope, positions(q_rows, kv_lens), rng


def _normed(x, w):
    return x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * w


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_forward(case):
    name, D, H, K, q_rows, kv_lens, rot, inter, norm, scale, pad, wide = case
    x, w, d, wd, seqs, f, rope, pos, rng = _make(case)
    T, n = sum(q_rows) + pad, sum(q_rows)
    out = {m: torch.full((T, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for m, h in (("q", H), ("k", K))}
    k = d["k"] if K else None
    msa.qk_norm_rope(d["q"], k, seqs, rope, wd["q"], wd["k"] if K else None, EPS, q_out=out["q"], k_out=out["k"] if K else None)
    for m in ("q", "k") if K else ("q",):
        pick = np.arange(n) if n * x[m].shape[1] < 3000 else np.unique(np.r_[0:40, n - 40:n, rng.integers(0, n, 300)])
        ref = O.norm_rope(x[m][pick], [pos[i] for i in pick], w[m], EPS, f, inter, scale)
        check_bf16(host(out[m])[pick], ref, amplitude(_normed(x[m][pick], w[m]), rot, inter, scale), f"{name} {m}")
        assert (out[m][n:] == 7.0).all()                   # rows behind the last sequence
    if norm:
        assert (out["q"][0, 0] == 0).all()
    # the same bits from newly allocated outputs, and into the inputs themselves
    q2, k2 = msa.qk_norm_rope(d["q"], k, seqs, rope, wd["q"], wd["k"] if K else None, EPS)
    assert torch.equal(q2[:n], out["q"][:n]) and (k is None or torch.equal(k2[:n], out["k"][:n]))
    qi, ki = d["q"].clone().contiguous(), d["k"].clone().contiguous()
    msa.qk_norm_rope(qi, ki if K else None, seqs, rope, wd["q"], wd["k"] if K else None, EPS, q_out=qi, k_out=ki if K else None)
    assert torch.equal(qi[:n], out["q"][:n]) and torch.equal(ki[:n], out["k"][:n])
    assert torch.equal(qi[n:], d["q"][n:])


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_codes(case):
    name, D, H, K, q_rows, kv_lens, rot, inter, norm, scale, pad, wide = case
    x, w, d, wd, seqs, f, rope, pos, rng = _make(case)
    n = sum(q_rows)
    scales = (2.0 ** -4, 0.013)                            # the second sends the largest values past 448
    q, k = msa.qk_norm_rope_fp8(d["q"], d["k"] if K else None, scales, seqs, rope, wd["q"], wd["k"] if K else None, EPS)
    for m, got, s in (("q", q, scales[0]), ("k", k, scales[1]))[:2 if K else 1]:
        pick = np.arange(n) if n * x[m].shape[1] < 3000 else np.unique(rng.integers(0, n, 300))
        ref = O.norm_rope(x[m][pick], [pos[i] for i in pick], w[m], EPS, f, inter, scale)
        check_codes(got.cpu().numpy()[pick], ref, s, amplitude(_normed(x[m][pick], w[m]), rot, inter, scale), f"{name} {m}")


def test_codes_saturate_and_keep_nan():
    x = torch.tensor([500.0, -1e30, 448.0, 464.0, 0.0, -0.0, 2.0 ** -10, 1e-9] * 8, device="cuda").to(torch.bfloat16)
    x = x.view(1, 1, 64).clone()
    x[0, 0, 63] = float("nan")
    q, _ = msa.qk_norm_rope_fp8(x, None, (1.0, 1.0), padded_seqs([1], [1]), None)
    got = q.view(torch.float8_e4m3fn).float().flatten().tolist()
    assert got[:4] == [448.0, -448.0, 448.0, 448.0] and got[4] == 0 and got[6] == 0.0
    assert got[63] != got[63]


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_backward(case):
    name, D, H, K, q_rows, kv_lens, rot, inter, norm, scale, pad, wide = case
    x, w, d, wd, seqs, f, rope, pos, rng = _make(case)
    T, n = sum(q_rows) + pad, sum(q_rows)
    g = {m: bf16(rng.standard_normal(x[m].shape)) for m in ("q", "k")}
    for m in ("q", "k"):                                   # what lies behind the last sequence takes no part
        g[m][n:] = 1e6
    gd = {m: dev(g[m]) for m in ("q", "k")}
    joint = torch.full((T, (H + K) * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    dx = {"q": joint[:, :H * D].view(T, H, D), "k": joint[:, H * D:(H + K) * D].view(T, K, D)}
    args = (d["q"], d["k"] if K else None, gd["q"], gd["k"] if K else None, seqs, rope, wd["q"], wd["k"] if K else None, EPS)
    _, _, dqw, dkw = msa.qk_norm_rope_backward(*args, d_q=dx["q"], d_k=dx["k"] if K else None)
    dw = {"q": dqw, "k": dkw}
    assert (joint[n:] == 7.0).all() and (joint[:, (H + K) * D:] == 7.0).all()
    for m in ("q", "k") if K else ("q",):
        heads = x[m].shape[1]
        small = n * heads < 3000
        pick = np.arange(n) if small else np.unique(np.r_[0:40, n - 40:n, rng.integers(0, n, 300)])
        p = [pos[i] for i in pick]
        ref, refw = O.norm_rope_backward(x[m][pick], g[m][pick], p, w[m], EPS, f, inter, scale)
        amp = amplitude(np.abs(g[m][pick]), rot, inter, scale)
        if w[m] is not None:
            rms = np.sqrt((x[m][pick] ** 2).mean(-1, keepdims=True) + EPS)
            u = np.abs(x[m][pick]) / rms
            hw = amp * np.abs(w[m])
            amp_w = (amp * u).sum((0, 1))
            amp = (hw + u * (hw * u).mean(-1, keepdims=True)) / rms
        check_bf16(host(dx[m])[pick], ref, amp, f"{name} d{m}")
        if w[m] is not None and small:
            # sums in fp32: a lane's heads in sequence, 32 lane groups, the CTAs in sixteenths: at most n * heads + 64 steps
            err = np.abs(host(dw[m]) - refw)
            assert (err <= (F32 + (n * heads + 64) * 2.0 ** -24) * amp_w).all(), f"{name} d{m}_weight"
        elif w[m] is not None:
            # all rows in float64 on the GPU, the rotation as a product of complex numbers
            h = gd[m][:n].double()
            a = torch.tensor(pos, dtype=torch.float64, device="cuda")[:, None, None] * torch.from_numpy(f).cuda()
            z = h[..., :rot].reshape(n, heads, rot // 2, 2) if inter else h[..., :rot].reshape(n, heads, 2, -1).transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * torch.polar(torch.full_like(a, scale), -a))
            z = z if inter else z.transpose(2, 3)
            h = torch.cat((z.reshape(n, heads, rot), h[..., rot:]), -1)
            xx = d[m][:n].double()
            uu = xx / ((xx * xx).mean(-1, keepdim=True) + EPS).sqrt()
            refw, size = (h * uu).sum((0, 1)), (gd[m][:n].double().abs() * 2 * uu.abs()).sum((0, 1))
            steps = n * heads / 1024 + 64 + 80             # heads of a lane, groups, CTAs
            assert bool(((dw[m].double() - refw).abs() <= (F32 + steps * 2.0 ** -24) * size).all()), f"{name} d{m}_weight"
        else:
            assert dw[m] is None
    again = msa.qk_norm_rope_backward(*args)
    assert torch.equal(again[0][:n], dx["q"][:n])
    for a, b in ((again[2], dqw), (again[3], dkw)):
        assert a is b is None or torch.equal(a, b)         # the same bits


def test_backward_against_differences():
    """d x and d weight along random directions against central differences of the forward kernel's own formula in
    64 bits (the oracle's), for a case with everything on."""
    rng = np.random.default_rng(5)
    q_rows, kv_lens, D = [6], [900], 64
    x, g, w = bf16(rng.standard_normal((6, 2, D))), bf16(rng.standard_normal((6, 2, D))), 1 + 0.2 * rng.standard_normal(D)
    w = w.astype(np.float32).astype(np.float64)
    f, rope = rope_pair(32, D, True, 1.2)
    pos = positions(q_rows, kv_lens)
    dq, _, dw, _ = msa.qk_norm_rope_backward(dev(x), None, dev(g), None, padded_seqs(q_rows, kv_lens), rope,
                                             torch.from_numpy(w.astype(np.float32)).cuda(), None, EPS)
    e = 1e-4
    for _ in range(4):
        vx, vw = rng.standard_normal(x.shape), rng.standard_normal(w.shape)
        loss = lambda t: (g * O.norm_rope(x + t * vx, pos, w + t * vw, EPS, f, True, 1.2)).sum()  # noqa: E731
        want = (loss(e) - loss(-e)) / (2 * e)
        got = (host(dq) * vx).sum() + (host(dw) * vw).sum()
        # bf16 d x: half a step each, independent of vx's sign at worst; differences are exact to e^2
        tol = BF16_HALF * (np.abs(host(dq)) * np.abs(vx)).sum() + 1e-4 * (np.abs(host(dw) * vw).sum() + 1)
        assert abs(got - want) <= tol


def test_gradient_may_replace_its_own_input():
    case = CASES[5]
    x, w, d, wd, seqs, f, rope, pos, rng = _make(case)
    gq, gk = dev(bf16(rng.standard_normal(x["q"].shape))), dev(bf16(rng.standard_normal(x["k"].shape)))
    want = msa.qk_norm_rope_backward(d["q"], d["k"], gq, gk, seqs, rope, wd["q"], wd["k"], EPS)
    a, b = gq.clone(), gk.clone()
    msa.qk_norm_rope_backward(d["q"], d["k"], a, b, seqs, rope, wd["q"], wd["k"], EPS, d_q=a, d_k=b)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_one_weight_only():
    case = CASES[2]
    x, w, d, wd, seqs, f, rope, pos, rng = _make(case)
    gq, gk = dev(bf16(rng.standard_normal(x["q"].shape))), dev(bf16(rng.standard_normal(x["k"].shape)))
    both = msa.qk_norm_rope_backward(d["q"], d["k"], gq, gk, seqs, rope, wd["q"], wd["k"], EPS)
    none = msa.qk_norm_rope_backward(None, None, gq, gk, seqs, rope)
    q, k, dqw, dkw = msa.qk_norm_rope_backward(None, d["k"], gq, gk, seqs, rope, None, wd["k"], EPS)
    assert dqw is None and torch.equal(q, none[0]) and torch.equal(k, both[1]) and torch.equal(dkw, both[3])
    _, k, _, dkw = msa.qk_norm_rope_backward(None, d["k"], None, gk, seqs, rope, None, wd["k"], EPS)
    assert torch.equal(k, both[1]) and torch.equal(dkw, both[3])


def test_no_rows():
    seqs = padded_seqs([0, 0], [4, 7])
    q = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(128, device="cuda")
    assert msa.qk_norm_rope(q, None, seqs, None, w)[0].shape == q.shape
    d_q, _, dw, _ = msa.qk_norm_rope_backward(q, None, q, None, seqs, None, w)
    assert d_q.shape == q.shape and bool((dw == 0).all())


def test_captured_and_other_stream():
    case = CASES[11]
    x, w, d, wd, seqs, f, rope, pos, rng = _make(case)
    g = [dev(bf16(rng.standard_normal(x[m].shape))) for m in ("q", "k")]
    n = sum(case[4])
    def fwd():
        q, k = msa.qk_norm_rope(d["q"], d["k"], seqs, rope, wd["q"], wd["k"], EPS)
        return q[:n], k[:n]
    ws = torch.empty(msa.qk_norm_rope_backward_workspace_size(seqs, 64, 8, 128), dtype=torch.uint8, device="cuda")
    def bwd():
        a, b, c, e = msa.qk_norm_rope_backward(d["q"], d["k"], g[0], g[1], seqs, rope, wd["q"], wd["k"], EPS, workspace=ws)
        return a[:n], b[:n], c, e
    want = fwd()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = fwd()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    replay(fwd, fwd)
    replay(bwd, bwd)
