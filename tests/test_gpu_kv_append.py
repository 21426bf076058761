"""msa_kv_append and its E4M3 form: which cache rows are written, and what they hold, against the float64 oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa
from tests.operators_util import (amplitude, bf16, check_bf16, check_codes, dev, host, padded_seqs, page_table, positions,
                                  rope_pair)

pytestmark = pytest.mark.gpu
EPS = 1e-6
D = 128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


# name, H_kv, d_idx (0: no index keys), q_rows, kv_lens, page (0: contiguous), rot, index rot, interleaved, norm, rows behind
CASES = [
    ("one_token", 8, 64, [1], [1], 64, 64, 32, False, True, 0),
    ("one_head", 1, 0, [3], [70], 16, 128, 0, True, True, 0),
    ("decode", 4, 128, [1] * 67, [1 + 61 * i for i in range(67)], 64, 64, 64, False, True, 0),
    ("chunks", 4, 128, [33, 0, 129, 1], [33, 17, 1000, 200], 128, 64, 128, False, True, 5),
    ("small_pages", 2, 64, [100, 50], [163, 50], 16, 24, 8, True, False, 3),
    ("no_rotation", 3, 64, [20], [4096], 1024, 0, 0, False, True, 0),
    ("contiguous", 8, 64, [40, 1, 9], [40, 300, 64], 0, 64, 64, False, True, 2),
    ("many_rows", 1, 64, [5000, 20000], [5000, 70000], 256, 32, 32, False, True, 0),
]


def _make(case, fp8):
    name, H, d_idx, q_rows, kv_lens, page, rot, irot, inter, norm, pad = case
    rng = np.random.default_rng(sum(map(ord, name)))
    T = sum(q_rows) + pad
    x = {"k": bf16(rng.standard_normal((T, H, D))), "v": bf16(rng.standard_normal((T, H, D)))}
    if d_idx:
        x["i"] = bf16(rng.standard_normal((T, 1, d_idx)))
    w = {n: (1 + 0.3 * rng.standard_normal(x[n].shape[-1])).astype(np.float32) if norm and n != "v" else None for n in x}
    if page:
        table, total, rows = page_table(rng, kv_lens, page)
        seqs = padded_seqs(q_rows, kv_lens, pad, total_kv=total, table=torch.from_numpy(table).cuda(), page=page)
    else:
        starts = np.cumsum([5] + [n + 3 for n in kv_lens])[:-1].tolist()
        total = starts[-1] + kv_lens[-1] + 7
        rows = [s + np.arange(n) for s, n in zip(starts, kv_lens)]
        seqs = padded_seqs(q_rows, kv_lens, pad, kv_starts=starts, total_kv=total)
    to = np.concatenate([r[n - q:] for r, q, n in zip(rows, q_rows, kv_lens)])
    # k and v as columns of a joint tensor
    joint = torch.zeros((T, 2 * H * D + 4), dtype=torch.bfloat16, device="cuda")
    kd, vd = joint[:, :H * D].view(T, H, D), joint[:, H * D:2 * H * D].view(T, H, D)
    kd.copy_(dev(x["k"]))
    vd.copy_(dev(x["v"]))
    f, rope = rope_pair(rot, D, inter, 1.0)
    fi, irope = rope_pair(irot, d_idx, inter, 1.1)
    dtype = torch.uint8 if fp8 else torch.bfloat16
    caches = [torch.full((total, H, D), 3, dtype=dtype, device="cuda") for _ in range(2)]
    kw = dict(k_weight=None if w["k"] is None else torch.from_numpy(w["k"]).cuda(), eps=EPS)
    if d_idx:
        caches.append(torch.full((total, d_idx), 3, dtype=torch.bfloat16, device="cuda"))
        kw.update(index_k=dev(x["i"][:, 0]), index_k_cache=caches[2],
                  index_k_weight=None if w["i"] is None else torch.from_numpy(w["i"]).cuda(), index_rope=irope)
    return x, w, kd, vd, seqs, (f, rope, rot), (fi, irope, irot), to, caches, kw, positions(q_rows, kv_lens), inter, rng


def _check_turned(got, x, w, pos, f, rot, inter, scale, rng, what, code_scale=None):
    n = len(pos)
    pick = np.arange(n) if n * x.shape[1] < 3000 else np.unique(np.r_[0:40, n - 40:n, rng.integers(0, n, 300)])
    xs = x[pick]
    ref = O.norm_rope(xs, [pos[i] for i in pick], w, EPS, f, inter, scale)
    normed = xs if w is None else xs / np.sqrt((xs * xs).mean(-1, keepdims=True) + EPS) * w
    amp = amplitude(normed, rot, inter, scale)
    if code_scale is None:
        check_bf16(host(got)[pick], ref, amp, what)
    else:
        check_codes(got.cpu().numpy()[pick], ref, code_scale, amp, what)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_append(case, fp8):
    x, w, kd, vd, seqs, (f, rope, rot), (fi, _, irot), to, caches, kw, pos, inter, rng = _make(case, fp8)
    scales = (2.0 ** -5, 2.0 ** -6)
    if fp8:
        msa.kv_append_fp8(kd, vd, scales, seqs, rope, caches[0], caches[1], **kw)
    else:
        msa.kv_append(kd, vd, seqs, rope, caches[0], caches[1], **kw)
    n = len(pos)
    rows = torch.from_numpy(to).cuda()
    others = torch.ones(caches[0].shape[0], dtype=torch.bool, device="cuda")
    others[rows] = False
    for c in caches:
        assert bool((c[others] == 3).all())                # nothing else is touched
    _check_turned(caches[0][rows], x["k"], w["k"], pos, f, rot, inter, 1.0, rng, "k", scales[0] if fp8 else None)
    if fp8:
        check_codes(caches[1][rows].cpu().numpy(), x["v"][:n], scales[1], 0 * x["v"][:n], "v")
    else:
        assert torch.equal(caches[1][rows], vd[:n])
    if len(caches) > 2:
        _check_turned(caches[2][rows].unsqueeze(1), x["i"], w["i"], pos, fi, irot, inter, 1.1, rng, "index_k")


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
def test_rows_without_a_page_are_dropped(fp8):
    """Pages -1 and past the pool, and positions past the table: nothing is written for them, all else as usual."""
    rng = np.random.default_rng(1)
    H, page = 2, 32
    table = torch.tensor([[0, -1, 2], [7, 1, 1 << 30]], dtype=torch.int32, device="cuda")
    q_rows, kv_lens = [96, 90], [96, 90]
    seqs = padded_seqs(q_rows, kv_lens, total_kv=4 * page, table=table, page=page)
    dtype = torch.uint8 if fp8 else torch.bfloat16
    k, v = dev(bf16(rng.standard_normal((186, H, D)))), dev(bf16(rng.standard_normal((186, H, D))))
    kc, vc = (torch.full((4 * page, H, D), 3, dtype=dtype, device="cuda") for _ in range(2))
    if fp8:
        msa.kv_append_fp8(k, v, (0.5, 0.5), seqs, None, kc, vc)
    else:
        msa.kv_append(k, v, seqs, None, kc, vc)
    want_k, want_v = torch.full_like(kc, 3), torch.full_like(vc, 3)
    enc = (lambda t: (t.float() * 2).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)) if fp8 else (lambda t: t)
    for dst, src in ((slice(0, 32), slice(0, 32)), (slice(64, 96), slice(64, 96)), (slice(32, 64), slice(96 + 32, 96 + 64))):
        want_k[dst], want_v[dst] = enc(k[src]), enc(v[src])
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


def test_contiguous_rows_past_the_cache_are_dropped():
    k = torch.arange(1, 9, device="cuda").to(torch.bfloat16).view(8, 1, 1).expand(8, 1, D).contiguous()
    guard = torch.full((64, 1, D), 99, dtype=torch.bfloat16, device="cuda")
    kc, vc = guard[:10], guard[20:30]
    msa.kv_append(k, k, padded_seqs([8], [8], kv_starts=[6], total_kv=10), None, kc, vc)
    want = torch.full_like(guard, 99)
    want[6:10] = want[26:30] = k[:4]
    assert torch.equal(guard, want)


def test_values_keep_their_bits():
    """Every bf16 pattern, NaN payloads, denormals and infinities among them, through v and the unrotated half of k."""
    bits = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(512, 1, D)
    seqs = padded_seqs([512], [512])
    kc, vc = (torch.zeros((512, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    _, rope = rope_pair(64, D, False, 1.0)
    msa.kv_append(bits, bits, seqs, rope, kc, vc)
    assert torch.equal(vc.view(torch.int16), bits.view(torch.int16))
    assert torch.equal(kc.view(torch.int16)[..., 64:], bits.view(torch.int16)[..., 64:])


def test_captured():
    case = CASES[2]
    x, w, kd, vd, seqs, (_, rope, _), _, to, caches, kw, pos, inter, rng = _make(case, False)
    rows = torch.from_numpy(to).cuda()
    def run():
        msa.kv_append(kd, vd, seqs, rope, caches[0], caches[1], **kw)
        return caches
    want = [c.clone() for c in run()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        for c in caches:
            c[rows] = 5
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(caches, want))
