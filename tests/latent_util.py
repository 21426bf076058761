"""Helpers of the latent attention tests: batches on shuffled pages, and bounds that count roundings."""
from __future__ import annotations

import numpy as np
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import synth
from tests.operators_util import BF16_HALF, bf16, dev, host, padded_seqs, page_table

ROT = 64
SCALE = 1.0 / np.sqrt(192.0)
# LSE: scores are fp32 sums of up to 576 exact products (36 matrix products of 16) whose sizes, scaled, sum to about 15 for
# N(0, 1) data: 40 roundings of 2^-24 of that are 3.6e-5; the sum of the weights and the logarithm stay below
# 1e-5 of their value (up to 20).  1e-4 covers both.
LSE_TOL = 1e-4


def e4m3(x: np.ndarray, scale: float) -> np.ndarray:
    """Codes of x / scale."""
    return (torch.from_numpy(np.asarray(x, np.float32)) / scale).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def check_o(got, ref, size, what):
    """O in bf16: every weight is rounded to bf16 for the value product and carries the score's error (2 LSE_TOL
    relative), both relative to the weight; the fp32 sums add less than 2^-12 of the sum of sizes (4096 roundings);
    one rounding of the result."""
    inner = (BF16_HALF + 2 * LSE_TOL + 2.0 ** -12) * size
    tol = inner + BF16_HALF * (np.abs(ref) + inner)
    err = np.abs(got - ref)
    assert (err <= tol).all(), f"{what}: {(err > tol).sum()} values off, worst {(err / np.maximum(tol, 1e-300)).max():.2f} tolerances"


def check_lse(got, ref, what, tol=LSE_TOL):
    empty = np.isneginf(ref)
    assert (np.isneginf(got) == empty).all(), what
    assert np.abs(got[~empty] - ref[~empty]).max(initial=0.0) <= tol, f"{what}: {np.abs(got[~empty] - ref[~empty]).max()}"


def some_rows(rng, q_offsets, n, most=48):
    """All rows, or the ends of the batch and of each sequence, and some others."""
    if n <= most:
        return np.arange(n)
    ends = np.asarray(q_offsets)
    rows = np.unique(np.r_[0:4, n - 4:n, rng.choice(ends[:-1], min(len(ends) - 1, 12)), rng.choice(ends[1:], min(len(ends) - 1, 12)) - 1,
                           rng.integers(0, n, 12)])
    return rows[(rows >= 0) & (rows < n)]


class PagedBatch:
    """Queries, a latent cache on shuffled pages that is NaN wherever no sequence's key lies, and the layout."""

    def __init__(self, name, q_rows, kv_lens, H, R, page, pad=0, fp8=False, scale=2.0 ** -4, change=lambda rows: rows):
        rng = self.rng = np.random.default_rng(sum(map(ord, name)))
        T, n = sum(q_rows) + pad, sum(kv_lens)
        self.n, self.H, self.R, self.fp8, self.scale = sum(q_rows), H, R, fp8, scale
        self.q = bf16(rng.standard_normal((T, H, R)) * np.sqrt(128 / R))
        self.q_rope = bf16(rng.standard_normal((T, H, ROT)))
        rows = change(rng.standard_normal((n, R + ROT)))
        table, total, where = page_table(rng, kv_lens, page)
        at = np.concatenate(where)
        if fp8:
            codes = e4m3(rows, scale)
            pool = np.full((total, R + ROT), 0x7F, dtype=np.uint8)
            pool[at] = codes
            self.cache = torch.from_numpy(pool).cuda()
            self.rows = O.decode_fp8_e4m3(codes) * scale
        else:
            bits = synth.bf16_bits_from_f32(rows.astype(np.float32))
            pool = np.full((total, R + ROT), 0x7FC0, dtype=np.uint16)
            pool[at] = bits
            self.cache = torch.from_numpy(pool.view(np.int16)).view(torch.bfloat16).cuda()
            self.rows = O.decode_bf16(bits).astype(np.float64)
        self.seqs = padded_seqs(q_rows, kv_lens, pad, total_kv=total, table=torch.from_numpy(table).cuda(), page=page)
        self.lay = O.Layout(q_rows, kv_lens, np.cumsum([0] + list(kv_lens))[:-1])
        # as a product head by head leaves them
        self.dq = dev(self.q.transpose(1, 0, 2)).transpose(0, 1)
        self.dq_rope = dev(self.q_rope)

    def reference(self, rows=None, scale=SCALE, lay=None):
        c = self.rows[:, None, :self.R]
        return O.latent_attention(self.q, self.q_rope, c, self.rows[:, self.R:], c, lay or self.lay, scale, rows)

    def check(self, o, lse, rows, what, **kw):
        ref, l_ref, size = self.reference(rows, **kw)
        check_o(host(o)[rows], ref, size, what)
        check_lse(host(lse)[rows], l_ref, what)


class ExpandedBatch:
    """Queries, per-head keys and values with NaN in the rows that no sequence owns, the shared key part as columns of a
    wider tensor, and the layout."""

    def __init__(self, name, q_rows, kv_lens, H, pad=0, gap=3):
        rng = self.rng = np.random.default_rng(sum(map(ord, name)))
        T = sum(q_rows) + pad
        starts = (gap + np.cumsum([0] + [m + gap for m in kv_lens])[:-1]).tolist()
        N = self.N = starts[-1] + kv_lens[-1] + gap
        self.n, self.H = sum(q_rows), H
        self.q, self.q_rope = bf16(rng.standard_normal((T, H, 128))), bf16(rng.standard_normal((T, H, ROT)))
        self.kv, self.k_rope = bf16(rng.standard_normal((N, H, 256))), bf16(rng.standard_normal((N, ROT)))
        self.lay = O.Layout(q_rows, kv_lens, starts)
        self.owned = np.zeros(N, dtype=bool)
        for s, m in zip(starts, kv_lens):
            self.owned[s:s + m] = True
        kv, k_rope = self.kv.copy(), self.k_rope.copy()
        kv[~self.owned] = np.nan
        k_rope[~self.owned] = np.nan
        joint = torch.zeros((T, H * (128 + ROT) + 8), dtype=torch.bfloat16, device="cuda")   # a query projection's rows
        self.dq, self.dq_rope = joint[:, :H * 128].view(T, H, 128), joint[:, H * 128:H * (128 + ROT)].view(T, H, ROT)
        self.dq.copy_(dev(self.q))
        self.dq_rope.copy_(dev(self.q_rope))
        wide = torch.zeros((N, 40 + ROT), dtype=torch.bfloat16, device="cuda")
        self.dkv, self.dk_rope = dev(kv), wide[:, 40:]
        self.dk_rope.copy_(dev(k_rope))
        self.seqs = padded_seqs(q_rows, kv_lens, pad, kv_starts=starts, total_kv=N)

    def reference(self, rows=None, scale=SCALE, lay=None):
        return O.latent_attention(self.q, self.q_rope, self.kv[..., :128], self.k_rope, self.kv[..., 128:], lay or self.lay, scale,
                                  rows)

    def check(self, o, lse, rows, what, **kw):
        ref, l_ref, size = self.reference(rows, **kw)
        check_o(host(o)[rows], ref, size, what)
        check_lse(host(lse)[rows], l_ref, what)


def check_grad(got, ref, size, what, terms=1.0):
    """A gradient in bf16: every term's factor (P or dS) carries the score's error (2 LSE_TOL of the weight), dS the error
    of its difference (fp32 sums of 128 exact products: 2^-18 of their sizes), and one rounding to bf16; the fp32
    sums add less than 2^-12 of the sum of sizes (4096 roundings); one rounding of the result.  ``size`` is the
    sum of the terms' sizes."""
    inner = (BF16_HALF + 2 * LSE_TOL + 2.0 ** -18 + 2.0 ** -12) * size * terms
    tol = inner + BF16_HALF * (np.abs(ref) + inner)
    err = np.abs(got - ref)
    assert (err <= tol).all(), f"{what}: {(err > tol).sum()} values off, worst {(err / np.maximum(tol, 1e-300)).max():.2f} tolerances"
