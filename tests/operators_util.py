"""Helpers of the tests of norms, rotation, cache append and paged attention:
batches with rows behind the last sequence, shuffled pages, error bounds."""
from __future__ import annotations

import ctypes

import numpy as np
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa, synth

BF16_HALF = 2.0 ** -8        # half a step of bf16 relative to the value, at most
E4M3_HALF = 2.0 ** -4        # the same for E4M3, of normal values
E4M3_TINY = 2.0 ** -10       # half the step of its subnormal values
# fp32 arithmetic of a head: the sum of 128 squares (a tree of 7 and its terms' products), the root, three
# products, the rotation's two products and sum, cosine and sine of an angle of up to half a turn known to
# 2^-25 of it (2 pi 2^-26 < 2^-23): below 16 roundings of 2^-24
F32 = 2.0 ** -20


def bf16(x: np.ndarray) -> np.ndarray:
    """x rounded to bf16, as float64 values."""
    bits = synth.bf16_bits_from_f32(np.asarray(x, dtype=np.float32))
    return O.decode_bf16(bits).astype(np.float64)


def dev(x: np.ndarray) -> torch.Tensor:
    """float64 array holding bf16 values -> bf16 tensor on the GPU."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()


def host(t: torch.Tensor) -> np.ndarray:
    return t.double().cpu().numpy()


def padded_seqs(q_rows, kv_lens, pad=0, kv_starts=None, total_kv=None, table=None, page=0, device="cuda"):
    """Seqs whose query side has ``pad`` rows behind the last sequence."""
    total_kv = sum(kv_lens) if total_kv is None else total_kv
    s = msa.Seqs(q_rows, kv_lens, [0] * len(q_rows) if kv_starts is None else kv_starts, total_kv, device,
                 block_table=table, page_size=page)
    if pad:
        s.total_q_rows += pad
        s.c.total_q_rows += pad
        s.c.max_q_rows = max(s.c.max_q_rows, -(-s.total_q_rows // s.num_seqs))
        s.c.max_kv_len = max(s.c.max_kv_len, s.c.max_q_rows)
    return s


def positions(q_rows, kv_lens):
    return [n - q + t for q, n in zip(q_rows, kv_lens) for t in range(q)]


def page_table(rng, kv_lens, page, spare=2):
    """(table [S, pages] with -1 behind each sequence's pages, rows of the pool, each sequence's rows)."""
    need = [-(-n // page) for n in kv_lens]
    total = sum(need) + spare
    order = rng.permutation(total)
    table = np.full((len(need), max(need) + 1), -1, dtype=np.int32)
    rows, at = [], 0
    for i, (n, length) in enumerate(zip(need, kv_lens)):
        table[i, :n] = order[at:at + n]
        at += n
        j = np.arange(length)
        rows.append(table[i, j // page].astype(np.int64) * page + j % page)
    return table, total * page, rows


def rope_pair(rot, dim, inter, scale, seed=0, base=10000.0):
    """(inv_freq as numpy, msa.Rope) with rot rotated dimensions; None for none."""
    if rot == 0:
        return np.zeros(0), None
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    return f, msa.Rope(torch.from_numpy(f).cuda(), interleaved=inter, scale=scale)


def amplitude(n: np.ndarray, rot: int, inter: bool, scale: float) -> np.ndarray:
    """Per element the sum of its pair's sizes before the rotation (times |scale|): what its fp32 error goes by."""
    a = np.abs(n)
    out = a.copy()
    if rot:
        if inter:
            s = a[..., 0:rot:2] + a[..., 1:rot:2]
            out[..., 0:rot:2] = out[..., 1:rot:2] = s * abs(scale)
        else:
            s = a[..., :rot // 2] + a[..., rot // 2:rot]
            out[..., :rot] = np.concatenate((s, s), -1) * abs(scale)
    return out


def check_bf16(got, ref, amp, what):
    """got = bf16 of a value within F32 * amp of ref."""
    err = np.abs(got - ref)
    tol = F32 * amp + BF16_HALF * (np.abs(ref) + F32 * amp)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} values off, worst {np.max(err / np.maximum(tol, 1e-300)):.2f} tolerances"


def check_codes(codes, ref, scale, amp, what):
    """codes = E4M3 of a value within F32 * amp of ref, divided by scale, at most 448 in size."""
    got = O.decode_fp8_e4m3(codes)
    assert np.isfinite(got).all(), what
    z = np.clip(ref / scale, -448.0, 448.0)
    d = F32 * amp / scale
    tol = d + np.maximum(E4M3_HALF * (np.abs(z) + d), E4M3_TINY)
    bad = ~(np.abs(got - z) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} codes off"


def replay(graph_of, eager, n=4):
    """Captures graph_of() and compares every replay's outputs with eager()'s, with eager work in between."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph_of()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = graph_of()
    for _ in range(n):
        for t in got:
            t.view(torch.uint8).random_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, eager()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


__all__ = [n for n in dir() if not n.startswith("_")]
