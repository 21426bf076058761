"""msa_latent_append and its E4M3 form: which cache rows are written, and what they hold, against the float64 oracle."""
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
ROT = 64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


# name, latent, q_rows, kv_lens, page (0: contiguous), rotated dimensions, interleaved, norm, rows behind
CASES = [
    ("one_token", 512, [1], [1], 64, 64, False, True, 0),
    ("decode", 512, [1] * 67, [1 + 61 * i for i in range(67)], 64, 64, False, True, 0),
    ("chunks", 512, [33, 0, 129, 1], [33, 17, 1000, 200], 128, 64, True, True, 5),
    ("small_pages", 256, [100, 50], [163, 50], 16, 24, True, False, 3),
    ("part_rotated", 256, [61, 2], [61, 900], 32, 40, False, True, 0),
    ("no_rotation", 512, [20], [4096], 1024, 0, False, True, 0),
    ("nothing_applied", 256, [20], [25], 64, 0, False, False, 0),
    ("contiguous", 512, [40, 1, 9], [40, 300, 64], 0, 64, False, True, 2),
    ("many_rows", 512, [5000, 9000], [5000, 70000], 256, 32, False, True, 0),
]


@pytest.mark.parametrize("fp8", [None, 2.0 ** -4, 0.3], ids=["bf16", "e4m3", "e4m3_odd_scale"])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_latent_append(case, fp8):
    name, R, q_rows, kv_lens, page, rot, inter, norm, pad = case
    rng = np.random.default_rng(sum(map(ord, name)))
    T, n = sum(q_rows) + pad, sum(q_rows)
    x = bf16(rng.standard_normal((T, R + ROT)))
    w = (1 + 0.3 * rng.standard_normal(R)).astype(np.float32) if norm else None
    if page:
        table, total, rows = page_table(rng, kv_lens, page)
        seqs = padded_seqs(q_rows, kv_lens, pad, total_kv=total, table=torch.from_numpy(table).cuda(), page=page)
    else:
        starts = np.cumsum([5] + [m + 3 for m in kv_lens])[:-1].tolist()
        total = starts[-1] + kv_lens[-1] + 7
        rows = [s + np.arange(m) for s, m in zip(starts, kv_lens)]
        seqs = padded_seqs(q_rows, kv_lens, pad, kv_starts=starts, total_kv=total)
    to = np.concatenate([r[m - q:] for r, q, m in zip(rows, q_rows, kv_lens)])
    joint = torch.zeros((T, R + ROT + 4), dtype=torch.bfloat16, device="cuda")     # columns of a wider tensor
    joint[:, :R + ROT] = dev(x)
    freq, rope = rope_pair(rot, ROT, inter, 1.25)
    old = torch.randint(0, 120, (total, R + ROT), dtype=torch.uint8, device="cuda")
    cache = old.clone() if fp8 else old.to(torch.bfloat16)
    before = cache.clone()
    args = (seqs, rope, cache, None if w is None else torch.from_numpy(w).cuda(), EPS)
    if fp8:
        msa.latent_append_fp8(joint[:, :R], joint[:, R:R + ROT], fp8, *args)
    else:
        msa.latent_append(joint[:, :R], joint[:, R:R + ROT], *args)
    keep = np.ones(total, dtype=bool)
    keep[to] = False
    keep = torch.from_numpy(keep).cuda()
    assert torch.equal(cache[keep], before[keep])
    got = cache[torch.from_numpy(to).cuda()]
    pos = positions(q_rows, kv_lens)
    c = O.norm_rope(x[:n, None, :R], [0] * n, w, EPS, np.zeros(0))[:, 0]
    plain = x[:n, None, R:]
    k = O.norm_rope(plain, pos, None, EPS, freq, inter, 1.25)[:, 0]
    ref = np.concatenate((c, k), -1)
    # the latent's sum of squares is a tree of 9 levels: as a head's of 128, below the 16 roundings of F32
    amp = np.concatenate((np.abs(c), amplitude(plain, rot, inter, 1.25)[:, 0]), -1)
    if fp8:
        check_codes(got.cpu().numpy(), ref, fp8, amp, name)
    else:
        check_bf16(host(got), ref, amp, name)


def test_untouched_elements_keep_their_bits():
    bits = torch.randint(0, 1 << 16, (9, 256 + ROT), dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).cuda()
    seqs = msa.Seqs([9], [9], [0], 9, "cuda")
    cache = torch.zeros_like(bits)
    msa.latent_append(bits[:, :256], bits[:, 256:], seqs, None, cache)
    assert torch.equal(cache.view(torch.int16), bits.view(torch.int16))


def test_rows_without_a_place_are_dropped():
    """Pages of -1 or outside the pool, and positions outside a contiguous cache: nothing else is written."""
    x = torch.ones((8, 512 + ROT), dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[-1, 1 << 20], [1, -1]], dtype=torch.int32, device="cuda")
    seqs = msa.Seqs([4, 4], [18, 18], [0, 0], 48, "cuda", block_table=table, page_size=16)
    cache = torch.zeros((48, 576), dtype=torch.bfloat16, device="cuda")
    msa.latent_append(x[:, :512], x[:, 512:], seqs, None, cache)
    assert bool((cache[30:32] == 1).all()) and float(cache.float().sum()) == 2 * 576   # positions 14, 15 of the second
    flat = msa.Seqs([4, 4], [4, 6], [40, 46], 48, "cuda")
    cache.zero_()
    msa.latent_append(x[:, :512], x[:, 512:], flat, None, cache)
    assert bool((cache[40:44] == 1).all()) and float(cache.float().sum()) == 4 * 576   # rows 48 .. 51 do not exist


def test_far_positions():
    """Angles of positions around 2^24 and beyond, where fp32 positions would be off."""
    p = [16777217, 400000003]
    freq, rope = rope_pair(64, 64, True, 1.0)
    table = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(3)
    x = bf16(rng.standard_normal((2, 256 + ROT)))
    page, stride = 8192, 400000003 // 8192 + 1
    table = torch.full((2, stride), -1, dtype=torch.int32, device="cuda")
    for i, q in enumerate(p):
        table[i, q // page] = i
    seqs = msa.Seqs([1, 1], [q + 1 for q in p], [0, 0], 2 * page, "cuda", block_table=table, page_size=page)
    cache = torch.zeros((2 * page, 320), dtype=torch.bfloat16, device="cuda")
    d = dev(x)
    msa.latent_append(d[:, :256], d[:, 256:], seqs, rope, cache)
    got = host(cache[[i * page + q % page for i, q in enumerate(p)]])[:, 256:]
    ref = O.norm_rope(x[:, None, 256:], p, None, 0.0, freq, True, 1.0)[:, 0]
    # the oracle's angles are products in 64 bits, as the kernel's: of 4e8 radians they are known to 2^-24
    check_bf16(got, ref, amplitude(x[:, 256:], 64, True, 1.0) * 2, "far")
