"""msa_latent_attn_paged and its E4M3 form against the float64 oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa
from tests.latent_util import ROT, SCALE, PagedBatch, check_lse, some_rows
from tests.operators_util import dev, host, padded_seqs, replay

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


# name, q_rows, kv_lens, heads, latent, page, rows behind the last sequence
CASES = [
    ("first_token", [1], [1], 8, 512, 64, 0),
    ("one_token_each", [1, 1, 1, 1, 1, 1], [1, 63, 64, 65, 1000, 4097], 64, 512, 64, 0),
    ("one_token_long", [1], [9001], 64, 512, 128, 0),
    ("two_head_blocks", [1, 1, 1], [300, 5000, 17], 128, 512, 64, 0),
    ("uneven_head_blocks", [1, 2], [700, 130], 100, 256, 32, 1),
    ("many_head_blocks", [1, 1], [200, 900], 520, 256, 64, 0),
    ("one_head", [1, 70], [500, 90], 1, 512, 64, 0),
    ("five_heads", [13, 1, 0, 40], [130, 2000, 50, 40], 5, 256, 16, 2),
    ("twenty_heads", [7, 3], [333, 900], 20, 512, 16, 0),
    ("forty_heads", [3, 5], [64, 1200], 40, 256, 1024, 0),
    ("draft_rows", [4, 3, 1, 5], [300, 1029, 64, 5], 64, 512, 64, 0),
    ("ragged_batch", [1] * 40, [1 + 97 * i for i in range(40)], 32, 512, 64, 3),
    ("prompt", [300], [300], 8, 512, 64, 0),
    ("prompt_many_tiles", [700], [700], 64, 256, 128, 0),
    ("chunk_on_long", [64], [12000], 8, 512, 1024, 0),
    ("mixed", [1, 130, 1, 0, 40, 1], [2000, 400, 64, 128, 41, 3333], 32, 512, 16, 0),
    ("200_sequences", [1, 2] * 100, [1 + 7 * i % 400 + 2 for i in range(200)], 8, 512, 64, 0),
]


def run(b, fp8, **kw):
    if fp8:
        return msa.latent_attn_paged_fp8(b.dq, b.dq_rope, b.cache, b.scale, b.seqs, **kw)
    return msa.latent_attn_paged(b.dq, b.dq_rope, b.cache, b.seqs, **kw)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_latent_paged(case, fp8):
    name, q_rows, kv_lens, H, R, page, pad = case
    b = PagedBatch(name, q_rows, kv_lens, H, R, page, pad, fp8)
    T, n = b.n + pad, b.n
    o = torch.full((T, H, R), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), 7.0, device="cuda")
    size = msa.latent_attn_paged_workspace_size(b.seqs, H, R)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")          # NaN where it is read unwritten
    run(b, fp8, out=o, lse=lse, workspace=ws)
    assert bool((o[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    assert bool(torch.isfinite(o[:n]).all()) and bool(torch.isfinite(lse[:n]).all())
    b.check(o, lse, some_rows(b.rng, b.lay.q_offsets, n), name)
    o2, l2 = run(b, fp8)                                                      # the same bits again
    assert torch.equal(o2[:n], o[:n]) and torch.equal(l2[:n], lse[:n])


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-30, 0.2])
def test_softmax_scales(scale, fp8):
    b = PagedBatch("scales", [3, 20], [70, 130], 8, 256, 64, 0, fp8)
    o, l = run(b, fp8, softmax_scale=scale)
    b.check(o, l, np.arange(b.n), "scale", scale=scale)


@pytest.mark.parametrize("cache_scale", [2.0 ** -20, 0.3, 1000.0])
def test_code_scales(cache_scale):
    """The scale multiplies keys and values, whatever its size; the softmax scale makes up for it in the scores."""
    b = PagedBatch("codes", [2, 5], [70, 300], 8, 512, 64, 0, True)
    unit = msa.latent_attn_paged_fp8(b.dq, b.dq_rope, b.cache, 1.0, b.seqs, softmax_scale=SCALE * b.scale)
    o, l = msa.latent_attn_paged_fp8(b.dq, b.dq_rope, b.cache, cache_scale, b.seqs, softmax_scale=SCALE * b.scale / cache_scale)
    # the scale of the scores, 2 roundings of 2^-24 apart, moves weights by the scores' size (below 60) times as much
    tol = 60 * 2.0 ** -22
    assert float((l - unit[1]).abs().max()) <= tol
    want = host(unit[0]) * cache_scale
    assert (np.abs(host(o) - want) <= (2 * 2.0 ** -8 + 4 * tol) * np.abs(want) + 4 * tol * cache_scale * 448).all()


def test_strides():
    """Queries with heads as columns, heads first, and padded rows give the same bits."""
    b = PagedBatch("strides", [2, 9], [200, 64], 20, 256, 64)
    o, l = run(b, False)
    T, H, R = b.dq.shape
    wide = torch.zeros((T, H, R + ROT + 8), dtype=torch.bfloat16, device="cuda")
    wide[..., :R], wide[..., R:R + ROT] = b.dq, b.dq_rope
    joint = torch.zeros((T + 1, H * (R + ROT) + 16), dtype=torch.bfloat16, device="cuda")
    jq, jr = joint[:T, :H * R].view(T, H, R), joint[:T, H * R:H * (R + ROT)].view(T, H, ROT)
    jq.copy_(b.dq)
    jr.copy_(b.dq_rope)
    for q, e in ((wide[..., :R], wide[..., R:R + ROT]), (jq, jr), (b.dq.contiguous(), b.dq_rope.transpose(0, 1).contiguous().transpose(0, 1))):
        o2, l2 = msa.latent_attn_paged(q, e, b.cache, b.seqs)
        assert torch.equal(o, o2) and torch.equal(l, l2)


def test_large_scores_and_infinite_neighbours():
    """Scores of thousands (the running maximum moves far between steps), and other sequences' keys infinite."""
    b = PagedBatch("large", [1, 2], [400, 200], 8, 256, 64)
    sign = b.rng.choice([-60.0, -30, 30, 60], size=(400, 1))
    b.rows[:400] = sign * np.ones(b.R + ROT)
    b.rows[400:] = np.inf
    at = np.concatenate([host(b.seqs.block_table)[i, np.arange(m) // 64] * 64 + np.arange(m) % 64 for i, m in enumerate((400, 200))])
    pool = torch.full_like(b.cache, float("inf"))
    pool[torch.from_numpy(at.astype(np.int64)).cuda()] = torch.from_numpy(b.rows).to(torch.bfloat16).cuda()
    b.cache = pool
    b.dq, b.q = torch.full_like(b.dq, 3.0), np.full_like(b.q, 3.0)
    b.dq_rope, b.q_rope = torch.full_like(b.dq_rope, 3.0), np.full_like(b.q_rope, 3.0)
    o, l = run(b, False)
    # ties of equal keys alone keep weight: exact values, and a log of their number
    assert bool((o[0] == 60.0).all())
    ref = 60.0 * 3 * (b.R + ROT) * SCALE + np.log((sign == 60).sum())
    # roundings of 2^-24: the scale to fp32, log2 e, their product, the score's, the sum with the logarithm, ln 2, its product
    assert np.abs(host(l)[0] - ref).max() <= 8 * 2.0 ** -24 * ref


@pytest.mark.parametrize("R", [256, 512])
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
def test_maxima_that_grow(fp8, R):
    """In every second step one key of one half, by turns, outgrows what the weights were relative to, for every second head
    alone: scores climb to 25 by 6.3 (9 in base 2).  The sizes of a score's terms sum to less than 32, so LSE_TOL's count
    of roundings covers them (7.6e-5, and 1e-5 for the rest)."""
    lens = [640, 300]
    def climb(rows):
        rows *= 0.25
        rows[:, 0] = 0
        for j0 in (0, lens[0]):
            for s in range(10):
                j = j0 + 64 * s + 32 * (s // 2 % 2) + 7
                if j < j0 + lens[j0 > 0]:
                    rows[j, 0] = 11 * (s // 2)
        return rows
    b = PagedBatch("grow", [3, 40], lens, 8, R, 64, 0, fp8, scale=2.0 ** -3, change=climb)
    b.q[..., 0] = np.where(np.arange(8) % 2, 0.0, 8.0)
    b.dq = dev(b.q.transpose(1, 0, 2)).transpose(0, 1)
    o, l = run(b, fp8)
    b.check(o, l, np.arange(b.n), "grow")


def test_row_without_keys():
    """A sequence whose lengths fall behind its rows: rows without a key get zeros and -inf."""
    b = PagedBatch("empty", [1, 4, 3], [5, 4, 70], 8, 512, 64)
    b.seqs.kv_lens.copy_(torch.tensor([0, 2, 70], dtype=torch.int32))
    o, l = run(b, False)
    assert bool((o[:3] == 0).all()) and bool((l[:3] == -float("inf")).all())
    lay = O.Layout([1, 4, 3], [0, 2, 70], b.lay.kv_starts)
    b.check(o, l, np.arange(8), "empty", lay=lay)


@pytest.mark.parametrize("case", [CASES[3], CASES[10], CASES[13]], ids=lambda c: c[0])
def test_captured_with_lengths_that_grow(case):
    """A graph captured once serves later steps: kv_lens change on the device below the captured bounds."""
    name, q_rows, kv_lens, H, R, page, pad = case
    b = PagedBatch(name, q_rows, kv_lens, H, R, page, pad)
    ws = torch.empty(msa.latent_attn_paged_workspace_size(b.seqs, H, R), dtype=torch.uint8, device="cuda")
    def step():
        return run(b, False, workspace=ws)
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
    """Calls on two streams, each with a workspace and outputs of its own, give the bits of calls one after the other."""
    made = [PagedBatch(*CASES[i]) for i in (2, 10)]
    want = [run(b, False) for b in made]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for st, b in zip(streams, made):
            with torch.cuda.stream(st):
                got.append(run(b, False))
        torch.cuda.synchronize()
        for (o, l), (o2, l2) in zip(want, got):
            assert torch.equal(o, o2) and torch.equal(l, l2)


@pytest.mark.parametrize("page", [16, 64])
def test_pool_past_4_gib(page):
    """Pages whose bytes lie past 2^32 (and whose elements lie past 2^31): appended there, read from there."""
    R = 512
    rows = 4400000 // page * page                          # 5.1 GB
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB")
    kv_lens, q_rows, H = [200, 90], [5, 1], 16
    rng = np.random.default_rng(8)
    need = [-(-n // page) for n in kv_lens]
    last = rows // page - 1
    table = np.zeros((2, max(need)), dtype=np.int32)
    table[0, :need[0]] = last - rng.permutation(need[0])
    table[1, :need[1]] = last - need[0] - rng.permutation(need[1])
    pool = torch.empty((rows, R + ROT), dtype=torch.bfloat16, device="cuda")
    tab = torch.from_numpy(table).cuda()
    b = PagedBatch("past", q_rows, kv_lens, H, R, page)
    x = torch.from_numpy(b.rows).to(torch.bfloat16).cuda()
    msa.latent_append(x[:, :R], x[:, R:], padded_seqs(kv_lens, kv_lens, total_kv=rows, table=tab, page=page), None, pool)
    seqs = padded_seqs(q_rows, kv_lens, total_kv=rows, table=tab, page=page)
    o, l = msa.latent_attn_paged(b.dq, b.dq_rope, pool, seqs)
    b.check(o, l, np.arange(6), "past 4 GiB")


def test_pages_outside_the_pool_stay_inside_it():
    """Bad page ids are clamped: the call ends and writes finite rows (what they are is unspecified)."""
    table = torch.tensor([[5, -3, 1 << 30, 0]], dtype=torch.int32, device="cuda")
    seqs = padded_seqs([2], [200], total_kv=6 * 64, table=table, page=64)
    q = torch.ones((2, 8, 512), dtype=torch.bfloat16, device="cuda")
    cache = torch.ones((6 * 64, 576), dtype=torch.bfloat16, device="cuda")
    o, l = msa.latent_attn_paged(q, q[..., :ROT], cache, seqs)
    assert bool((o == 1).all()) and bool(torch.isfinite(l).all())
