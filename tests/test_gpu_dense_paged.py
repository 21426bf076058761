"""msa_dense_attn_paged and its E4M3 form against the float64 oracle's dense attention.

Bars of the other attention calls (O within 1e-2 before output rounding and 5e-3 relative L2), and LSE within
1e-4: its terms are fp32 sums of fp32 weights, scores of exact products of magnitude below 50 carry 128 roundings
of 2^-24 at most.  The pool is NaN wherever no sequence's key lies.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa, synth
from tests.operators_util import padded_seqs, page_table, replay
from tests.util import check_outputs, to_dev

pytestmark = pytest.mark.gpu
D = 128
LSE_TOL = 1e-4


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


# name, q_rows, kv_lens, H_q, H_kv, page, rows behind the last sequence
CASES = [
    ("first_token", [1], [1], 8, 8, 64, 0),
    ("one_token_each", [1, 1, 1, 1, 1, 1], [1, 63, 64, 65, 1000, 4097], 16, 2, 64, 0),
    ("one_token_long", [1], [9001], 64, 8, 128, 0),
    ("ragged_batch", [1] * 40, [1 + 97 * i for i in range(40)], 32, 4, 64, 3),
    ("draft_rows", [4, 3, 1, 5], [300, 1029, 64, 5], 16, 1, 64, 0),
    ("group_of_three", [2, 9], [130, 515], 6, 2, 32, 0),
    ("group_of_one", [31, 1], [700, 2], 4, 4, 16, 2),
    ("group_of_16_chunks", [65, 17], [65, 333], 32, 2, 128, 0),
    ("group_of_12", [40], [1500], 12, 1, 256, 0),
    ("small_pages", [70, 1, 0, 33], [200, 77, 50, 33], 8, 2, 16, 1),
    ("prompt", [600], [600], 16, 2, 64, 0),
    ("mixed", [1, 300, 1, 0, 40, 1], [2000, 900, 64, 128, 41, 3333], 16, 2, 64, 0),
    ("chunk_on_long", [64], [12000], 8, 1, 1024, 0),
    ("chunks_on_long", [130, 20], [5000, 9000], 8, 1, 32, 0),
    ("300_sequences", [1, 2] * 150, [1 + 7 * i % 400 + 2 for i in range(300)], 8, 2, 64, 0),
    ("300_prompts_small_pages", [5 + i % 30 for i in range(300)], [5 + i % 30 for i in range(300)], 8, 2, 16, 0),
    ("many_tiles", [700, 900, 1, 500], [700, 1000, 40, 500], 64, 64, 64, 0),
    ("many_few_row_tiles", [1] * 90, [1 + 5 * i for i in range(90)], 64, 64, 32, 0),
]


def _make(case, fp8):
    name, q_rows, kv_lens, H_q, H_kv, page, pad = case
    rng = np.random.default_rng(sum(map(ord, name)))
    T, n = sum(q_rows) + pad, sum(kv_lens)
    if fp8:
        draw = lambda s: (torch.from_numpy(rng.standard_normal(s).astype(np.float32)) * 16).to(torch.float8_e4m3fn).view(torch.uint8).numpy()  # noqa: E731,E501
    else:
        draw = lambda s: synth.bf16_bits_from_f32(rng.standard_normal(s).astype(np.float32))  # noqa: E731
    q, k, v = draw((T, H_q, D)), draw((n, H_kv, D)), draw((n, H_kv, D))
    table, total, rows = page_table(rng, kv_lens, page)
    at = np.concatenate(rows)
    nan = 0x7F if fp8 else 0x7FC0
    pools = []
    for x in (k, v):
        pool = np.full((total, H_kv, D), nan, dtype=x.dtype)
        pool[at] = x
        pools.append(torch.from_numpy(pool).cuda() if fp8 else to_dev(pool))
    seqs = padded_seqs(q_rows, kv_lens, pad, total_kv=total, table=torch.from_numpy(table).cuda(), page=page)
    lay = O.Layout(q_rows, kv_lens, np.cumsum([0] + kv_lens)[:-1])
    qd = torch.from_numpy(q).cuda() if fp8 else to_dev(q)
    return (q, k, v), (qd, *pools), seqs, lay, rng


SCALES = (2.0 ** -4, 2.0 ** -4, 2.0 ** -5)


def _reference(case, x, lay, fp8, rows, scale=None):
    q, k, v = x
    if fp8:                                                # E4M3 values are bf16 values
        q, k, v = (synth.bf16_bits_from_f32((O.decode_fp8_e4m3(t) * s).astype(np.float32)) for t, s in zip(x, SCALES))
    return O.dense_causal_attention(q, k, v, lay, scale=scale, rows=rows)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_dense_paged(case, fp8):
    name, q_rows, kv_lens, H_q, H_kv, page, pad = case
    x, d, seqs, lay, rng = _make(case, fp8)
    T, n = sum(q_rows) + pad, sum(q_rows)
    o = torch.full((T, H_q, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H_q), 7.0, device="cuda")
    size = max(1, msa.dense_attn_paged_workspace_size(seqs, H_q, H_kv, D))
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")          # NaN where it is read unwritten
    if fp8:
        msa.dense_attn_paged_fp8(*d, SCALES, seqs, out=o, lse=lse, workspace=ws)
    else:
        msa.dense_attn_paged(*d, seqs, out=o, lse=lse, workspace=ws)
    assert bool((o[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    rows = np.arange(n) if n <= 64 else np.unique(np.r_[0:8, n - 8:n, lay.q_offsets[:-1], rng.integers(0, n, 40)])
    rows = rows[rows < n]
    o_ref, l_ref = _reference(case, x, lay, fp8, rows)
    oh, lh = o.float().cpu().numpy(), lse.cpu().numpy()
    assert np.isfinite(oh[:n]).all() and np.isfinite(lh[:n]).all()
    stats = check_outputs(oh[rows], lh[rows], o_ref, l_ref, name)
    assert stats[2] <= LSE_TOL, stats
    # the same bits again
    if fp8:
        o2, l2 = msa.dense_attn_paged_fp8(*d, SCALES, seqs)
    else:
        o2, l2 = msa.dense_attn_paged(*d, seqs)
    assert torch.equal(o2[:n], o[:n]) and torch.equal(l2[:n], lse[:n])


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("q_rows", [[3, 8], [3, 40]], ids=["few_rows", "tiles"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 0.9])
def test_softmax_scales(scale, q_rows, fp8):
    case = ("scales", q_rows, [70, 130], 4, 2, 64, 0)
    x, d, seqs, lay, _ = _make(case, fp8)
    if fp8:
        o, l = msa.dense_attn_paged_fp8(*d, SCALES, seqs, softmax_scale=scale)
    else:
        o, l = msa.dense_attn_paged(*d, seqs, softmax_scale=scale)
    o_ref, l_ref = _reference(case, x, lay, fp8, None, scale)
    check_outputs(o.float().cpu().numpy(), l.cpu().numpy(), o_ref, l_ref, "scale")


def test_large_scores_and_infinite_neighbours():
    """Scores of +-2000 (the running maximum moves by thousands between sub-blocks), and other sequences' keys infinite."""
    q_rows, kv_lens, page = [1, 2], [400, 200], 64
    rng = np.random.default_rng(2)
    table, total, rows = page_table(rng, kv_lens, page)
    k = np.full((total, 1, D), np.inf)
    v = np.full((total, 1, D), np.inf)
    k[rows[0], 0] = rng.choice([-60.0, -30, 30, 60], size=(400, 1)) * np.ones(D)
    v[rows[0], 0] = rng.standard_normal((400, D))
    tb = lambda a: synth.bf16_bits_from_f32(a.astype(np.float32))  # noqa: E731
    q = tb(rng.standard_normal((3, 2, D)) * 0.2 + 3.0)
    seqs = padded_seqs(q_rows, kv_lens, total_kv=total, table=torch.from_numpy(table).cuda(), page=page)
    o, l = msa.dense_attn_paged(to_dev(q), to_dev(tb(k)), to_dev(tb(v)), seqs)
    lay = O.Layout(q_rows, kv_lens, [0, 0])
    o_ref, l_ref = O.dense_causal_attention(q, tb(k[rows[0]]), tb(v[rows[0]]), lay, rows=[0])
    err = np.abs(o[:1].double().cpu().numpy() - o_ref)
    assert np.isfinite(err).all() and err.max() < 4e-2 and np.abs(l[:1].cpu().numpy() - l_ref).max() < 2e-2


def test_row_without_keys():
    """A sequence whose table holds fewer keys than its rows count on: rows without a key get zeros and -inf."""
    table = torch.tensor([[1], [0]], dtype=torch.int32, device="cuda")
    seqs = msa.Seqs([1, 1], [0 + 1, 5], [0, 0], 128, "cuda", block_table=table, page_size=64)
    seqs.kv_lens.copy_(torch.tensor([0, 5], dtype=torch.int32))
    q = torch.ones((2, 4, D), dtype=torch.bfloat16, device="cuda")
    kv = torch.ones((128, 2, D), dtype=torch.bfloat16, device="cuda")
    o, l = msa.dense_attn_paged(q, kv, kv, seqs)
    assert bool((o[0] == 0).all()) and bool((l[0] == -float("inf")).all())
    assert bool((o[1] == 1).all()) and bool(torch.isfinite(l[1]).all())


@pytest.mark.parametrize("case", [CASES[3], CASES[11], CASES[13]], ids=lambda c: c[0])
def test_captured_with_lengths_that_grow(case):
    """A graph captured once serves later steps: kv_lens change on the device below the captured bounds."""
    name, q_rows, kv_lens, H_q, H_kv, page, pad = case
    x, d, seqs, lay, rng = _make(case, False)
    n = sum(q_rows)
    ws = torch.empty(max(1, msa.dense_attn_paged_workspace_size(seqs, H_q, H_kv, D)), dtype=torch.uint8, device="cuda")
    def run():
        o, l = msa.dense_attn_paged(*d, seqs, workspace=ws)
        return o[:n], l[:n]
    replay(run, run)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    shorter = [max(q, 1, int(m * f)) for q, m, f in zip(q_rows, kv_lens, rng.uniform(0.1, 1.0, len(q_rows)))]
    for lens in (shorter, kv_lens):
        seqs.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        rows = np.unique(rng.integers(0, n, 12))
        now = O.Layout(q_rows, lens, lay.kv_starts)
        o_ref, l_ref = _reference(case, x, now, False, rows)
        check_outputs(got[0].float().cpu().numpy()[rows], got[1].cpu().numpy()[rows], o_ref, l_ref, name)


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace and outputs of its own, give the bits of calls one after the other."""
    made = [_make(CASES[i], False) for i in (12, 3)]
    want = [msa.dense_attn_paged(*d, seqs) for _, d, seqs, _, _ in made]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for st, (_, d, seqs, _, _) in zip(streams, made):
            with torch.cuda.stream(st):
                got.append(msa.dense_attn_paged(*d, seqs))
        torch.cuda.synchronize()
        for (o, l), (o2, l2), case in zip(want, got, (CASES[12], CASES[3])):
            n = sum(case[1])
            assert torch.equal(o[:n], o2[:n]) and torch.equal(l[:n], l2[:n])


@pytest.mark.parametrize("page", [16, 64])
def test_pool_past_4_gib(page):
    """Pages whose bytes lie past 2^32 (and whose elements lie past 2^31): appended there, read from there."""
    H, rows = 8, 2200000 // page * page                    # 4.5 GB each for k and v
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB")
    kv_lens, q_rows = [200, 90], [200, 1]
    rng = np.random.default_rng(8)
    need = [-(-n // page) for n in kv_lens]
    last = rows // page - 1
    table = np.zeros((2, max(need)), dtype=np.int32)
    table[0, :need[0]] = last - rng.permutation(need[0])
    table[1, :need[1]] = last - need[0] - rng.permutation(need[1])
    pools = [torch.empty((rows, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tab = torch.from_numpy(table).cuda()
    x = [synth.bf16_bits_from_f32(rng.standard_normal((sum(kv_lens), H, D)).astype(np.float32)) for _ in range(2)]
    whole = padded_seqs(kv_lens, kv_lens, total_kv=rows, table=tab, page=page)
    msa.kv_append(to_dev(x[0]), to_dev(x[1]), whole, None, *pools)
    q = synth.bf16_bits_from_f32(rng.standard_normal((sum(q_rows), 2 * H, D)).astype(np.float32))
    seqs = padded_seqs(q_rows, kv_lens, total_kv=rows, table=tab, page=page)
    o, l = msa.dense_attn_paged(to_dev(q), *pools, seqs)
    one = padded_seqs([1, 1], kv_lens, total_kv=rows, table=tab, page=page)
    o1, l1 = msa.dense_attn_paged(to_dev(q[[199, 200]]), *pools, one)
    pick = [0, 63, 64, 130, 199, 200]
    o_ref, l_ref = O.dense_causal_attention(q, *x, O.Layout(q_rows, kv_lens, [0, 200]), rows=pick)
    check_outputs(o[pick].float().cpu().numpy(), l[pick].cpu().numpy(), o_ref, l_ref, "tiles")
    check_outputs(o1.float().cpu().numpy(), l1.cpu().numpy(), o_ref[4:], l_ref[4:], "few rows")


def test_pages_outside_the_pool_stay_inside_it():
    """Bad page ids are clamped: the call ends and writes finite rows (what they are is unspecified)."""
    table = torch.tensor([[5, -3, 1 << 30, 0]], dtype=torch.int32, device="cuda")
    seqs = padded_seqs([2], [200], total_kv=6 * 64, table=table, page=64)
    q = torch.ones((2, 4, D), dtype=torch.bfloat16, device="cuda")
    kv = torch.ones((6 * 64, 2, D), dtype=torch.bfloat16, device="cuda")
    o, l = msa.dense_attn_paged(q, kv, kv, seqs)
    assert bool((o == 1).all()) and bool(torch.isfinite(l).all())
