"""msa_latent_attn_backward: gradients in every layout that its strides allow, and long sequences."""
from __future__ import annotations

import pytest
import torch

from paper_2606_13392_amd import msa
from tests.latent_util import ROT
from tests.test_gpu_latent_backward import check, make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


def joint(T, H, pad):
    """A head's own and rotated part side by side, ``pad`` elements behind them."""
    t = torch.full((T, H, 128 + ROT + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    return t, t[..., :128], t[..., 128:128 + ROT]


def heads_first(T, H, pad):
    own = torch.full((H, T, 128 + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    rot = torch.full((H, T, ROT + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    return (own, rot), own[..., :128].transpose(0, 1), rot[..., :ROT].transpose(0, 1)


@pytest.mark.parametrize("many", [False, True], ids=["32_a_wave", "64_a_wave"])
@pytest.mark.parametrize("layout,pad", [(joint, 0), (joint, 8), (heads_first, 0), (heads_first, 8)],
                         ids=["joint", "joint_padded", "heads_first", "heads_first_padded"])
def test_strides(layout, pad, many):
    """Inputs and gradients in other layouts: the bits of contiguous ones, and nothing written beside them."""
    q_rows, kv_lens = ([300, 1, 40] + [2] * 300, [300, 7, 170] + [2] * 300) if many else ([70, 1, 130], [70, 7, 200])
    b, o, lse = make(("strides", q_rows, kv_lens, 3, 1))
    T, n = b.n + 1, b.n
    want = run(b, o, lse)
    _, q, e = layout(T, 3, pad)
    q.copy_(b.dq)
    e.copy_(b.dq_rope)
    whole, d_q, d_e = layout(T, 3, 4 if pad else 0)         # rows that are 8 bytes aligned alone
    wide = torch.full((b.N, ROT + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    got = msa.latent_attn_backward(q, e, b.dkv, b.dk_rope.contiguous(), o, lse, b.d_o_dev, b.seqs, d_q=d_q, d_q_rope=d_e,
                                   d_k_rope=wide[:, 1:])    # 2 bytes aligned
    for x, y in zip(got[:2], want[:2]):
        assert torch.equal(x[:n], y[:n]) and bool((x[n:] == 7.0).all())
    assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])
    assert bool((wide[:, 0] == 7.0).all())
    if pad:
        beside = (whole[..., 128 + ROT:],) if layout is joint else (whole[0][..., 128:], whole[1][..., ROT:])
        assert all(bool((x == 7.0).all()) for x in beside)


@pytest.mark.parametrize("case", [("long_prompt", [1500], [1500], 1, 0), ("long_chunk", [600], [1900], 1, 0),
                                  # so many tiles that a wave takes 64 queries
                                  ("long_among_many", [1500] + [2] * 780, [1500] + [2] * 780, 1, 0)], ids=lambda c: c[0])
def test_long(case):
    b, o, lse = make(case)
    check(b, o, lse, run(b, o, lse))


def test_no_key_rows():
    """Query rows and a key side of no rows: O and the queries' gradients are zeros, as for other rows without a key."""
    T, H = 70, 3
    seqs = msa.Seqs([60, 10], [60, 10], [0, 0], 0, "cuda")
    t = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, e, d_o, kv, k_rope = t(T, H, 128), t(T, H, ROT), t(T, H, 128), t(0, H, 256), t(0, ROT)
    o, lse = msa.latent_attn(q, e, kv, k_rope, seqs, out=t(T, H, 128))
    assert bool((o == 0).all()) and bool((lse == -float("inf")).all())
    d_q, d_e, d_kv, d_r = msa.latent_attn_backward(q, e, kv, k_rope, o, lse, d_o, seqs, d_q=t(T, H, 128), d_q_rope=t(T, H, ROT))
    assert bool((d_q == 0).all()) and bool((d_e == 0).all()) and d_kv.numel() == d_r.numel() == 0


@pytest.mark.parametrize("sequences", [1, 3])
def test_sequences_without_keys(sequences):
    """No sequence has a key, but the key side has rows: they get zeros."""
    seqs = msa.Seqs([0] * sequences, [0] * sequences, [5] * sequences, 60, "cuda")
    t = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    d_kv, d_r = t(60, 4, 256), t(60, ROT)
    msa.latent_attn_backward(t(0, 4, 128), t(0, 4, ROT), t(60, 4, 256), t(60, ROT), t(0, 4, 128), torch.ones((0, 4), device="cuda"),
                             t(0, 4, 128), seqs, d_kv=d_kv, d_k_rope=d_r)
    assert bool((d_kv == 0).all()) and bool((d_r == 0).all())


def test_keys_past_4_gib():
    """Key rows, and gradients of them, whose bytes lie past 2^32 of their tensors: the bits of the same rows in a small one."""
    H, rows, keys = 64, 140000, 300                         # 32 KiB each: 4.6 GB, and 2.3 GB of workspace
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    b, o, lse = make(("past", [100], [keys], H, 0))
    want = run(b, o, lse)
    kv = torch.empty((rows, H, 256), dtype=torch.bfloat16, device="cuda")
    k_rope = torch.empty((rows, ROT), dtype=torch.bfloat16, device="cuda")
    at, first = rows - keys - 10, b.lay.kv_starts[0]
    kv[at:at + keys], k_rope[at:at + keys] = b.dkv[first:first + keys], b.dk_rope[first:first + keys]
    d_kv = torch.full_like(kv, 7.0)
    got = msa.latent_attn_backward(b.dq, b.dq_rope, kv, k_rope, o, lse, b.d_o_dev, msa.Seqs([100], [keys], [at], rows, "cuda"), d_kv=d_kv)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for x, y in zip(got[2:], want[2:]):
        assert torch.equal(x[at:at + keys], y[first:first + keys])
        assert bool((x[:at] == 0).all()) and bool((x[at + keys:] == 0).all())
