"""E4M3 codes of values that nothing else is done to: exactly those of the fp32 quotient value / scale, to nearest even."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.msa_oracle as O
from paper_2606_13392_amd import msa
from tests.operators_util import padded_seqs

pytestmark = pytest.mark.gpu
D = 128
# 0.4375: 0.01068115234375 / 0.4375 = 0.0244140625 lies midway between two codes; the next three have such values too
SCALES = [0.4375, 0.203125, 0.8125, 0.9375, 0.013, 3.0, 1.0 / 3.0, 0.1, 1.3e-38, 5e37, 2.0 ** -4, 2.0 ** 100]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    msa.lib()
    yield
    torch.cuda.synchronize()


def codes_of(x: np.ndarray, scale: float) -> np.ndarray:
    """E4M3 codes (uint8) of float32 x / scale: to nearest even, at most 448 in size; 0x7F for NaN."""
    with np.errstate(over="ignore", invalid="ignore"):
        z = np.clip((x / np.float32(scale)).astype(np.float64), -448.0, 448.0)
        size = np.abs(z)
        step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(size, 2.0 ** -20))), -6) - 3)
        near = np.rint(size / step) * step                 # to even: a code's step divides it into even and odd
        values = O.decode_fp8_e4m3(np.arange(127, dtype=np.uint8))
        code = np.searchsorted(values, np.where(np.isnan(near), 0.0, near)).astype(np.uint8)
    code |= np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(np.isnan(x), 0x7F, code).astype(np.uint8)


def _same(got: torch.Tensor, want: np.ndarray, x: np.ndarray, scale: float):
    got = got.cpu().numpy().reshape(want.shape)
    nan = np.isnan(x)
    assert ((got[nan] & 0x7F) == 0x7F).all()
    bad = ~nan & (got != want)
    assert not bad.any(), f"scale {scale}: {bad.sum()} codes off, first {x[bad][0]!r}: {got[bad][0]:#x} for {want[bad][0]:#x}"


@pytest.mark.parametrize("scale", SCALES)
def test_every_value(scale):
    """All 65536 bf16 patterns through queries, keys and values."""
    bits = np.arange(65536, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    t = torch.from_numpy(np.arange(65536, dtype=np.uint16).view(np.int16)).cuda().view(torch.bfloat16).view(512, 1, D)
    want = codes_of(x, scale)
    seqs = padded_seqs([512], [512])
    q, k = msa.qk_norm_rope_fp8(t, t, (scale, scale), seqs, None)
    kc, vc = (torch.zeros((512, 1, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    msa.kv_append_fp8(t, t, (scale, scale), seqs, None, kc, vc)
    for got in (q, k, kc, vc):
        _same(got, want, x, scale)
