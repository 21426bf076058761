"""Which form of the paged dense attention a call takes, told from its workspace: the GPU cases of paged_cases.py reach
the forms that they are named for."""
from __future__ import annotations

import pytest

from tests.paged_cases import LONG, VARIANTS, run_length, waves_of, workspace


@pytest.mark.parametrize("group", [1, 3, 8, 16])
def test_waves_by_rows(group):
    per = 32 // group
    for waves, (lo, hi) in {1: (1, per), 2: (per + 1, 2 * per), 4: (2 * per + 1, 4 * per), 8: (4 * per + 1, 9 * per)}.items():
        assert waves_of(lo, group) == waves_of(hi, group) == waves


@pytest.mark.parametrize("case", VARIANTS + LONG, ids=[c[0] for c in VARIANTS] + ["long_" + c[0] for c in LONG])
def test_case_reaches_its_form(case):
    name, waves, split, q_rows, kv_lens, H_q, H_kv, page, pad = case
    assert waves_of(max(q_rows), H_q // H_kv) == waves
    assert (workspace(q_rows, kv_lens, H_q, H_kv, page) > 0) == split


def test_every_form_has_a_case():
    """Few rows and 8 waves on pages of 64 rows and more are the cases of test_gpu_dense_paged.py."""
    reached = {(w, split, page < 64) for _, w, split, _, _, _, _, page, _ in VARIANTS}
    want = {(w, split, small) for w in (2, 4) for split in (False, True) for small in (False, True)}
    assert reached >= want | {(w, split, True) for w in (1, 8) for split in (False, True)}


@pytest.mark.parametrize("case", LONG, ids=[c[0] for c in LONG])
def test_long_runs_cross_two_windows(case):
    run, window = run_length(case)
    assert run > 2 * window
    if case[2]:                                            # the second CTA begins inside a window
        assert run % window != 0
