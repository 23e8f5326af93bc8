"""Paged attention where infinities and NaN stand in places that some rows see and others do not: against the 64-bit reference.

Tolerances: what a finite row is off by is bounded in test_gpu_paged.py; here 2^-6 (bf16) and 2^-16 (fp32) of the largest value are far above that
and far below what a token too many or too few would change.
"""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from tests.test_gpu_paged import _attend_problem, _f64, _run_attend

pytestmark = pytest.mark.gpu


def _spoil(p, b, pos, key, value):
    """Key and value of the token at `pos` of sequence b."""
    page = p["K"].shape[2]
    at = int(p["table"][b, pos // page])
    if key is not None:
        p["K"][at, :, pos % page] = key
    if value is not None:
        p["V"][at, :, pos % page] = value


def _check(p, out, lse, dtype, **kw):
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.attend(_f64(p["Q"]), _f64(p["K"]), _f64(p["V"]), p["table"], p["q_start"], p["lens"], **kw)
    got, got_lse = _f64(out), _f64(lse)
    seen = np.isnan(want_lse)                                        # rows that see a key that is NaN
    assert (np.isnan(got_lse) == seen).all() and np.isnan(got[seen]).all()
    assert (np.isfinite(got) == np.isfinite(want)).all()
    fin = np.isfinite(want)
    values = _f64(p["V"])
    A = np.abs(values[np.isfinite(values)]).max()
    assert (np.abs(got[fin] - want[fin]) <= (2.0 ** -6 if dtype == "bf16" else 2.0 ** -16) * A).all()
    fin = np.isfinite(want_lse)
    assert (np.abs(got_lse[fin] - want_lse[fin]) <= 1e-4).all()
    return seen


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("window", [0, 5000])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_more_new_tokens_than_the_host_expected(dtype, group, window, bad):
    """A decoding step whose hint says one new token, and three sequences that have more: a block of rows is one token's heads, and its neighbours'
    tokens are not its own."""
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(1, 60, 100)]
    news = [1] * 100
    several = ((3, 5040, 3), (50, 6000, 5), (99, 7500, 2)) if window else ((3, 40, 3), (50, 300, 5), (99, 1500, 2))
    for b, n, m in several:
        lens[b], news[b] = n, m
    p = _attend_problem(21, dtype, lens, news, 2 * group, 2, 64, 16, W=512)               # (a table of 8192 tokens: not cut by units)
    for b, n, m in several:
        # with a window: a token that the first new one alone sees; without: the last new one
        _spoil(p, b, n - m - window + 1 if window else n - 1, float("nan"), float(bad))
    out, lse = _run_attend(p, window=window, max_new=1, max_len=8192)
    seen = _check(p, out, lse, dtype, window=window)
    assert seen.sum() == 3 * 2 * group
