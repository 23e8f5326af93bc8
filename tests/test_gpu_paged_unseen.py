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


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 3, 70])
@pytest.mark.parametrize("hidden", [False, True])
def test_an_infinite_value_of_no_weight_is_the_same_in_every_kernel(dtype, new, hidden):
    """Its weight underflows to 0 in every row, and 0 times infinity is no number, as in the plain sum of fp32 products: whether rows are of one
    new token or of several, and whether another value, that the rows do not see, has them looked at again."""
    p = _attend_problem(22, dtype, [200, 90], [new, 1], 4, 2, 64, 16)
    p["Q"][..., 0] = p["Q"][..., 0].abs() + 1.0
    page, row = int(p["table"][0, 1]), 5                               # position 21 of sequence 0: logits of -1000 and less
    p["K"][page, :, row] = 0.0
    p["K"][page, :, row, 0] = -8192.0
    p["V"][page, :, row, 7] = float("inf")
    if hidden and new > 1:
        p["V"][int(p["table"][0, 199 // 16]), :, 199 % 16, 9] = float("inf")         # of the last new token: the others do not see it
    out, lse = _run_attend(p)
    got = _f64(out)[:new]
    assert np.isfinite(_f64(lse)).all() and np.isfinite(_f64(out)[new:]).all()
    assert np.isnan(got[..., 7]).all()
    rest = np.delete(got, 7, -1)
    if hidden and new > 1:
        assert np.isposinf(rest[-1, :, 8]).all()
        rest[-1, :, 8] = 0.0
    assert np.isfinite(rest).all()


def _time(call):
    call()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    call()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new,length", [(512, 8192), (3, 40000)])
@pytest.mark.parametrize("what", ["key", "value"])
def test_rows_that_see_a_bad_token_are_not_worked_out_twice(dtype, new, length, what):
    """A NaN that all rows see is in their sums for good.  Ten times the time of the clean call is far above what it costs and far below a second pass, row
    after row (hundreds of times)."""
    p = _attend_problem(23, dtype, [length, 50], [new, 1], 8, 2, 64, 16)
    torch.cuda.synchronize()
    clean = min(_time(lambda: _run_attend(p)) for _ in range(3))
    _spoil(p, 0, 100, *((float("nan"), None) if what == "key" else (None, float("nan"))))
    out, lse = _run_attend(p)
    assert torch.isnan(out[:new]).all() and torch.isfinite(out[new:]).all() and torch.isfinite(lse[new:]).all()
    assert torch.isnan(lse[:new]).all() if what == "key" else torch.isfinite(lse).all()
    spoilt = min(_time(lambda: _run_attend(p)) for _ in range(2))
    print(f"clean {clean:.3f} ms, spoilt {spoilt:.3f} ms")
    assert spoilt <= 10 * clean
