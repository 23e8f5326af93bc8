"""Paged attention with far more slots than sequences that have anything to do.

Tolerances as in test_gpu_paged.py; the reference looks at the sequences that have new tokens.
"""
import numpy as np
import pytest
import torch

from paper_2410_01518_amd import infinipot as ip
from tests.test_gpu_paged import DT, _check_attend, _dev

pytestmark = pytest.mark.gpu


def _problem(slots, live, Hq, Hkv, d, page, dtype, W, seed=31):
    """live: slot -> (cached tokens, new ones); the other slots have neither."""
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    news, lens, table = np.zeros(slots, np.int64), np.zeros(slots, np.int32), np.full((slots, W), -1, np.int32)
    n_pages = sum(-(-n // page) for n, _ in live.values()) + 1
    ids, at = rng.permutation(n_pages).astype(np.int32), 0
    for b, (n, m) in live.items():
        held = -(-n // page)
        table[b, :held] = ids[at: at + held]
        at += held
        lens[b], news[b] = n, m
    K, V = (torch.randn((n_pages, Hkv, page, d), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    Q = torch.randn((int(news.sum()), Hq, d), generator=g, device="cuda").to(DT[dtype])
    q_start = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    few = sorted(live)
    small = dict(Q=Q, K=K, V=V, table=table[few], q_start=np.concatenate([[0], np.cumsum(news[few])]).astype(np.int32), lens=lens[few], T=Q.shape[0])
    return dict(Q=Q, K=K, V=V, table=_dev(table), q_start=_dev(q_start), lens=_dev(lens)), small


def _attend(p, max_new, max_len):
    out, lse = torch.full_like(p["Q"], 5.0), torch.full(p["Q"].shape[:2], 5.0, device="cuda")
    paged = ip.make_paged(p["K"], tokens=p["Q"].shape[0], block_table=p["table"], Q=p["Q"], out=out, lse=lse, max_new=max_new, max_len=max_len)
    ws = ip.alloc_paged_workspace(paged)
    assert ip.ccd_paged_attend(paged, p["Q"], p["K"], p["V"], p["table"], p["q_start"], p["lens"], out, lse, ws) == ip.CCD_OK
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("max_new", [256, 64, 0])
def test_as_many_slots_as_a_call_takes(dtype, max_new):
    """B * Hkv = 2^21, a handful of them with chunks and single tokens, wherever they are: a valid call, whatever the hint."""
    slots = 1 << 18
    live = {0: (40, 1), 77: (300, 64), 1000: (33, 33), 131072: (90, 5), 200000: (500, 40), slots - 2: (1, 1), slots - 1: (700, 112)}
    p, small = _problem(slots, live, 16, 8, 64, 64, dtype, 256)
    out, lse = _attend(p, max_new, 16384)
    _check_attend(small, out, lse, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", [(8, 2), (40, 1)])
def test_a_chunk_among_idle_slots(dtype, heads):
    live = {3: (200, 1), 100: (500, 129), 101: (90, 17), 300: (7, 1), 511: (65, 4)}
    p, small = _problem(512, live, *heads, 64, 16, dtype, 40)
    for max_new in (129, 0, 3):
        out, lse = _attend(p, max_new, 500)
        _check_attend(small, out, lse, dtype)
