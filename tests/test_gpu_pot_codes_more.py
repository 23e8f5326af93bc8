"""Distillation of pots and pools in 8 bits: log-sum-exps handed in, novelty with strides of its own, groups of pots, refusals.

Scores with log-sum-exps are compared with a plain pot's that holds the numbers read back and takes the same log-sum-exps: the same keys and normalisers in other kernels' order of sums,
so 3e-5 relative as in test_gpu_pot_codes (fp32 2e-3).
"""
import numpy as np
import pytest
import torch

from oracle import codes_oracle as C
from paper_2410_01518_amd import infinipot as ip
from paper_2410_01518_amd.pot import MemoryPot, PagedPots
from tests import gpu_util as gu
from tests.test_gpu_codes import CODE, _bytes
from tests.test_gpu_paged import DT
from tests.test_gpu_pot_codes import _fill

pytestmark = pytest.mark.gpu


def _plain(pot, kind):
    """A pot of numbers that holds what `pot` stands for."""
    plain = MemoryPot(pot.B, pot.L, pot.Hkv, pot.d, pot.n_cap, pot.k, pot.T, dtype=pot.dtype)
    for to, x, s in ((plain.K, pot.K, pot.K_scales), (plain.V, pot.V, pot.V_scales)):
        to.copy_(torch.from_numpy(C.decode(_bytes(x.flatten(0, 1)), s.flatten(0, 1).cpu().numpy(), kind, 1)).view(to.shape).cuda().to(pot.dtype))
    plain.novelty.copy_(pot.novelty)
    plain.n_valid = pot.n_valid
    return plain


def _off(a, b):
    """The largest relative difference of finite scores; infinite ones are in the same places."""
    a, b = (x.cpu().numpy().astype(np.float64) for x in (a, b))
    assert (np.isinf(a) == np.isinf(b)).all()
    fin = np.isfinite(b)
    return (np.abs(a[fin] - b[fin]) / (np.abs(b[fin]) + 1e-30)).max()


def _compacted(pot, before, keep):
    """Codes, scales and novelty are the kept rows of `before`, in order, and behind them what stood there."""
    after = [_bytes(pot.K), _bytes(pot.V), pot.K_scales.cpu().numpy(), pot.V_scales.cpu().numpy(), pot.novelty.cpu().numpy()]
    flat = keep.reshape(-1, pot.Hkv, pot.k)
    for x, y in zip(after, before):
        np.testing.assert_array_equal(x.reshape(-1, pot.Hkv, *x.shape[3:]), C.compact(y.reshape(-1, pot.Hkv, *y.shape[3:]), flat))


def _held(pot):
    return [_bytes(pot.K), _bytes(pot.V), pot.K_scales.cpu().numpy(), pot.V_scales.cpu().numpy(), pot.novelty.cpu().numpy()]


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,P", [("bf16", 128, 32), ("bf16", 64, 5), ("fp32", 64, 9)])
def test_distillation_takes_the_log_sum_exps_it_is_given(kind, dtype, d, P):
    B, L, Hkv, Hq, n, k = 2, 3, 2, 8, 512, 200
    g = torch.Generator(device="cuda").manual_seed(7)
    pot = MemoryPot(B, L, Hkv, d, n, k, 40, dtype=DT[dtype], codes=CODE[kind])
    _fill(pot, n, g)
    plain, before = _plain(pot, kind), _held(pot)
    Q = torch.randn((B, L, Hq, P, d), generator=g, device="cuda").to(DT[dtype])
    lse = pot.attend(Q, behind=True)[1]
    scores = [torch.zeros((B, L, Hkv, n), device="cuda") for _ in range(3)]
    assert pot.distill(Q, scores=scores[0], lse=lse) == ip.CCD_OK
    shape = ip.make_shape(Q, plain.K, plain.novelty, k=k, T=40, pool_w=7)
    ip.ccd_score_lse(shape, Q, plain.K, lse.flip(1).contiguous(), plain.novelty, scores[2], ip.alloc_workspace(shape))
    assert plain.distill(Q, scores=scores[1], lse=lse) == ip.CCD_OK
    torch.cuda.synchronize()
    tol = 3e-5 if dtype == "bf16" else 2e-3
    assert _off(scores[0], scores[1]) <= tol
    assert not torch.allclose(scores[2], scores[0], rtol=0.05)            # (other rows' log-sum-exps give other scores)
    keep, a = gu.to_host(pot.keep_idx), scores[0].cpu().numpy()
    np.testing.assert_array_equal(keep, gu.replay_select(a, k))
    gu.assert_keep_matches(keep, gu.to_host(plain.keep_idx), scores[1].cpu().numpy(), k)
    _compacted(pot, before, keep)


def _full_pool(kind, pots=1, L=2, Hkv=2, n=256, d=64, Hq=4, P=16, **kw):
    """A pool of pots whose first sequence's is full, and what a distillation of it takes."""
    pool = PagedPots(pots + 1, pots + 2, n, n, n, L, Hq, Hkv, d, codes=CODE[kind], **kw)
    g = torch.Generator(device="cuda").manual_seed(3)
    assert pool.step([n] + [0] * pots) == n
    for layer in range(L):
        pool.append(layer, *(torch.randn((n, Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2)))
    return pool, int(pool.table[0, 0]), torch.randn((1, L, Hq, P, d), generator=g, device="cuda").bfloat16()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("how", ["dense", "layers first", "wide rows", "shared", "shared by expansion"])
def test_a_pool_takes_novelty_of_any_strides(kind, how):
    """The same tokens are kept and the same novelty stands beside them, however it is laid out; what lies between its rows is left alone."""
    L, Hkv, n, k = 2, 2, 256, 96
    pool, page, Q_cat = _full_pool(kind)
    values = torch.rand((1, L, Hkv, n), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    if "shared" in how:
        values = values[:, :1, :1].expand(1, L, Hkv, n)
    dense = values.contiguous()
    room = torch.full((L, 3, Hkv, n + 8), -1.0, device="cuda")
    nov = dense.clone()
    if how == "layers first":
        nov = room[..., :n].transpose(0, 1)[1:2]
        nov.copy_(dense)
    elif how == "wide rows":
        nov = room.transpose(0, 1)[:1, ..., :n]
        nov.copy_(dense)
    elif how == "shared":
        nov = dense[:, 0, 0].contiguous()
    elif how == "shared by expansion":
        nov = dense[:, :1, :1].contiguous().expand(1, L, Hkv, n)
    keep = torch.empty((1, L, Hkv, k), dtype=torch.int32, device="cuda")
    assert pool.distill(0, page, Q_cat, nov, keep, None, k=k, T=30) == ip.CCD_OK
    other, other_page, _ = _full_pool(kind)
    want, want_keep = dense.clone(), torch.empty_like(keep)
    assert other.distill(0, other_page, Q_cat, want, want_keep, None, k=k, T=30) == ip.CCD_OK
    torch.cuda.synchronize()
    assert torch.equal(keep, want_keep)
    assert torch.equal(nov, {"shared": values[:, 0, 0], "shared by expansion": values}.get(how, want))
    assert torch.equal(want, torch.cat([torch.gather(dense, 3, want_keep.long()), dense[..., k:]], 3))
    for a, b in ((pool.K, other.K), (pool.V, other.V), (pool.K_scales, other.K_scales), (pool.V_scales, other.V_scales)):
        assert torch.equal(a[page].view(torch.uint8), b[other_page].view(torch.uint8))
    if how in ("layers first", "wide rows"):
        nov.fill_(-1.0)
        assert (room == -1.0).all()


@pytest.mark.parametrize("B,L,Hkv,d,P", [(2, 40, 16, 64, 4), (5, 3, 32, 128, 2), (2, 150, 5, 64, 1)])         # layers by 14, sequences by two, layers by 50 (log-sum-exps not on 16 bytes)
@pytest.mark.parametrize("with_lse", [False, True])
def test_keys_are_read_back_some_pots_at_a_time(B, L, Hkv, d, P, with_lse):
    """Scores, kept rows and what is left as of a plain pot that holds the same numbers; no buffer for all keys at once."""
    n, k = 64, 24
    pot = MemoryPot(B, L, Hkv, d, n, k, 6, codes=torch.int8)
    g = torch.Generator(device="cuda").manual_seed(B)
    _fill(pot, n, g)
    plain, before = _plain(pot, "int8"), _held(pot)
    Q = torch.randn((B, L, Hkv, P, d), generator=g, device="cuda").bfloat16()
    lse = pot.attend(Q, behind=True)[1] if with_lse else None
    scores = [torch.zeros((B, L, Hkv, n), device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    assert pot.distill(Q, scores=scores[0], lse=lse) == ip.CCD_OK
    assert torch.cuda.max_memory_allocated() - held < 0.6 * 2 * pot.K.numel()
    assert plain.distill(Q, scores=scores[1], lse=lse) == ip.CCD_OK
    torch.cuda.synchronize()
    assert _off(*scores) <= 3e-5
    keep = gu.to_host(pot.keep_idx)
    np.testing.assert_array_equal(keep, gu.replay_select(scores[0].cpu().numpy(), k))
    gu.assert_keep_matches(keep, gu.to_host(plain.keep_idx), scores[1].cpu().numpy(), k)
    _compacted(pot, before, keep)
