"""Pots and pools in 8 bits: the drivers of pot.py end to end, against the references.

Codes and scales of appended rows are compared bit for bit, attention within test_gpu_codes' tolerances against the numbers that the pot's own codes stand for.  A distillation's
scores are those of a plain pot that holds the numbers read back: the same keys, in other kernels' order of sums, so 3e-5 relative as in test_gpu_pot_attention (bf16; fp32 2e-3).
With attention's log-sum-exps, which are of the codes themselves, bf16 numbers differ by their rounding: half a step, 2^-9 of every |q k|.  With M the largest scale * sum|q k| of a row
a logit is off by 2^-9 M, a log-sum-exp by no more, and a score by exp(2^-8 M) - 1 relative.
"""
import numpy as np
import pytest
import torch

from oracle import codes_oracle as C
from paper_2410_01518_amd import infinipot as ip
from paper_2410_01518_amd.pot import MemoryPot, PagedPots
from tests import gpu_util as gu
from tests.test_gpu_codes import CODE, _bytes, _check_attend
from tests.test_gpu_paged import DT, _f64

pytestmark = pytest.mark.gpu


def _new(g, *shape, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * torch.exp(torch.randn((*shape[:-1], 1), generator=g, device="cuda"))).to(dtype)


def _fill(pot, n, g):
    shape = (pot.B, pot.L, pot.Hkv, n, pot.d)
    K, V, nov = _new(g, *shape, dtype=pot.dtype), _new(g, *shape, dtype=pot.dtype), torch.rand((pot.B, n), generator=g, device="cuda")
    pot.append(K, V, nov)
    return K, V, nov


def _seen(pot, Q, kind, m):
    """What _check_attend takes: pages are the pots of all sequences and layers."""
    pages, Hq = pot.B * pot.L, Q.shape[2]
    flat = {n: x.flatten(0, 1) for n, x in (("K", pot.K), ("V", pot.V), ("Ks", pot.K_scales), ("Vs", pot.V_scales))}
    return dict(flat, Q=Q.transpose(2, 3).reshape(pages * m, Hq, pot.d), kind=kind, rows=1, table=np.arange(pages)[:, None], q_start=np.arange(pages + 1) * m,
                lens=np.full(pages, pot.n_valid), T=pages * m)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,behind", [(1, False), (40, False), (16, True)])
def test_memory_pot(kind, dtype, m, behind):
    B, L, Hkv, d, n_cap, Hq = 2, 2, 2, 64, 300, 6
    g = torch.Generator(device="cuda").manual_seed(1)
    pot = MemoryPot(B, L, Hkv, d, n_cap, 100, 50, dtype=DT[dtype], codes=CODE[kind])
    want = [(_bytes(x.flatten(0, 1)), s.flatten(0, 1).cpu().numpy()) for x, s in ((pot.K, pot.K_scales), (pot.V, pot.V_scales))]
    for n in (170, 47):
        slots = (np.arange(B * L)[:, None] * n_cap + pot.n_valid + np.arange(n)).reshape(-1)
        K, V, nov = _fill(pot, n, g)
        for x, w in zip((K, V), want):
            C.append(_f64(x.transpose(2, 3).reshape(B * L * n, Hkv, d)), slots, *w, kind, 1)
    torch.cuda.synchronize()
    for (bits, scales), x, s in zip(want, (pot.K, pot.V), (pot.K_scales, pot.V_scales)):
        np.testing.assert_array_equal(_bytes(x.flatten(0, 1)), bits)
        np.testing.assert_array_equal(s.flatten(0, 1).cpu().numpy(), scales)
    assert torch.equal(pot.novelty[:, :, :, 170:217], nov[:, None, None].expand(B, L, Hkv, 47))
    Q = torch.randn((B, L, Hq, m, d), generator=g, device="cuda").to(DT[dtype])
    out, lse = pot.attend(Q, behind=behind)
    one, one_lse = pot.attend(Q[:, 1], layer=1, behind=behind)
    other, other_lse = pot.attend(Q, behind=behind, K=(pot.V, pot.V_scales))
    torch.cuda.synchronize()
    assert torch.equal(one, out[:, 1]) and torch.equal(one_lse, lse[:, 1])
    p = _seen(pot, Q, kind, m)
    rows = lambda x: x.transpose(2, 3).reshape(p["T"], Hq, *x.shape[4:])                               # noqa: E731
    _check_attend(p, rows(out), rows(lse), dtype, behind=behind)
    _check_attend({**p, "K": p["V"], "Ks": p["Vs"]}, rows(other), rows(other_lse), dtype, behind=behind)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,P,with_lse", [("bf16", 128, 32, False), ("bf16", 128, 32, True), ("fp32", 64, 9, True), ("bf16", 64, 16, False)])
def test_distillation(kind, dtype, d, P, with_lse):
    """A pot in 8 bits against a plain one that holds the same numbers; then tokens behind the kept ones, and a second distillation."""
    B, L, Hkv, Hq, n, k = 1, 2, 2, 8, 512, 200
    g = torch.Generator(device="cuda").manual_seed(5)
    pot = MemoryPot(B, L, Hkv, d, n, k, 40, dtype=DT[dtype], codes=CODE[kind])
    for part in (n, n - k):
        if part < n:
            assert pot.distill(Q) == ip.CCD_NOOP                       # not full
        _fill(pot, part, g)
        plain = MemoryPot(B, L, Hkv, d, n, k, 40, dtype=DT[dtype])
        numbers = [torch.from_numpy(C.decode(_bytes(x.flatten(0, 1)), s.flatten(0, 1).cpu().numpy(), kind, 1)).view(B, L, Hkv, n, d).cuda().to(DT[dtype])
                   for x, s in ((pot.K, pot.K_scales), (pot.V, pot.V_scales))]
        plain.K.copy_(numbers[0])
        plain.V.copy_(numbers[1])
        plain.novelty.copy_(pot.novelty)
        plain.n_valid = n
        Q = torch.randn((B, L, Hq, P, d), generator=g, device="cuda").to(DT[dtype])
        before = [_bytes(pot.K), _bytes(pot.V), pot.K_scales.cpu().numpy(), pot.V_scales.cpu().numpy(), pot.novelty.cpu().numpy()]
        scores = [torch.zeros((B, L, Hkv, n), device="cuda") for _ in range(2)]
        lse = pot.attend(Q, behind=True)[1] if with_lse else None
        assert pot.distill(Q, scores=scores[0], lse=lse) == ip.CCD_OK
        assert plain.distill(Q, scores=scores[1]) == ip.CCD_OK
        torch.cuda.synchronize()
        a, b = (x.cpu().numpy() for x in scores)
        assert (np.isinf(a) == np.isinf(b)).all()
        fin = np.isfinite(b)
        M = float(torch.matmul(Q.abs().float().view(B, L, Hkv, -1, d), numbers[0].abs().float().transpose(-1, -2).contiguous()).max()) / d ** 0.5
        tol = 2e-3 if dtype == "fp32" else 3e-5 + (np.expm1(2.0 ** -8 * M) if with_lse else 0.0)
        assert (np.abs(a[fin] - b[fin]) <= tol * np.abs(b[fin]) + 1e-30).all()
        keep = gu.to_host(pot.keep_idx)
        gu.check_keep_valid(keep, n, k)
        np.testing.assert_array_equal(keep, gu.replay_select(a, k))
        if not with_lse:
            gu.assert_keep_matches(keep, gu.to_host(plain.keep_idx), b, k)
        got = [_bytes(pot.K), _bytes(pot.V), pot.K_scales.cpu().numpy(), pot.V_scales.cpu().numpy(), pot.novelty.cpu().numpy()]
        flat = keep.reshape(B * L, Hkv, k)
        for x, y in zip(got, before):
            np.testing.assert_array_equal(x.reshape(B * L, Hkv, *x.shape[3:]), C.compact(y.reshape(B * L, Hkv, *y.shape[3:]), flat))
        assert pot.n_valid == k
        _fill(pot, 3, g)
        Q2 = torch.randn((B, L, Hq, 3, d), generator=g, device="cuda").to(DT[dtype])
        out, lse2 = pot.attend(Q2)
        torch.cuda.synchronize()
        p = _seen(pot, Q2, kind, 3)
        _check_attend(p, out.transpose(2, 3).reshape(p["T"], Hq, d), lse2.transpose(2, 3).reshape(p["T"], Hq), dtype)
        pot.n_valid = k
    assert pot.calls == 2


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 16)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_paged_pots_serve_sequences_of_different_lengths(kind, rows, dtype):
    """Five sequences, two layers, pages of 16: chunks and single tokens, ends and starts; every layer's codes, scales and attention of every step, eagerly and in a graph of
    its own that is replayed among them."""
    S, L, Hq, Hkv, d, cap, n_pages = 5, 2, 4, 2, 64, 150, 60
    pool = PagedPots(S, n_pages, 16, 180, cap, L, Hq, Hkv, d, dtype=DT[dtype], codes=CODE[kind], scale_rows=rows)
    rng, g = np.random.default_rng(1), torch.Generator(device="cuda").manual_seed(1)
    want = [[(_bytes(x[:, i]), s[:, i].cpu().numpy()) for x, s in ((pool.K, pool.K_scales), (pool.V, pool.V_scales))] for i in range(L)]
    x = torch.zeros((cap, Hq + 2 * Hkv, d), dtype=DT[dtype], device="cuda")
    Q, K, V = x[:, :Hq], x[:, Hq: Hq + Hkv], x[:, Hq + Hkv:]
    out, lse = torch.zeros((cap, Hq, d), dtype=DT[dtype], device="cuda"), torch.zeros((cap, Hq), device="cuda")
    graph = None

    def layer_step(layer):
        pool.append(layer, K, V)
        pool.attend(layer, Q, out, lse)

    for step in range(8):
        lengths = [0 if rng.random() < 0.15 else min(180, n + (1 if rng.random() < 0.5 else int(rng.integers(0, 30)))) for n in pool.lengths]
        total = pool.step(lengths)
        for layer in range(L):
            x.copy_(_new(g, cap, Hq + 2 * Hkv, d, dtype=DT[dtype]))
            out.fill_(5.0)
            lse.fill_(5.0)
            if step >= 3 and layer == 1:
                if graph is None:
                    pool._most = (cap, 180)                             # (hints that hold for all steps)
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        layer_step(layer)
                graph.replay()
            else:
                layer_step(layer)
            torch.cuda.synchronize()
            slots = pool.slots.cpu().numpy()
            for t, w in zip((K, V), want[layer]):
                C.append(_f64(t), slots, *w, kind, rows)
            for (bits, scales), c, s in zip(want[layer], (pool.K, pool.V), (pool.K_scales, pool.V_scales)):
                np.testing.assert_array_equal(_bytes(c[:, layer]), bits)
                np.testing.assert_array_equal(s[:, layer].cpu().numpy(), scales)
            p = dict(Q=Q, K=pool.K[:, layer], V=pool.V[:, layer], Ks=pool.K_scales[:, layer], Vs=pool.V_scales[:, layer], kind=kind, rows=rows, table=pool.table.cpu().numpy(),
                     q_start=pool.q_start.cpu().numpy(), lens=np.array(lengths), T=total)
            _check_attend(p, out, lse, dtype)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_a_pool_of_pots_distils_one_sequence(kind):
    L, Hq, Hkv, d, n, k, P = 2, 4, 2, 128, 256, 96, 16
    pool = PagedPots(2, 3, n, n, n + 10, L, Hq, Hkv, d, codes=CODE[kind])
    g = torch.Generator(device="cuda").manual_seed(2)
    assert pool.step([n, 7]) == n + 7
    for layer in range(L):
        pool.append(layer, _new(g, n + 7, Hkv, d, dtype=torch.bfloat16), _new(g, n + 7, Hkv, d, dtype=torch.bfloat16))
    page, other = int(pool.table[0, 0]), int(pool.table[1, 0])
    before = [_bytes(pool.K), _bytes(pool.V), pool.K_scales.cpu().numpy(), pool.V_scales.cpu().numpy()]
    Q_cat = torch.randn((1, L, Hq, P, d), generator=g, device="cuda").bfloat16()
    nov = torch.rand((1, n), generator=g, device="cuda")
    keep = torch.empty((1, L, Hkv, k), dtype=torch.int32, device="cuda")
    args = dict(k=k, T=30)
    assert pool.distill(1, other, Q_cat, nov, keep, None, **args) == ip.CCD_NOOP
    assert pool.distill(0, page, Q_cat, nov, keep, None, **args) == ip.CCD_OK
    torch.cuda.synchronize()
    assert pool.lengths == [k, 7]
    kh = keep.cpu().numpy()[0]
    gu.check_keep_valid(kh, n, k)
    for x, y in zip((_bytes(pool.K), _bytes(pool.V), pool.K_scales.cpu().numpy(), pool.V_scales.cpu().numpy()), before):
        np.testing.assert_array_equal(x[page], C.compact(y[page], kh))
        rest = [i for i in range(3) if i != page]
        np.testing.assert_array_equal(x[rest], y[rest])
    assert pool.step([k + 1, 8]) == 2
    Q = torch.randn((2, Hq, d), generator=g, device="cuda").bfloat16()
    pool.append(1, _new(g, 2, Hkv, d, dtype=torch.bfloat16), _new(g, 2, Hkv, d, dtype=torch.bfloat16))
    out, lse = pool.attend(1, Q)
    torch.cuda.synchronize()
    p = dict(Q=Q, K=pool.K[:, 1], V=pool.V[:, 1], Ks=pool.K_scales[:, 1], Vs=pool.V_scales[:, 1], kind=kind, rows=1, table=pool.table.cpu().numpy(), q_start=np.array([0, 1, 2]),
             lens=np.array([k + 1, 8]), T=2)
    _check_attend(p, out, lse, "bf16")


def test_types_of_code_that_there_are_not():
    with pytest.raises(TypeError):
        MemoryPot(1, 1, 1, 64, 16, 8, 4, codes=torch.uint8)
    with pytest.raises(TypeError):
        PagedPots(1, 1, 16, 16, 16, 1, 1, 1, 64, codes=torch.float8_e5m2)
