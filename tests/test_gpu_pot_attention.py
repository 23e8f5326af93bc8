"""Attention over memory pots: the drivers of pot.py end to end, against the references.

Tolerances as in test_gpu_paged.py for one attention call.  Scores from attention's own log-sum-exps against scores whose normalisers the score kernels
compute themselves: both are fp32 log-sum-exps of the same logits, 2e-5 off at most, and exp turns that into 2e-5 relative.
"""
import numpy as np
import pytest
import torch

from oracle import ccd_oracle as C
from oracle import paged_oracle as O
from paper_2410_01518_amd import infinipot as ip
from paper_2410_01518_amd import synth
from paper_2410_01518_amd.pot import MemoryPot, PagedPots
from tests import gpu_util as gu
from tests.test_gpu_paged import DT, _check_attend, _f64

pytestmark = pytest.mark.gpu


def _fill(pot, n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (pot.B, pot.L, pot.Hkv, n, pot.d)
    K, V = (torch.randn(shape, generator=g, device="cuda").to(pot.K.dtype) for _ in range(2))
    nov = torch.rand((pot.B, n), generator=g, device="cuda")
    pot.append(K, V, nov)
    return K, V, nov


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,behind", [(1, False), (40, False), (16, True)])
def test_memory_pot_attends(dtype, m, behind):
    B, L, Hkv, d, n_cap, Hq = 2, 2, 2, 64, 300, 6
    pot = MemoryPot(B, L, Hkv, d, n_cap, 100, 50, dtype=DT[dtype])
    _fill(pot, 170, 1)
    _fill(pot, 47, 2)
    Q = torch.randn((B, L, Hq, m, d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(DT[dtype])
    out, lse = pot.attend(Q, behind=behind)
    one, one_lse = pot.attend(Q[:, 1], layer=1, behind=behind)
    torch.cuda.synchronize()
    assert torch.equal(one, out[:, 1]) and torch.equal(one_lse, lse[:, 1])
    rows = B * L * m
    p = dict(Q=Q.transpose(2, 3).reshape(rows, Hq, d), K=pot.K.flatten(0, 1), V=pot.V.flatten(0, 1), table=np.arange(B * L)[:, None], q_start=np.arange(B * L + 1) * m,
             lens=np.full(B * L, 217), T=rows)
    _check_attend(p, out.transpose(2, 3).reshape(rows, Hq, d), lse.transpose(2, 3).reshape(rows, Hq), dtype, behind=behind)


@pytest.mark.parametrize("dtype,d,P", [("bf16", 128, 32), ("fp32", 64, 9)])
def test_distillation_with_attentions_own_log_sum_exps(dtype, d, P):
    """The catalyst prompt attends to the full pot; its log-sum-exps go into the compression.  Scores, kept tokens and rows as of the plain compression."""
    B, L, Hkv, Hq, n, k = 1, 2, 2, 8, 512, 200
    pots = [MemoryPot(B, L, Hkv, d, n, k, 40, dtype=DT[dtype]) for _ in range(2)]
    for pot in pots:
        _fill(pot, n, 5)
    Q = torch.randn((B, L, Hq, P, d), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(DT[dtype])
    scores = [torch.zeros((B, L, Hkv, n), device="cuda") for _ in pots]
    _, lse = pots[0].attend(Q, behind=True)
    assert pots[0].distill(Q, scores=scores[0], lse=lse) == ip.CCD_OK
    assert pots[1].distill(Q, scores=scores[1]) == ip.CCD_OK
    torch.cuda.synchronize()
    a, b = (x.cpu().numpy() for x in scores)
    assert (np.isinf(a) == np.isinf(b)).all()
    fin = np.isfinite(b)
    tol = 3e-5 if dtype == "bf16" else 2e-3            # (fp32, 64 elements: the score kernels split values, 1e-3 as in test_gpu_parity)
    assert (np.abs(a[fin] - b[fin]) <= tol * np.abs(b[fin]) + 1e-30).all()
    gu.assert_keep_matches(gu.to_host(pots[0].keep_idx), gu.to_host(pots[1].keep_idx), b, k)
    assert pots[0].n_valid == k
    # the pot goes on: new tokens behind the kept ones see them all
    _fill(pots[0], 30, 7)
    Q2 = torch.randn((B, Hq, 30, d), generator=torch.Generator(device="cuda").manual_seed(8), device="cuda").to(DT[dtype])
    out, lse = pots[0].attend(Q2, layer=0)
    torch.cuda.synchronize()
    p = dict(Q=Q2.transpose(1, 2).reshape(30, Hq, d), K=pots[0].K[:, 0], V=pots[0].V[:, 0], table=np.array([[0]]), q_start=np.array([0, 30]), lens=np.array([k + 30]), T=30)
    _check_attend(p, out.transpose(1, 2).reshape(30, Hq, d), lse.transpose(1, 2).reshape(30, Hq), dtype)


def test_paged_pots_serve_sequences_of_different_lengths():
    """Five sequences, two layers, pages of 16: chunks and single tokens, ends and starts; every layer's attention of every step."""
    S, L, Hq, Hkv, d, cap = 5, 2, 4, 2, 64, 150
    pool = PagedPots(S, 60, 16, 180, cap, L, Hq, Hkv, d, window=0)
    rng, g = np.random.default_rng(1), torch.Generator(device="cuda").manual_seed(1)
    hist = [[[] for _ in range(L)] for _ in range(S)]
    for step in range(7):
        lengths = [0 if rng.random() < 0.15 else min(180, n + (1 if rng.random() < 0.5 else int(rng.integers(0, 30)))) for n in pool.lengths]
        old = list(pool.lengths)
        total = pool.step(lengths)
        for layer in range(L):
            x = torch.randn((cap, Hq + 2 * Hkv, d), generator=g, device="cuda").bfloat16()
            Q, K, V = x[:, :Hq], x[:, Hq: Hq + Hkv], x[:, Hq + Hkv:]
            out, lse = torch.full((cap, Hq, d), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((cap, Hq), 5.0, device="cuda")
            pool.append(layer, K, V)
            pool.attend(layer, Q, out, lse)
            torch.cuda.synchronize()
            starts = pool.q_start.tolist()
            assert starts[-1] == total
            longest = max(1, max(lengths))
            Kp, Vp = (torch.zeros((S, Hkv, longest, d), device="cuda") for _ in range(2))
            for b in range(S):
                h = hist[b][layer] = [] if lengths[b] < old[b] else hist[b][layer]
                h += [(K[i], V[i]) for i in range(starts[b], starts[b + 1])]
                for t, (k, v) in enumerate(h):
                    Kp[b, :, t], Vp[b, :, t] = k.float(), v.float()
            p = dict(Q=Q, K=Kp, V=Vp, table=np.arange(S)[:, None], q_start=np.array(starts), lens=np.array(lengths), T=total)
            _check_attend(p, out, lse, "bf16")
    with pytest.raises(ValueError):
        pool.step([181] + pool.lengths[1:])
    with pytest.raises(ValueError):
        pool.step([n + 40 for n in pool.lengths])
    with pytest.raises(ValueError):
        PagedPots(S, 2, 16, 180, 1000, L, Hq, Hkv, d).step([30] * S)


def test_a_pool_of_pots_distils_one_sequence():
    """Pages that are whole pots: one sequence fills its pot and is distilled while the other goes on."""
    L, Hq, Hkv, d, n, k, P = 2, 4, 2, 128, 256, 96, 16
    pool = PagedPots(2, 3, n, n, n, L, Hq, Hkv, d)
    g = torch.Generator(device="cuda").manual_seed(2)
    assert pool.step([n, 0]) == n
    K, V = (torch.randn((L, n, Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    for layer in range(L):
        pool.append(layer, K[layer], V[layer])
    page = int(pool.table[0, 0])
    Q_cat = torch.randn((1, L, Hq, P, d), generator=g, device="cuda").bfloat16()
    nov = torch.rand((1, n), generator=g, device="cuda")
    keep = torch.empty((1, L, Hkv, k), dtype=torch.int32, device="cuda")
    shape = ip.make_shape(Q_cat, pool.K[page: page + 1], nov, k=k, T=30, pool_w=7)
    assert pool.distill(0, page, Q_cat, nov, keep, ip.alloc_workspace(shape), k=k, T=30) == ip.CCD_OK
    assert pool.lengths == [k, 0]
    kh = keep.cpu().numpy()
    ref = C.compress(gu.to_host(Q_cat), gu.to_host(K.transpose(1, 2)[None].contiguous()), gu.to_host(V.transpose(1, 2)[None].contiguous()), gu.to_host(nov), k=k, T=30, pool_w=7)
    gu.assert_keep_matches(kh, ref["keep_idx"], ref["scores"], k)
    assert pool.step([k + 3, 40]) == 43
    layer = 1
    x = torch.randn((43, Hq + 2 * Hkv, d), generator=g, device="cuda").bfloat16()
    pool.append(layer, x[:, Hq: Hq + Hkv], x[:, Hq + Hkv:])
    out, lse = pool.attend(layer, x[:, :Hq])
    torch.cuda.synchronize()
    assert int(pool.table[0, 0]) == page
    idx = torch.from_numpy(kh[0, layer].astype(np.int64)).cuda()
    Kp, Vp = (torch.zeros((2, Hkv, n, d), device="cuda") for _ in range(2))
    for h in range(Hkv):
        Kp[0, h, :k], Vp[0, h, :k] = K[layer, idx[h], h].float(), V[layer, idx[h], h].float()
    for b, (at, new, start) in enumerate(((k, 3, 0), (0, 40, 3))):
        Kp[b, :, at: at + new], Vp[b, :, at: at + new] = (x[start: start + new, Hq + o: Hq + o + Hkv].transpose(0, 1).float() for o in (0, Hkv))
    p = dict(Q=x[:, :Hq], K=Kp, V=Vp, table=np.array([[0], [1]]), q_start=np.array([0, 3, 43]), lens=np.array([k + 3, 40]), T=43)
    _check_attend(p, out, lse, "bf16")


def test_tensors_of_another_device_are_refused():
    x = torch.zeros((4, 2, 64), device="cuda")
    rope = ip.make_rope(x)
    with pytest.raises(ValueError):
        ip.ccd_rope(rope, x.cpu(), torch.zeros(4, dtype=torch.int32), ip.rope_turns(rope), x)


def test_streaming_recipe_runs():
    """A pot over a long context as a program has it: chunks appended and attending, distilled with the attention's log-sum-exps when full."""
    cfg = synth.scaled(synth.CONFIGS["c2"], Hq=8, Hkv=2, N=512, k=256, T=128)
    pot = MemoryPot(1, 1, cfg.Hkv, cfg.d, cfg.N, cfg.k, cfg.T)
    g = torch.Generator(device="cuda").manual_seed(9)
    for step in range(6):
        if pot.room < 128:
            Q_cat = torch.randn((1, 1, cfg.Hq, 16, cfg.d), generator=g, device="cuda").bfloat16()
            _, lse = pot.attend(Q_cat, behind=True)
            assert pot.distill(Q_cat, lse=lse) == ip.CCD_OK
        _fill(pot, 128, 20 + step)
        out, lse = pot.attend(torch.randn((1, 1, cfg.Hq, 128, cfg.d), generator=g, device="cuda").bfloat16())
        assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    assert pot.calls == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_attention_of_pots_stands_for_itself(dtype):
    """A graph captured before anything ran eagerly, replayed among eager calls over other lengths, other numbers of tokens and larger workspaces."""
    pot = MemoryPot(2, 2, 2, 64, 3000, 100, 50, dtype=DT[dtype])
    _fill(pot, 217, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    Q = torch.randn((2, 2, 6, 3, 64), generator=g, device="cuda").to(DT[dtype])
    big = torch.randn((2, 2, 6, 500, 64), generator=g, device="cuda").to(DT[dtype])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, lse = pot.attend(Q)
    before = pot.attend(Q)                                   # eager, before the first replay
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, before[0]) and torch.equal(lse, before[1])
    for n in (1, 1500):
        _fill(pot, n, 3)
        pot.attend(Q)
        _, large = pot.attend(big, behind=True)
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, before[0]) and torch.equal(lse, before[1])
        assert torch.isfinite(large).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_attention_over_a_pool(dtype):
    """append and attend of a decoding step in a graph: replayed for later steps of the same number of rows, between eager calls of others."""
    lens, L, Hq, Hkv, d = [40, 700, 1], 2, 4, 2, 64
    pools = [PagedPots(3, 80, 16, 1100, 64, L, Hq, Hkv, d, dtype=DT[dtype]) for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(4)
    make = lambda rows, heads: torch.randn((rows, heads, d), generator=g, device="cuda").to(DT[dtype])            # noqa: E731
    for start in range(0, 700, 20):                          # fill both alike
        now = [min(n, start + 20) for n in lens]
        rows = [p.step(now) for p in pools][0]
        K, V = make(64, Hkv), make(64, Hkv)
        for p in pools:
            for layer in range(L):
                p.append(layer, K, V)
    K, V, Q = make(3, Hkv), make(3, Hkv), make(3, Hq)
    now = [n + 1 for n in lens]
    for p in pools:
        assert p.step(now) == 3
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for layer in range(L):
            pools[0].append(layer, K, V)
        outs = [pools[0].attend(layer, Q) for layer in range(L)]
    for step in range(4):
        if step:
            now = [n + 1 for n in now]
            for p in pools:
                assert p.step(now) == 3
            for t, heads in ((K, Hkv), (V, Hkv), (Q, Hq)):
                t.copy_(make(3, heads))
        graph.replay()
        for layer in range(L):
            pools[1].append(layer, K, V)
        want = [pools[1].attend(layer, Q) for layer in range(L)]
        torch.cuda.synchronize()
        for (o, s), (wo, ws) in zip(outs, want):
            # (the cut may differ: the graph keeps the lengths that the host knew at its capture)
            slack = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -18
            A = pools[1].V.abs().max().double()
            assert ((o.double() - wo.double()).abs() <= slack * A).all() and ((s - ws).abs() <= 1e-4).all()
        if step == 1:                                        # a chunk in between, on both
            now = [now[0] + 50, now[1], now[2] + 3]
            k, v, q = make(64, Hkv), make(64, Hkv), make(64, Hq)
            for p in pools:
                assert p.step(now) == 53
                for layer in range(L):
                    p.append(layer, k, v)
                    p.attend(layer, q)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_pots_attention_on_two_streams_at_once(dtype):
    """Calls that nothing orders share no workspace and no index tensor."""
    pot = MemoryPot(2, 2, 2, 64, 3000, 100, 50, dtype=DT[dtype])
    _fill(pot, 2900, 5)
    g = torch.Generator(device="cuda").manual_seed(6)
    Qs = [torch.randn((2, 2, 6, m, 64), generator=g, device="cuda").to(DT[dtype]) for m in (1, 40)]
    want = [pot.attend(Q, behind=True) for Q in Qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in Qs]
    outs = [[], []]
    for _ in range(20):
        for i, (Q, stream) in enumerate(zip(Qs, streams)):
            with torch.cuda.stream(stream):
                outs[i].append(pot.attend(Q, behind=True))
    torch.cuda.synchronize()
    for (w, wl), got in zip(want, outs):
        for o, lse in got:
            assert torch.equal(o, w) and torch.equal(lse, wl)
