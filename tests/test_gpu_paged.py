"""GPU parity of the paged cache's operators through the C ABI, against the 64-bit reference.

Tolerances (derived from the arithmetic).
Rotary positions: cosine and sine are within 2^-22 (the angle within an eighth of a turn is rounded once, 2^-24 of at most pi/4, and the
sums of ten terms round by a few 2^-24 of 1); a product and an fma add 2^-23 of each product: |dy| <= 2^-21 a (|x_1| + |x_2|), and a bf16
result half a step more, 2^-8 |y|.
Attention: a logit is off by at most e = (d + 8) 2^-24 scale sum|q k| (fp32 sums of exact products in any order, one scaling), so a
weight by 2 e relative; 2^x adds 2^-22; sums of n weights and of n products by n 2^-24.  With A = sum w|v| / sum w:
|do| <= A (2 e + 2 n 2^-24 + 2^-20), and with bf16 caches half a step of the weights and of the result more: 2^-8 A + 2^-8 |o|.
|d lse| <= e + n 2^-24 + 2^-20 + 2^-22 |lse|.
"""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2410_01518_amd import infinipot as ip

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _dev(a):
    return torch.as_tensor(np.ascontiguousarray(a), device="cuda")


def _f64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ plan

def _plan_problem(rng, B, W, page, spare, grow=3.0, broken=0.0):
    longest = W * page
    before = rng.integers(0, longest + 1, B)
    what = rng.integers(0, 6, B)
    after = np.where(what == 0, 0, np.where(what == 1, before // 2, np.where(what == 2, before, np.minimum(longest, before + 1 + (rng.random(B) ** 4 * grow * page).astype(int)))))
    before = np.where(what == 5, 0, before)
    held = -(-before // page)
    need = np.maximum(0, -(-after // page) - held).sum()
    n_pages = int(held.sum() + max(0, need + spare) + 1)
    ids = rng.permutation(n_pages).astype(np.int32)
    table, at = np.full((B, W), -1, np.int32), 0
    for b in range(B):
        table[b, :held[b]] = ids[at: at + held[b]]
        at += held[b]
    free = ids[at:]
    head = int(rng.integers(0, n_pages))
    ring = np.full(n_pages, -1, np.int32)
    ring[(head + np.arange(len(free))) % n_pages] = free
    if broken:
        hit = rng.random(table.shape) < broken
        table[hit] = rng.choice([-1, -5, n_pages, 1 << 30], hit.sum())
    tokens = int(np.maximum(0, after - before).sum())
    return before.astype(np.int32), after.astype(np.int32), table, ring, np.array([head, len(free), 0, 0], np.int32), n_pages, tokens


def _run_plan(before, after, table, ring, cursor, *, page, n_pages, tokens, in_place, stream=None):
    t = {k: _dev(v) for k, v in dict(before=before, after=after, table=table, ring=ring, cursor=cursor).items()}
    nxt = t["table"] if in_place else torch.full_like(t["table"], 77)
    cur = t["cursor"] if in_place else torch.full_like(t["cursor"], 77)
    q_start = torch.full((len(before) + 1,), 77, dtype=torch.int32, device="cuda")
    slots, pos = (torch.full((tokens + 4,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    plan = ip.make_plan(t["table"], tokens=tokens, page=page, n_pages=n_pages)
    torch.cuda.synchronize()
    assert ip.ccd_paged_plan(plan, t["before"], t["after"], t["table"], nxt, t["ring"], t["cursor"], cur, q_start, slots, pos, stream=stream) == ip.CCD_OK
    torch.cuda.synchronize()
    assert (slots[tokens:] == 77).all() and (pos[tokens:] == 77).all()
    if not in_place:
        np.testing.assert_array_equal(t["table"].cpu().numpy(), table)
        np.testing.assert_array_equal(t["cursor"].cpu().numpy(), cursor)
    return [x.cpu().numpy() for x in (nxt, t["ring"], cur, q_start, slots[:tokens], pos[:tokens])]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,W,page,spare,pad,broken", [
    (1, 1, 1, 0, 0, 0), (1, 300, 3, 2, 5, 0), (7, 5, 16, 9, 0, 0), (64, 33, 100, -20, 3, 0), (511, 9, 4, 50, 0, 0), (512, 9, 7, 50, 1, 0), (513, 9, 4, -100, 0, 0),
    (1500, 70, 1, 0, 9, 0), (4096, 3, 5, 7, 0, 0), (4095, 3, 5, 7, 0, 0), (40, 600, 2, 30, 0, 0), (40, 20, 8, -3, 0, 0.1), (3, 4096, 1, 0, 0, 0),
])
def test_plan(B, W, page, spare, pad, broken, in_place):
    print(f"plan B={B} W={W} page={page} spare={spare} broken={broken} in_place={in_place}", flush=True)
    rng = np.random.default_rng(B * 1000 + W)
    before, after, table, ring, cursor, n_pages, tokens = _plan_problem(rng, B, W, page, spare, broken=broken)
    tokens = max(0, tokens + pad)
    got = _run_plan(before, after, table, ring, cursor, page=page, n_pages=n_pages, tokens=tokens, in_place=in_place)
    want = O.plan(before, after, table, ring, cursor, page=page, n_pages=n_pages, tokens=tokens)
    if in_place and broken:              # entries behind the held ones that are neither taken nor given back stay
        kept = np.arange(W)[None, :] >= np.maximum(-(-before // page), -(-after // page))[:, None]
        want[0][kept] = table[kept]
    for name, g, w in zip(("table", "ring", "cursor", "q_start", "slots", "positions"), got, want):
        np.testing.assert_array_equal(g, w, err_msg=name)


def test_plan_with_lengths_beyond_the_table_and_negative_ones():
    """More tokens than a row of the table holds: counted as missing, their slots -1; negative lengths are 0; a slot map too short is cut."""
    before, after = np.array([5, -3, 30, -7], np.int32), np.array([40, 2, -1, -2], np.int32)
    table = np.array([[4, 5, -1], [-1, -1, -1], [6, 7, 8], [-1, -1, -1]], np.int32)
    ring, cursor = np.array([0, 1, 2, 3, -1, -1, -1, -1, -1], np.int32), np.array([0, 4, 0, 0], np.int32)
    for tokens in (37, 50, 3, 0):
        got = _run_plan(before, after, table, ring, cursor, page=4, n_pages=9, tokens=tokens, in_place=False)
        want = O.plan(before, after, table, ring, cursor, page=4, n_pages=9, tokens=tokens)
        for g, w in zip(got, want):
            np.testing.assert_array_equal(g, w)


def test_plans_follow_each_other_in_place_and_in_a_replayed_graph():
    """A scheduler's loop: lengths change on the device, table, ring and cursor move in place.  Every page is held or free once at every step."""
    rng = np.random.default_rng(3)
    B, W, page, n_pages = 37, 24, 8, 500
    table, cursor = np.full((B, W), -1, np.int32), np.array([123, n_pages, 0, 0], np.int32)
    ring = rng.permutation(n_pages).astype(np.int32)
    lens = np.zeros(B, np.int32)
    d = {k: _dev(v) for k, v in dict(table=table, ring=ring, cursor=cursor, before=lens, after=lens).items()}
    q_start, slots, pos = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, 900, 900))
    plan = ip.make_plan(d["table"], tokens=900, page=page, n_pages=n_pages)

    def call():
        ip.ccd_paged_plan(plan, d["before"], d["after"], d["table"], d["table"], d["ring"], d["cursor"], d["cursor"], q_start, slots, pos)

    call()                                  # (nothing grows yet)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(12):
        nxt = np.where(rng.random(B) < 0.2, 0, np.minimum(W * page, lens + rng.integers(0, 40, B))).astype(np.int32)
        d["before"].copy_(torch.from_numpy(lens))
        d["after"].copy_(torch.from_numpy(nxt))
        want = O.plan(lens, nxt, table, ring, cursor, page=page, n_pages=n_pages, tokens=900)
        graph.replay() if step % 3 else call()
        torch.cuda.synchronize()
        got = [x.cpu().numpy() for x in (d["table"], d["ring"], d["cursor"], q_start, slots, pos)]
        for g, w in zip(got, want):
            np.testing.assert_array_equal(g, w)
        table, ring, cursor, lens = got[0], got[1], got[2], nxt
        held = table[table >= 0]
        free = ring[(cursor[0] + np.arange(cursor[1])) % n_pages]
        if want[2][2] == 0:
            assert sorted(np.concatenate([held, free])) == list(range(n_pages))


# ------------------------------------------------------------------------------------------------ rotary positions

def _rope_bound(x, y, rot, half, dtype, amplitude):
    n = rot // 2
    size = np.zeros_like(y)
    one, two = (np.arange(n), np.arange(n) + n) if half else (2 * np.arange(n), 2 * np.arange(n) + 1)
    size[..., one] = size[..., two] = np.abs(x[..., one]) + np.abs(x[..., two])
    return 2.0 ** -21 * amplitude * size + (2.0 ** -8 * np.abs(y) if dtype == "bf16" else 0.0) + 1e-37


ROPE = [  # dtype, tokens, heads, d, rot, layout
    ("bf16", 1, 1, 128, 128, "half"), ("bf16", 37, 40, 128, 128, "half"), ("bf16", 37, 40, 128, 128, "pairs"), ("bf16", 5, 3, 64, 32, "half"), ("bf16", 5, 3, 64, 32, "pairs"),
    ("bf16", 9, 7, 128, 90, "half"), ("bf16", 9, 7, 128, 90, "pairs"), ("bf16", 300, 12, 80, 80, "half"), ("bf16", 2, 5, 1024, 512, "half"), ("bf16", 2, 5, 1024, 1024, "pairs"),
    ("bf16", 2, 2, 8, 2, "half"), ("fp32", 37, 5, 128, 128, "half"), ("fp32", 37, 5, 64, 64, "pairs"), ("fp32", 11, 33, 128, 64, "half"), ("fp32", 3, 2, 4, 4, "pairs"),
    ("fp32", 3, 2, 1024, 1000, "half"), ("fp32", 4, 9, 128, 66, "pairs"), ("fp32", 1100, 2, 64, 24, "half"),
    # turned parts of no whole pieces, through more heads than one batch
    ("bf16", 1050, 72, 64, 60, "half"), ("bf16", 1050, 72, 64, 58, "pairs"), ("fp32", 1030, 40, 128, 118, "half"), ("fp32", 7, 40, 128, 126, "pairs"), ("bf16", 6, 131, 64, 2, "pairs"),
    ("bf16", 3, 20, 512, 300, "pairs"),
]


@pytest.mark.parametrize("case", range(len(ROPE)))
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(case, inverse):
    dtype, T, H, d, rot, layout = ROPE[case]
    print("rope", ROPE[case], inverse, flush=True)
    rng = np.random.default_rng(case)
    amplitude = 1.0 if case % 2 else 1.25
    scaling = (ip.CCD_ROPE_PLAIN, ip.CCD_ROPE_LINEAR, ip.CCD_ROPE_NTK, ip.CCD_ROPE_PARTS)[case % 4]
    wide = torch.randn((T, H + 2, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(case)).to(DT[dtype])
    X = wide[:, 1: H + 1]                                                     # heads in the middle of a projection
    positions = rng.integers(0, (1 << 31) - 1, T).astype(np.int32)
    positions[0] = 0
    if T > 4:
        positions[3], positions[4] = -1, 2 ** 31 - 1                          # padding; the last position there is
    Y = torch.full((T + 1, H, d), 7.0, dtype=DT[dtype], device="cuda")
    rope = ip.make_rope(X, Y[:T], rot=rot, layout=ip.CCD_ROPE_HALF if layout == "half" else ip.CCD_ROPE_PAIRS, base=500000.0, scaling=scaling, factor=8.0,
                        context=8192, amplitude=amplitude if case % 2 == 0 else 0.0, inverse=inverse)
    turns = ip.rope_turns(rope)
    assert ip.ccd_rope(rope, X, _dev(positions), turns, Y) == ip.CCD_OK
    torch.cuda.synchronize()
    # angles from the library's own frequencies, whole turns taken off in exact arithmetic: 64-bit floats lose 2^-22 turns at the last positions
    whole = [int(v) for v in turns.cpu().numpy().view(np.uint64)]
    x, got = _f64(X), _f64(Y)
    want = np.empty_like(x)
    for t in range(T):
        f = np.array([(int(positions[t]) * w % 2 ** 64) / 2.0 ** 64 * 2 * np.pi for w in whole])
        want[t] = O.rope(x[t: t + 1], [1], f, half=layout == "half", inverse=inverse, amplitude=amplitude)[0]
    here = positions >= 0
    assert (got[:T][~here] == 7.0).all() and (got[T:] == 7.0).all()
    err = np.abs(got[:T] - want)[here]
    assert (err <= _rope_bound(x, want, rot, layout == "half", dtype, amplitude)[here]).all(), err.max()
    if rot < d:
        np.testing.assert_array_equal(got[:T][here][..., rot:], x[here][..., rot:])
    # in place
    before = wide.clone()
    rope = ip.make_rope(X, rot=rot, layout=rope.layout, amplitude=rope.amplitude, inverse=inverse)
    assert ip.ccd_rope(rope, X, _dev(positions), turns, X) == ip.CCD_OK
    torch.cuda.synchronize()
    assert torch.equal(X[torch.from_numpy(here).cuda()], Y[:T][torch.from_numpy(here).cuda()])
    assert torch.equal(X[torch.from_numpy(~here).cuda()], before[:, 1: H + 1][torch.from_numpy(~here).cuda()])
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, -1], before[:, -1])


@pytest.mark.parametrize("layout", [0, 1])
def test_rope_inverse_is_the_gradient(layout):
    """<dy, rope(x)> is linear in x: its gradient is rope turned back, which is `inverse`; checked against autograd of the formula and
    against differences (linear: exact up to rounding, 2^-20 of the terms' size)."""
    T, H, d, rot = 6, 3, 64, 48
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((T, H, d), generator=g, device="cuda") for _ in range(2))
    pos = torch.randint(0, 100000, (T,), generator=g, device="cuda", dtype=torch.int32)
    fwd, bwd = ip.make_rope(x, rot=rot, layout=layout, amplitude=1.5), ip.make_rope(x, rot=rot, layout=layout, amplitude=1.5, inverse=True)
    turns, y, dx = ip.rope_turns(fwd), torch.empty_like(x), torch.empty_like(x)
    ip.ccd_rope(bwd, dy, pos, turns, dx)
    leaf = x.double().requires_grad_()
    ang = pos.double()[:, None] * torch.from_numpy(O.frequencies(rot, 10000.0)).cuda()
    z = torch.polar(torch.full_like(ang, 1.5), ang)[:, None]
    if layout == 0:
        w = torch.complex(leaf[..., :rot // 2], leaf[..., rot // 2: rot]) * z
        out = torch.cat([w.real, w.imag, leaf[..., rot:]], -1)
    else:
        w = torch.complex(leaf[..., 0:rot:2], leaf[..., 1:rot:2]) * z
        out = torch.cat([torch.stack([w.real, w.imag], -1).flatten(-2), leaf[..., rot:]], -1)
    (grad,) = torch.autograd.grad(out, leaf, dy.double())
    assert (dx.double() - grad).abs().max() <= 2.0 ** -20 * 1.5 * 2 * dy.abs().max()
    h = torch.randn((T, H, d), generator=g, device="cuda")
    lo, hi = torch.empty_like(x), torch.empty_like(x)
    ip.ccd_rope(fwd, x + h, pos, turns, hi)
    ip.ccd_rope(fwd, x - h, pos, turns, lo)
    slope = ((hi.double() - lo.double()) / 2 * dy.double()).sum()
    assert (slope - (dx.double() * ((x + h).double() - (x - h).double()) / 2).sum()).abs() <= 2.0 ** -20 * 1.5 * 4 * (dy.abs() * (x.abs() + h.abs()).amax()).sum()


# ------------------------------------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype,T,Hkv,d,page,n_pages,rot,layout", [
    ("bf16", 1, 1, 128, 1, 3, 0, 0), ("bf16", 70, 8, 128, 16, 9, 128, 0), ("bf16", 70, 8, 128, 16, 9, 128, 1), ("bf16", 33, 3, 64, 37, 4, 32, 1), ("bf16", 1030, 2, 64, 100, 11, 0, 0),
    ("fp32", 45, 5, 64, 7, 20, 64, 0), ("fp32", 45, 1, 128, 64, 3, 128, 1), ("fp32", 9, 13, 128, 5, 5, 50, 0), ("fp32", 9, 3, 64, 5, 5, 0, 0), ("bf16", 20, 3, 128, 3000, 1, 90, 0),
])
@pytest.mark.parametrize("order", ["heads first", "rows first"])
def test_append(dtype, T, Hkv, d, page, n_pages, rot, layout, order):
    print("append", dtype, T, Hkv, d, page, n_pages, rot, layout, order, flush=True)
    rng = np.random.default_rng(T + d)
    g = torch.Generator(device="cuda").manual_seed(T)
    shape = (n_pages, Hkv, page, d) if order == "heads first" else (n_pages, page, Hkv, d)
    Kb, Vb = (torch.full(shape, v, dtype=DT[dtype], device="cuda") for v in (7.0, 9.0))
    K, V = (x if order == "heads first" else x.transpose(1, 2) for x in (Kb, Vb))
    new = torch.randn((T + 2, 2, Hkv, d), generator=g, device="cuda").to(DT[dtype])
    K_new, V_new = new[:T, 0], new[:T, 1]
    slots = rng.permutation(page * n_pages)[:T].astype(np.int32)
    dead = rng.random(T) < 0.1
    slots[dead] = rng.choice([-1, -9, page * n_pages, 2 ** 31 - 1], dead.sum())
    positions = rng.integers(0, 1 << 20, T).astype(np.int32)
    paged = ip.make_paged(K, tokens=T, K_new=K_new)
    kw, want_k = {}, _f64(K_new)
    if rot:
        rope = ip.make_rope(K_new, rot=rot, layout=layout)
        kw = dict(rope=rope, positions=_dev(positions), turns=ip.rope_turns(rope))
        want_k = O.rope(want_k, positions, O.frequencies(rot, 10000.0), half=layout == ip.CCD_ROPE_HALF)
    assert ip.ccd_paged_append(paged, K_new, V_new, _dev(slots), K, V, **kw) == ip.CCD_OK
    torch.cuda.synchronize()
    gk, gv = _f64(K), _f64(V)
    wk, wv, tol = np.full(gk.shape, 7.0), np.full(gv.shape, 9.0), np.zeros(gk.shape)
    x = _f64(K_new)
    for t in range(T):
        if 0 <= slots[t] < page * n_pages:
            wk[slots[t] // page, :, slots[t] % page], wv[slots[t] // page, :, slots[t] % page] = want_k[t], _f64(V_new)[t]
            if rot:
                tol[slots[t] // page, :, slots[t] % page] = _rope_bound(x[t], want_k[t], rot, layout == 0, dtype, 1.0)
                tol[slots[t] // page, :, slots[t] % page, rot:] = 0.0
    np.testing.assert_array_equal(gv, wv)
    assert (np.abs(gk - wk) <= tol).all(), np.abs(gk - wk).max()


# ------------------------------------------------------------------------------------------------ attention

def _attend_problem(seed, dtype, lens, news, Hq, Hkv, d, page, *, W=None, pad=0, rows_first=False, holes=0.0, gain=1.0):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    W = W or max(1, max(-(-max(0, n) // page) for n in lens))
    held = [min(W, -(-max(0, n) // page)) for n in lens]
    n_pages = sum(held) + 2
    ids, at = rng.permutation(n_pages).astype(np.int32), 0
    table = np.full((len(lens), W), -1, np.int32)
    for b, h in enumerate(held):
        table[b, :h] = ids[at: at + h]
        at += h
    shape = (n_pages, page, Hkv, d) if rows_first else (n_pages, Hkv, page, d)
    K, V = ((torch.randn(shape, generator=g, device="cuda") * s).to(DT[dtype]) for s in (gain, 1.0))
    if rows_first:
        K, V = K.transpose(1, 2), V.transpose(1, 2)
    # what no sequence holds is not a number: pages of nobody, rows behind the last token
    used = np.zeros((n_pages, page), bool)
    for b, n in enumerate(lens):
        for c in range(held[b]):
            used[table[b, c], :max(0, min(page, n - c * page))] = True
    dead = torch.from_numpy(~used).cuda()[:, None, :, None]
    K.masked_fill_(dead, float("nan"))
    V.masked_fill_(dead, float("nan"))
    if holes:
        hit = rng.random(table.shape) < holes
        table[hit] = rng.choice([-1, n_pages, -(1 << 31), (1 << 31) - 1], hit.sum())
    T = sum(news)
    Q = torch.randn((T + pad, Hq, d), generator=g, device="cuda").to(DT[dtype])
    q_start = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    return dict(Q=Q, K=K, V=V, table=table, q_start=q_start, lens=np.array(lens, np.int32), T=T, pad=pad)


def _check_attend(p, out, lse, dtype, *, window=0, behind=False, scale=0.0, sentinel=5.0):
    K, V = (np.nan_to_num(_f64(p[x]), nan=0.0, posinf=np.inf, neginf=-np.inf) for x in "KV")
    want, want_lse, size, logit = O.attend(_f64(p["Q"]), K, V, p["table"], p["q_start"], p["lens"], window=window, behind=behind, scale=scale)
    got, T, d = _f64(out), p["T"], p["Q"].shape[-1]
    assert (got[T:] == sentinel).all()
    e = (d + 8) * 2.0 ** -24 * logit
    n = np.maximum(1, p["lens"].max()) * 2.0 ** -24
    tol = size * (2 * e[..., None] + 2 * n + 2.0 ** -20) + 1e-30
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (size + np.abs(want)) + 2.0 ** -134
    err = np.abs(got - want)[:T]
    bad = ~(err <= tol[:T])
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first {np.argwhere(bad)[:4].tolist()}: {got[:T][bad][:4]} want {want[:T][bad][:4]} tol {tol[:T][bad][:4]}"
    if lse is not None:
        gl, wl = _f64(lse), want_lse
        assert (gl[T:] == sentinel).all()
        assert (np.isneginf(gl[:T]) == np.isneginf(wl[:T])).all()
        fin = np.isfinite(wl[:T])
        assert (np.abs(gl[:T][fin] - wl[:T][fin]) <= (e + n + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(np.isfinite(wl), wl, 0.0)))[:T][fin]).all()


def _run_attend(p, *, window=0, behind=False, scale=0.0, with_lse=True, max_new=None, max_len=None, stream=None):
    Q = p["Q"]
    out = torch.full_like(Q, 5.0)
    lse = torch.full(Q.shape[:2], 5.0, device="cuda") if with_lse else None
    table, q_start, lens = (_dev(p[x]) for x in ("table", "q_start", "lens"))
    news = np.diff(p["q_start"])
    paged = ip.make_paged(p["K"], tokens=Q.shape[0], block_table=table, Q=Q, out=out, lse=lse, window=window, behind=behind, scale=scale,
                          max_new=int(news.max()) if max_new is None else max_new, max_len=int(p["lens"].max()) if max_len is None else max_len)
    ws = ip.alloc_paged_workspace(paged)
    ws.fill_(0xFF)                                       # scratch may start at any value
    torch.cuda.synchronize()
    assert ip.ccd_paged_attend(paged, Q, p["K"], p["V"], table, q_start, lens, out, lse, ws, stream=stream) == ip.CCD_OK
    torch.cuda.synchronize()
    return out, lse


# lengths, new tokens, Hq, Hkv, d, page
ATTEND = [
    ([1], [1], 1, 1, 64, 1), ([1], [1], 4, 1, 128, 16), ([2, 0, 5], [1, 0, 5], 4, 2, 128, 16), ([33], [1], 8, 1, 128, 16), ([64, 65, 63, 31, 32], [1] * 5, 32, 8, 128, 16),
    ([129, 1000, 7], [1, 1, 1], 12, 3, 64, 37), ([700], [1], 16, 1, 128, 64), ([700], [1], 34, 2, 64, 64), ([5000], [1], 4, 4, 128, 256), ([3001, 17, 2500], [1, 1, 1], 8, 2, 128, 100),
    ([40], [40], 4, 2, 128, 16), ([130], [129], 2, 2, 64, 16), ([300], [65], 6, 2, 128, 1), ([257, 31], [5, 31], 8, 4, 128, 8), ([90, 200, 1], [3, 64, 1], 9, 3, 64, 37),
    ([513], [257], 3, 1, 128, 4096), ([1000, 600, 5, 0, 90], [130, 1, 5, 0, 33], 8, 2, 128, 64), ([20], [33], 4, 2, 64, 16), ([0, 3], [2, 7], 4, 2, 128, 16), ([600], [200], 16, 2, 64, 37),
    ([2100], [16], 8, 8, 128, 128), ([2100], [17], 10, 2, 64, 128), ([999], [4], 96, 4, 128, 32),
]


@pytest.mark.parametrize("case", range(len(ATTEND)))
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("option", ["plain", "window", "behind", "behind_window", "holes"])
def test_attend(case, dtype, option):
    lens, news, Hq, Hkv, d, page = ATTEND[case]
    print("attend", ATTEND[case], dtype, option, flush=True)
    p = _attend_problem(case, dtype, lens, news, Hq, Hkv, d, page, pad=case % 3, rows_first=case % 2 == 1, holes=0.3 if option == "holes" else 0.0,
                        gain=3.0 if case % 4 == 0 else 1.0)
    # a window of a few tokens, that leaves rows behind the cache empty, or one about as long as the cache
    window = 0 if "window" not in option else (5, max(1, max(lens) - 3), 70)[case % 3]
    behind = option.startswith("behind")
    out, lse = _run_attend(p, window=window, behind=behind, with_lse=case % 5 != 4)
    _check_attend(p, out, lse, dtype, window=window, behind=behind)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("max_new,max_len", [(0, 0), (1, 1), (3, 100000), (1000, 64)])
def test_hints_change_no_result(dtype, max_new, max_len):
    """The largest numbers of new and cached tokens that the host names choose kernels only: too small and too large ones."""
    p = _attend_problem(5, dtype, [800, 1, 333, 2000], [40, 1, 333, 2], 8, 2, 128, 16, pad=2)
    out, lse = _run_attend(p, max_new=max_new, max_len=max_len)
    _check_attend(p, out, lse, dtype)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 60), ("fp32", 1), ("fp32", 60)])
def test_attend_with_a_length_that_the_table_cannot_hold(dtype, new):
    """kv_len is cut at table_width * page, rows at `tokens`: a q_start beyond it writes nothing there."""
    p = _attend_problem(8, dtype, [96], [new], 4, 2, 64, 16, pad=1)
    p["lens"] = np.array([1 << 30], np.int32)
    out, lse = _run_attend(p, max_len=96)
    _check_attend({**p, "lens": np.array([96], np.int32)}, out, lse, dtype)
    p = _attend_problem(8, dtype, [96], [new + 5], 4, 2, 64, 16)
    p["Q"], p["T"] = p["Q"][:new].contiguous(), new
    out, lse = _run_attend(p)
    _check_attend(p, out, lse, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 50])
def test_attend_scale_and_large_logits(dtype, new):
    """Logits of hundreds that grow along the sequence: the running reference rises again and again."""
    p = _attend_problem(9, dtype, [700], [new], 4, 2, 128, 16, gain=4.0)
    ramp = torch.ones(p["K"].shape[0], device="cuda")
    for c in range(44):
        ramp[int(p["table"][0, c])] = 0.1 + 0.2 * c
    p["K"].mul_(ramp[:, None, None, None].to(p["K"].dtype))
    out, lse = _run_attend(p, scale=0.3)
    _check_attend(p, out, lse, dtype, scale=0.3)
    p["K"].mul_(-1.0)
    out, lse = _run_attend(p, scale=0.3)
    _check_attend(p, out, lse, dtype, scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 50])
def test_attend_with_infinite_keys(dtype, new):
    """A key whose logit is -inf has no weight; a row all of whose logits are -inf is an empty one.  NaN in a visible key makes the rows that see it
    NaN, and no others."""
    p = _attend_problem(10, dtype, [200, 150], [new, new], 2, 1, 64, 16)
    p["Q"][..., 0] = p["Q"][..., 0].abs() + 0.5
    K, base = p["K"], p["K"].clone()
    page = int(p["table"][0, 1])
    K[page, :, 4, 0] = float("-inf")                        # position 20 of sequence 0
    out, lse = _run_attend(p)
    q = {**p, "V": p["V"].clone(), "K": base.clone()}
    q["K"][page, :, 4, 0] = -1e30                           # the same to 64 bits: a weight of 0
    q["Q"] = p["Q"]
    want, want_lse, size, _ = O.attend(_f64(p["Q"]), np.nan_to_num(_f64(q["K"])), np.nan_to_num(_f64(p["V"])), p["table"], p["q_start"], p["lens"])
    assert np.isfinite(_f64(out)).all() and np.isfinite(_f64(lse)).all()
    assert (np.abs(_f64(out) - want) <= size * 2.0 ** (-6 if dtype == "bf16" else -14) + 1e-6).all()
    assert (np.abs(_f64(lse) - want_lse) <= 1e-3).all()
    K.copy_(base)
    for c in range(13):                                     # every key of sequence 0
        K[int(p["table"][0, c]), :, :, 0] = float("-inf")
    out, lse = _run_attend(p)
    assert (_f64(out)[:new] == 0.0).all() and np.isneginf(_f64(lse)[:new]).all()
    assert np.isfinite(_f64(out)[new:]).all()
    K.copy_(base)
    K[page, :, 4, 3] = float("nan")
    out, lse = _run_attend(p)
    assert np.isnan(_f64(out)[:new]).all() and np.isnan(_f64(lse)[:new]).all()
    assert np.isfinite(_f64(out)[new:]).all() and np.isfinite(_f64(lse)[new:]).all()


def _same(a, b, dtype):
    """Two orders of summation of the same rows."""
    return (a.double() - b.double()).abs().max().item() <= (2.0 ** -6 if dtype == torch.bfloat16 else 2.0 ** -17)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 70), ("fp32", 1), ("fp32", 70)])
def test_attend_is_repeatable_on_other_streams_and_in_replayed_graphs(dtype, new):
    """The same bits on every run; a captured call replayed with other inputs in its buffers, eager work and other calls on the same
    workspace in between; the workspace of two captured graphs shared."""
    p = _attend_problem(11, dtype, [900, 333], [new, new], 8, 2, 128, 16)
    first, first_lse = _run_attend(p)
    side = torch.cuda.Stream()
    out, lse = _run_attend(p, stream=side)
    assert torch.equal(out, first) and torch.equal(lse, first_lse)
    table, q_start, lens = (_dev(p[x]) for x in ("table", "q_start", "lens"))
    Q2 = p["Q"].flip(0).contiguous()
    outs = [torch.empty_like(p["Q"]) for _ in range(2)]
    lses = [torch.empty(p["Q"].shape[:2], device="cuda") for _ in range(2)]
    paged = ip.make_paged(p["K"], tokens=p["T"], block_table=table, Q=Q2, out=outs[0], lse=lses[0], max_new=new, max_len=900)
    ws = ip.alloc_paged_workspace(paged)
    q_in = Q2.clone()
    graphs = []
    for o, l in zip(outs, lses):
        ip.ccd_paged_attend(paged, q_in, p["K"], p["V"], table, q_start, lens, o, l, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ip.ccd_paged_attend(paged, q_in, p["K"], p["V"], table, q_start, lens, o, l, ws)
        graphs.append(g)
    for step in range(4):
        q_in.copy_(p["Q"] if step % 2 == 0 else Q2)
        for o in outs:
            o.fill_(3.0)
        graphs[step % 2].replay()
        graphs[1 - step % 2].replay()
        torch.cuda.synchronize()
        again, again_lse = _run_attend({**p, "Q": q_in.clone()})
        for o, l in zip(outs, lses):
            assert torch.equal(o, again) and torch.equal(l, again_lse)
        ws.fill_(0xA5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_over_offsets_that_pass_32_bits(dtype):
    """A cache of more than 2^32 elements: pages at both ends of it."""
    d, page, Hkv, esz = 128, 512, 8, 2 if dtype == "bf16" else 4
    n_pages = (1 << 32) // (d * page * Hkv) + 6
    store = torch.empty((n_pages, Hkv, page, d), dtype=DT[dtype], device="cuda")
    ids = [n_pages - 1, 0, n_pages // 2 + 1]
    g = torch.Generator(device="cuda").manual_seed(2)
    for i in ids:
        store[i] = torch.randn((Hkv, page, d), generator=g, device="cuda").to(DT[dtype])
    small = torch.stack([store[i] for i in ids])
    for new in (1, 40):
        Q = torch.randn((new, 16, d), generator=g, device="cuda").to(DT[dtype])
        p = dict(Q=Q, K=store, V=store, table=np.array([ids], np.int32), q_start=np.array([0, new], np.int32), lens=np.array([1100], np.int32), T=new)
        out, lse = _run_attend(p)
        _check_attend({**p, "K": small, "V": small, "table": np.array([[0, 1, 2]])}, out, lse, dtype)
    other = torch.empty_like(store)
    K_new, V_new = (torch.randn((3, Hkv, d), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    slots = torch.tensor([n_pages * page - 1, 5, (n_pages // 2 + 2) * page + 7], dtype=torch.int32, device="cuda")
    paged = ip.make_paged(store, tokens=3, K_new=K_new)
    assert ip.ccd_paged_append(paged, K_new, V_new, slots, store, other) == ip.CCD_OK
    torch.cuda.synchronize()
    for t, s in enumerate(slots.tolist()):
        assert torch.equal(store[s // page, :, s % page], K_new[t]) and torch.equal(other[s // page, :, s % page], V_new[t])


def test_batched_layout_and_pots_strides():
    """Q, out [B, Hq, m, d], lse [B, Hq, m], the cache a memory pot [B, L, Hkv, n_cap, d] of which one layer is read: its pages are the sequences."""
    B, L, Hkv, n_cap, d, Hq, m = 3, 2, 2, 300, 128, 8, 21
    g = torch.Generator(device="cuda").manual_seed(4)
    K, V = (torch.randn((B, L, Hkv, n_cap, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    Q = torch.randn((B, L, Hq, m, d), generator=g, device="cuda").bfloat16()[:, 1]
    out, lse = torch.full((B, Hq, m, d), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq, m), 5.0, device="cuda")
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None]
    q_start = torch.arange(B + 1, dtype=torch.int32, device="cuda") * m
    lens = torch.tensor([300, 211, 21], dtype=torch.int32, device="cuda")
    paged = ip.make_paged(K[:, 1], tokens=B * m, block_table=table, Q=Q, out=out, lse=lse, max_new=m)
    ip.ccd_paged_attend(paged, Q, K[:, 1], V[:, 1], table, q_start, lens, out, lse, ip.alloc_paged_workspace(paged))
    torch.cuda.synchronize()
    p = dict(Q=Q.transpose(1, 2).reshape(B * m, Hq, d), K=K[:, 1], V=V[:, 1], table=table.cpu().numpy(), q_start=q_start.cpu().numpy(), lens=lens.cpu().numpy(), T=B * m)
    _check_attend(p, out.transpose(1, 2).reshape(B * m, Hq, d), lse.transpose(1, 2).reshape(B * m, Hq), "bf16")


# ------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype,layout", [("bf16", 0), ("fp32", 1)])
def test_a_serving_loop(dtype, layout):
    """Plan, embed, append, attend, step after step, with sequences that start, grow by chunks and tokens, and finish: every step's outputs
    against attention over the plain history of each sequence."""
    rng, g = np.random.default_rng(6), torch.Generator(device="cuda").manual_seed(6)
    B, W, page, n_pages, Hq, Hkv, d, cap = 5, 12, 16, 40, 8, 2, 64, 200
    K, V = (torch.full((n_pages, Hkv, page, d), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2))
    table, ring = torch.full((B, W), -1, dtype=torch.int32, device="cuda"), torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    cursor = torch.tensor([7, n_pages, 0, 0], dtype=torch.int32, device="cuda")
    before, after, q_start = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B, B, B + 1))
    slots, pos = (torch.zeros(cap, dtype=torch.int32, device="cuda") for _ in range(2))
    qkv = torch.zeros((cap, Hq + 2 * Hkv, d), dtype=DT[dtype], device="cuda")
    out, lse = torch.full((cap, Hq, d), 5.0, dtype=DT[dtype], device="cuda"), torch.full((cap, Hq), 5.0, device="cuda")
    Q, K_new, V_new = qkv[:, :Hq], qkv[:, Hq: Hq + Hkv], qkv[:, Hq + Hkv:]
    plan = ip.make_plan(table, tokens=cap, page=page, n_pages=n_pages)
    rope_q, rope_k = ip.make_rope(Q, layout=layout, rot=48), ip.make_rope(K_new, layout=layout, rot=48)
    turns = ip.rope_turns(rope_q)
    paged = ip.make_paged(K, tokens=cap, block_table=table, Q=Q, out=out, lse=lse, K_new=K_new, max_new=0, max_len=0)
    ws = ip.alloc_paged_workspace(paged)
    lens, hist = np.zeros(B, int), [[] for _ in range(B)]
    f = O.frequencies(48, 10000.0)
    for step in range(8):
        grow = np.where(rng.random(B) < 0.4, 1, rng.integers(0, 40, B))
        nxt = np.where((rng.random(B) < 0.15) | (lens + grow > W * page - 1), 0, lens + grow)
        before.copy_(torch.from_numpy(lens.astype(np.int32)))
        after.copy_(torch.from_numpy(nxt.astype(np.int32)))
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda").to(DT[dtype]))
        out.fill_(5.0)
        lse.fill_(5.0)
        plain = _f64(qkv)
        assert ip.ccd_paged_plan(plan, before, after, table, table, ring, cursor, cursor, q_start, slots, pos) == ip.CCD_OK
        assert ip.ccd_rope(rope_q, Q, pos, turns, Q) == ip.CCD_OK
        assert ip.ccd_paged_append(paged, K_new, V_new, slots, K, V, rope=rope_k, positions=pos, turns=turns) == ip.CCD_OK
        assert ip.ccd_paged_attend(paged, Q, K, V, table, q_start, after, out, lse, ws) == ip.CCD_OK
        torch.cuda.synchronize()
        assert cursor[2] == 0
        starts, rows_q = [0], _f64(qkv)[:, :Hq]
        for b in range(B):
            m = max(0, nxt[b] - lens[b])
            if nxt[b] < lens[b]:
                hist[b] = []
            i = starts[-1]
            k = O.rope(plain[i: i + m, Hq: Hq + Hkv], range(lens[b], lens[b] + m), f, half=layout == 0)
            k = _f64(torch.from_numpy(k).to(DT[dtype]))
            hist[b] += list(zip(k, plain[i: i + m, Hq + Hkv:]))
            starts.append(i + m)
        assert q_start.tolist() == starts
        pages = max(1, max(len(h) for h in hist))
        Kp, Vp = (np.zeros((B, Hkv, pages, d)) for _ in range(2))
        for b in range(B):
            for t, (k, v) in enumerate(hist[b]):
                Kp[b, :, t], Vp[b, :, t] = k, v
        want_q = O.rope(plain[:starts[-1], :Hq], pos.tolist()[:starts[-1]], f, half=layout == 0)
        assert (np.abs(rows_q[:starts[-1]] - want_q) <= np.abs(want_q) * (2.0 ** -8 if dtype == "bf16" else 0) + 2.0 ** -20 * 8).all()
        want, want_lse, size, _ = O.attend(rows_q[:starts[-1]], Kp, Vp, np.arange(B)[:, None], starts, nxt)
        # keys rounded to the cache's type on both sides, at times to neighbouring values (an fp32 cosine off by 2^-22): a step of a key in a logit
        slack = 2.0 ** -6 if dtype == "bf16" else 2.0 ** -15
        assert (np.abs(_f64(out)[:starts[-1]] - want) <= slack * size + 2.0 ** -8 * np.abs(want) * (dtype == "bf16") + 1e-6).all()
        assert (np.abs(_f64(lse)[:starts[-1]] - want_lse) <= slack).all()
        assert (out[starts[-1]:] == 5.0).all() and (lse[starts[-1]:] == 5.0).all()
        lens = nxt


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new,window", [(3, 0), (8, 0), (70, 0), (200, 0), (40, 25), (1, 30)])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, new, window, bad):
    """Keys and values of a token are NaN or infinite: rows before it, and rows whose window has passed it, are as if it were not there."""
    p = _attend_problem(12, dtype, [330, 90], [new, 1], 4, 2, 64, 16)
    first = 330 - new
    for pos in (first - 40, first + new // 2, first + new - 1) if window else (first + new // 2, first + new - 1):
        page, row = int(p["table"][0, pos // 16]), pos % 16
        p["K"][page, :, row] = float("nan")
        p["V"][page, :, row] = float("nan") if bad == "nan" else float("inf")
    p["V"][int(p["table"][1, 0]), 0, 3, 5] = float(bad)
    out, lse = _run_attend(p, window=window)
    K, V = _f64(p["K"]), _f64(p["V"])
    with np.errstate(invalid="ignore"):
        want, want_lse, _, logit = O.attend(_f64(p["Q"]), K, V, p["table"], p["q_start"], p["lens"], window=window)
    got, got_lse = _f64(out), _f64(lse)
    seen = np.isnan(want_lse)                                       # rows that see a NaN key: NaN throughout
    assert np.isnan(got[seen]).all() and np.isnan(got_lse[seen]).all()
    ok = ~seen
    assert ok[:new // 2].all()
    assert (np.abs(got_lse[ok] - want_lse[ok]) <= 1e-4).all()
    fin = np.isfinite(want) & ok[..., None]
    assert (np.isfinite(got) == np.isfinite(want))[ok].all()
    A = np.nan_to_num(np.abs(V), nan=0.0, posinf=0.0).max()
    assert (np.abs(got[fin] - want[fin]) <= (2.0 ** -6 if dtype == "bf16" else 2.0 ** -16) * A).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [[3, 3, 2], [3, 40, 2], [16, 2, 1]])
def test_what_a_row_does_not_see_in_long_caches(dtype, new):
    """The same where sequences share workgroups and rows are joined from many stretches, among chunks too."""
    lens = [20000, 700, 5000]
    p = _attend_problem(13, dtype, lens, new, 4, 2, 64, 16)
    for b, n in enumerate(lens):
        page, row = int(p["table"][b, (n - 1) // 16]), (n - 1) % 16
        p["K"][page, :, row] = float("nan")
        p["V"][page, :, row] = float("nan")
    out, lse = _run_attend(p)
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.attend(_f64(p["Q"]), _f64(p["K"]), _f64(p["V"]), p["table"], p["q_start"], p["lens"])
    got, got_lse = _f64(out), _f64(lse)
    seen = np.isnan(want_lse)
    last = np.zeros(sum(new), dtype=bool)
    last[np.cumsum(new) - 1] = True
    assert (seen == last[:, None]).all()                            # the last rows alone see the last tokens
    assert np.isnan(got[seen]).all() and np.isnan(got_lse[seen]).all()
    assert (np.abs(got_lse[~seen] - want_lse[~seen]) <= 1e-4).all()
    A = np.nan_to_num(np.abs(_f64(p["V"])), nan=0.0).max()
    assert (np.abs(got[~seen] - want[~seen]) <= (2.0 ** -6 if dtype == "bf16" else 2.0 ** -16) * A).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", [(4, 2), (40, 1)])
@pytest.mark.parametrize("option", ["plain", "window", "behind", "max_new"])
def test_chunks_among_many_sequences(dtype, heads, option):
    """More than 64 sequences of very different numbers of new tokens, none among them: blocks of rows are found from their sums.  max_new: fewer
    expected than there are."""
    rng = np.random.default_rng(14)
    news = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 9, 17, 40], 150)]
    news[70], news[149], news[0] = 300, 70, 129
    lens = [n + int(rng.integers(0, 260)) for n in news]
    lens[3] = 0
    p = _attend_problem(15, dtype, lens, news, heads[0], heads[1], 64, 16, pad=9)
    kw = dict(window=50) if option == "window" else dict(behind=True) if option == "behind" else {}
    out, lse = _run_attend(p, max_new=33 if option == "max_new" else None, **kw)
    _check_attend(p, out, lse, dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decoding_of_many_sequences_cut_evenly(dtype):
    """More sequences than a workgroup has threads, a few of them long, some without a token."""
    rng = np.random.default_rng(16)
    lens = [int(x) for x in rng.integers(0, 60, 700)]
    for b, n in ((0, 2300), (255, 1), (256, 1700), (511, 0), (699, 2500)):
        lens[b] = n
    news = [min(1, n) if b % 7 else 0 for b, n in enumerate(lens)]
    news[699] = news[256] = 1
    p = _attend_problem(17, dtype, lens, news, 4, 2, 64, 16, pad=2)
    out, lse = _run_attend(p)
    _check_attend(p, out, lse, dtype)


def test_rows_at_the_end_of_more_than_one_launch_of_joins():
    """16.8 million rows of padding before a sequence's one new token: its stretches are joined, the padding is left alone."""
    p = _attend_problem(18, "bf16", [1500], [1], 4, 1, 64, 16)
    T = (1 << 22) + 8
    Q = torch.zeros((T, 4, 64), dtype=torch.bfloat16, device="cuda")
    Q[-1] = p["Q"][0]
    out = torch.full_like(Q, 5.0)
    lse = torch.full((T, 4), 5.0, device="cuda")
    table, lens = _dev(p["table"]), _dev(p["lens"])
    q_start = torch.tensor([T - 1, T], dtype=torch.int32, device="cuda")
    paged = ip.make_paged(p["K"], tokens=T, block_table=table, Q=Q, out=out, lse=lse, max_new=1, max_len=1500)
    ws = ip.alloc_paged_workspace(paged)
    assert ws.numel() > T * 4 * 64 * 4                                # several stretches
    assert ip.ccd_paged_attend(paged, Q, p["K"], p["V"], table, q_start, lens, out, lse, ws) == ip.CCD_OK
    torch.cuda.synchronize()
    _check_attend(p, out[-1:].clone(), lse[-1:].clone(), "bf16")
    assert bool((out[:-1] == 5.0).all()) and bool((lse[:-1] == 5.0).all())
    del ws, Q, out, lse
    torch.cuda.empty_cache()


def test_decoding_of_thousands_of_sequences():
    """More units than several rounds of the chip: whole, whatever their lengths."""
    rng = np.random.default_rng(19)
    lens = [int(x) for x in rng.integers(0, 20, 2100)]
    for b, n in ((0, 2300), (1024, 700), (2099, 4100)):
        lens[b] = n
    news = [min(1, n) if b % 5 else 0 for b, n in enumerate(lens)]
    news[2099] = 3
    p = _attend_problem(20, "bf16", lens, news, 4, 2, 64, 16, pad=1)
    out, lse = _run_attend(p)
    _check_attend(p, out, lse, "bf16")


@pytest.mark.parametrize("in_place", [False, True])
def test_plan_counts_that_pass_31_bits_stop_there(in_place):
    top = (1 << 31) - 1
    before, after = np.array([0, 1, 0], np.int32), np.array([top, top, top], np.int32)
    table = np.array([[-1] * 4, [8, -1, -1, -1], [-1] * 4], np.int32)
    ring, cursor = np.arange(9, dtype=np.int32), np.array([0, 8, 0, 0], np.int32)
    t, r, c, q, slots, pos = _run_plan(before, after, table, ring, cursor, page=1, n_pages=9, tokens=9, in_place=in_place)
    np.testing.assert_array_equal(t, [[0, 1, 2, 3], [8, 4, 5, 6], [7, -1, -1, -1]])
    np.testing.assert_array_equal(r, ring)
    np.testing.assert_array_equal(c, [8, 0, top, 0])
    np.testing.assert_array_equal(q, [0, top, top, top])
    np.testing.assert_array_equal(slots, [0, 1, 2, 3] + [-1] * 5)
    np.testing.assert_array_equal(pos, np.arange(9))
