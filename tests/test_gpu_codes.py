"""GPU parity of the cache in 8 bits through the C ABI, against the 64-bit reference.

Tolerances (derived from the arithmetic).
Append without rotation: codes and scales are what the definition says, bit for bit (quotients are rounded exactly).
Append with rotation: the turned key is off by at most r = 2^-21 a (|x_1| + |x_2|) (as in test_gpu_paged) and the number its code stands for by at most
half a step of its scale more: s / 2 (int8); e4m3 2^-4 of the number, or 2^-10 s below 2^-6 s.  The scale is within 2^-20 of |y|max / 127 relative (r against |y|max
>= |x| / sqrt 2 over pairs is at most 2^-21 * 2, a division 2^-24), or the same power of two but for a factor of 2 where |y|max is within 2^-20 of 448 s.
Read: one product, rounded to fp32 (2^-24 relative) and to bf16 (2^-8).
Attention, with k and v the numbers that codes stand for: products of codes with queries are exact in the matrix cores, an fp32 query and weight being three
bf16 parts, so a logit sums at most 3 d exact products and is scaled by a product of two scales: off by e = (3 d + 12) 2^-24 scale sum|q k|.  A weight is off by
2 e relative, 2^x and the value's scale add 2^-22; sums of n weights and 3 n products by 3 n 2^-24: |do| <= A (2 e + 6 n 2^-24 + 2^-20), A = sum w|v| / sum w.
With bf16 queries half a step of the weights and of the result more: 2^-8 A + 2^-8 |o|.  |d lse| <= e + n 2^-24 + 2^-20 + 2^-22 |lse|.
"""
import numpy as np
import pytest
import torch

from oracle import codes_oracle as C
from oracle import paged_oracle as O
from paper_2410_01518_amd import infinipot as ip
from tests.test_gpu_paged import DT, _dev, _f64

pytestmark = pytest.mark.gpu
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy().copy()


def _empty_cache(kind, n_pages, Hkv, page, d, rows, *, rows_first=False, byte=0x55, scale=3.0):
    """Codes and scales K, V, Ks, Vs; every byte and scale given."""
    def codes():
        x = torch.full((n_pages, page, Hkv, d) if rows_first else (n_pages, Hkv, page, d), byte, dtype=torch.uint8, device="cuda").view(CODE[kind])
        return x.transpose(1, 2) if rows_first else x

    def scales():
        x = torch.full((n_pages, Hkv, page // rows), scale, dtype=torch.float32, device="cuda")
        return x
    return codes(), codes(), scales(), scales()


# ------------------------------------------------------------------------------------------------ append

def _runs(rng, T, page, n_pages, rows):
    """Slots of T tokens: runs of neighbouring rows in separate blocks of pages, in order."""
    slots, free = [], list(rng.permutation(n_pages * page // rows))
    while len(slots) < T and free:
        b = int(free.pop()) * rows
        lo = int(rng.integers(0, rows)) if rng.random() < 0.6 else 0
        hi = int(rng.integers(lo, rows)) + 1
        slots += list(range(b + lo, b + hi))
    return np.array(slots[:T], np.int32)


# kind, rows, dtype, T, Hkv, d, page, n_pages, rot, layout
APPEND = [
    ("int8", 1, "bf16", 1, 1, 128, 1, 3, 0, 0), ("int8", 1, "bf16", 70, 8, 128, 16, 9, 128, 0), ("int8", 1, "bf16", 33, 3, 64, 37, 4, 32, 1), ("int8", 1, "fp32", 45, 5, 64, 7, 20, 0, 0),
    ("int8", 1, "fp32", 9, 13, 128, 5, 5, 50, 0), ("int8", 1, "bf16", 1030, 2, 64, 100, 11, 60, 0), ("int8", 1, "fp32", 300, 9, 128, 64, 6, 0, 0), ("int8", 1, "bf16", 20, 3, 128, 3000, 1, 90, 1),
    ("e4m3", 1, "bf16", 1, 1, 64, 1, 3, 0, 0), ("e4m3", 1, "bf16", 70, 8, 128, 16, 9, 128, 1), ("e4m3", 4, "fp32", 61, 3, 64, 100, 3, 0, 0), ("e4m3", 16, "bf16", 150, 8, 128, 64, 6, 0, 0),
    ("e4m3", 16, "bf16", 150, 5, 128, 48, 8, 128, 0), ("e4m3", 64, "fp32", 500, 2, 64, 64, 11, 0, 0), ("e4m3", 32, "bf16", 90, 11, 64, 32, 9, 24, 1), ("e4m3", 2, "bf16", 1, 2, 128, 2, 2, 0, 0),
    ("e4m3", 256, "bf16", 700, 2, 128, 256, 5, 0, 0), ("e4m3", 128, "fp32", 200, 3, 128, 256, 3, 128, 0), ("e4m3", 16, "bf16", 64, 8, 128, 64, 40, 128, 0),
]


@pytest.mark.parametrize("case", range(len(APPEND)))
@pytest.mark.parametrize("order", ["heads first", "rows first"])
def test_append(case, order):
    kind, rows, dtype, T, Hkv, d, page, n_pages, rot, layout = APPEND[case]
    print("append codes", APPEND[case], order, flush=True)
    rng, g = np.random.default_rng(case), torch.Generator(device="cuda").manual_seed(case)
    K, V, Ks, Vs = _empty_cache(kind, n_pages, Hkv, page, d, rows, rows_first=order == "rows first", scale=2.0 ** -9)
    if rows > 1:                                         # blocks of many sizes, some larger than what comes
        for s in (Ks, Vs):
            s.copy_(torch.exp2(torch.randint(-16, 0, s.shape, generator=g, device="cuda").float()))
        for x in (K, V):
            x.view(torch.uint8).copy_(torch.randint(0, 127, x.shape, generator=g, device="cuda").to(torch.uint8))
    slots = rng.permutation(page * n_pages)[:T].astype(np.int32) if rows == 1 else _runs(rng, T, page, n_pages, rows)
    T = len(slots)
    new = (torch.randn((T + 2, 2, Hkv, d), generator=g, device="cuda") * torch.exp(2.0 * torch.randn((T + 2, 2, Hkv, 1), generator=g, device="cuda"))).to(DT[dtype])
    new[T // 2, 0, 0] = 0.0                              # a row of zeros
    K_new, V_new = new[:T, 0], new[:T, 1]
    dead = rng.random(T) < 0.1
    if rows == 1:
        slots[dead] = rng.choice([-1, -9, page * n_pages, 2 ** 31 - 1], dead.sum())
    positions = rng.integers(0, 1 << 20, T).astype(np.int32)
    paged, codes = ip.make_paged(K, tokens=T, dtype=DT[dtype], K_new=K_new), ip.make_codes(K, Ks)
    assert codes.scale_rows == rows
    kw, y = {}, _f64(K_new)
    slack = np.zeros_like(y)
    if rot:
        rope = ip.make_rope(K_new, rot=rot, layout=layout)
        kw = dict(rope=rope, positions=_dev(positions), turns=ip.rope_turns(rope))
        n = rot // 2
        one, two = (np.arange(n), np.arange(n) + n) if layout == ip.CCD_ROPE_HALF else (2 * np.arange(n), 2 * np.arange(n) + 1)
        slack[..., one] = slack[..., two] = 2.0 ** -21 * (np.abs(y[..., one]) + np.abs(y[..., two]))
        y = O.rope(y, positions, O.frequencies(rot, 10000.0), half=layout == ip.CCD_ROPE_HALF)
    want = [(_bytes(x), s.cpu().numpy()) for x, s in ((K, Ks), (V, Vs))]
    assert ip.ccd_paged_append_codes(paged, codes, K_new, V_new, _dev(slots), K, V, Ks, Vs, **kw) == ip.CCD_OK
    torch.cuda.synchronize()
    C.append(_f64(V_new), slots, *want[1], kind, rows)
    np.testing.assert_array_equal(_bytes(V), want[1][0])
    np.testing.assert_array_equal(Vs.cpu().numpy(), want[1][1])
    before = want[0][0].copy()
    C.append(y, slots, *want[0], kind, rows)
    if not rot:
        np.testing.assert_array_equal(_bytes(K), want[0][0])
        np.testing.assert_array_equal(Ks.cpu().numpy(), want[0][1])
        return
    got, gs, ws = _bytes(K), Ks.cpu().numpy().astype(np.float64), want[0][1].astype(np.float64)
    if kind == "int8":
        assert (np.abs(gs - ws) <= 2.0 ** -20 * ws).all()
    else:
        assert np.isin(gs / ws, [0.5, 1.0, 2.0]).all() and (gs != ws).mean() < 0.01
    x = C.decode(got, gs, kind, rows)
    written = np.zeros((n_pages, page), bool)
    for t, s in enumerate(slots):
        if not 0 <= s < page * n_pages:
            continue
        p, r = s // page, s % page
        written[p, r] = True
        sc = gs[p, :, r // rows][:, None]
        half = sc / 2 if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(y[t]), 2.0 ** -10 * sc)
        assert (np.abs(x[p, :, r] - y[t]) <= half * (1 + 2.0 ** -20) + slack[t]).all()
    # what is not written is as it was, or, in a block that grew, as the reference has it (but for a scale that went the other way)
    same = (np.repeat(gs, rows, axis=2) == np.repeat(ws, rows, axis=2)) & ~written[:, None]
    np.testing.assert_array_equal(got[same], want[0][0][same])
    assert (got[~written.repeat(rows if rows == 1 else 1, 1)[:, None].repeat(Hkv, 1)] == before[~written[:, None].repeat(Hkv, 1)]).all() if rows == 1 else True


def test_append_of_ties_and_borders():
    """Quotients that are halves exactly or next to them, largest elements at and beside 448 and 2^-120: fp32 values chosen by hand."""
    d = 64
    rows = []
    for top in (127.0, 1.0, 0.37, 3.0e38, 1e-30, 2.0 ** -119, 1e-44, 0.0):
        s = max(float(np.float32(top / 127.0)), C.LEAST)
        h = np.array([(i + 0.5) * s for i in range(20)], np.float64).astype(np.float32)
        rows.append(np.concatenate([[np.float32(top)], h, np.nextafter(h, np.float32(0)), np.nextafter(h, np.float32(np.inf)), [np.float32(-top), 0.0, -0.0]]))
    for e in (0, 5, -9, 118, -126):
        base = np.ldexp(np.float32(1.75), e)
        for top in (base, np.nextafter(base, np.float32(np.inf)), np.nextafter(base, np.float32(0)), np.ldexp(np.float32(1.0), e)):
            m = np.ldexp(np.arange(1, 61, dtype=np.float32), e - 11)                     # through numbers, halves and what lies below 2^-6
            rows.append(np.concatenate([[top], m, [-top, 0.0, -0.0]]))
    x = np.stack(rows).astype(np.float32)
    x = np.minimum(np.abs(x), np.abs(x[:, :1])) * np.where(np.signbit(x), -1, 1).astype(np.float32)
    T = len(x)
    new = _dev(x.reshape(T, 1, d))
    for kind in ("int8", "e4m3"):
        K, V, Ks, Vs = _empty_cache(kind, T, 1, 1, d, 1)
        paged, codes = ip.make_paged(K, tokens=T, dtype=torch.float32, K_new=new), ip.make_codes(K, Ks)
        assert ip.ccd_paged_append_codes(paged, codes, new, -new, torch.arange(T, dtype=torch.int32, device="cuda"), K, V, Ks, Vs) == ip.CCD_OK
        torch.cuda.synchronize()
        for sign, X, S in ((1, K, Ks), (-1, V, Vs)):
            bits, scales = np.zeros((T, 1, 1, d), np.uint8), np.zeros((T, 1, 1), np.float32)
            C.append(sign * x.reshape(T, 1, d).astype(np.float64), np.arange(T), bits, scales, kind, 1)
            np.testing.assert_array_equal(S.cpu().numpy(), scales)
            np.testing.assert_array_equal(_bytes(X), bits)


def test_append_of_many_quotients_next_to_halves():
    """fp32 rows of which every element is (k + 1/2) times the scale, rounded, or next to that: a half is one only where the quotient is one exactly."""
    rng, T, d = np.random.default_rng(5), 3000, 128
    top = (rng.random((T, 1)) + 1) * 2.0 ** rng.integers(-60, 60, (T, 1))
    top = top.astype(np.float32)
    top[::3] = np.float32(127.0) * np.float32(2.0) ** rng.integers(-30, 30, top[::3].shape).astype(np.float32)       # scales with few bits: halves that are exact
    scale = (top.astype(np.float64) / 127.0).astype(np.float32).astype(np.float64)
    x = ((rng.integers(-126, 126, (T, d)) + 0.5) * scale).astype(np.float32)
    for _ in range(2):
        move = rng.integers(-1, 2, x.shape)
        x = np.where(move < 0, np.nextafter(x, np.float32(-np.inf)), np.where(move > 0, np.nextafter(x, np.float32(np.inf)), x))
    x[:, :1] = top
    new = _dev(x.reshape(T, 1, d))
    K, V, Ks, Vs = _empty_cache("int8", T, 1, 1, d, 1)
    paged, codes = ip.make_paged(K, tokens=T, dtype=torch.float32, K_new=new), ip.make_codes(K, Ks)
    assert ip.ccd_paged_append_codes(paged, codes, new, -new, torch.arange(T, dtype=torch.int32, device="cuda"), K, V, Ks, Vs) == ip.CCD_OK
    torch.cuda.synchronize()
    for sign, X, S in ((1, K, Ks), (-1, V, Vs)):
        bits, scales = np.zeros((T, 1, 1, d), np.uint8), np.zeros((T, 1, 1), np.float32)
        C.append(sign * x.reshape(T, 1, d).astype(np.float64), np.arange(T), bits, scales, "int8", 1)
        np.testing.assert_array_equal(S.cpu().numpy(), scales)
        np.testing.assert_array_equal(_bytes(X), bits)


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 1), ("e4m3", 4)])
@pytest.mark.parametrize("Hkv,d", [(4, 128), (5, 128), (12, 128), (13, 128), (17, 64), (33, 64)])
@pytest.mark.parametrize("rot,layout", [(0, 0), (16, 0), (48, 0), (60, 0), (64, 0), (64, 1), (2, 1)])
def test_append_of_many_heads(kind, rows, Hkv, d, rot, layout):
    """Every head of a token comes out as it does alone: sets of heads, partners in pieces and one by one."""
    T, page = 11, 4
    new = torch.randn((T, 2, Hkv, d), generator=torch.Generator(device="cuda").manual_seed(rot + Hkv), device="cuda").bfloat16()
    positions, slots = torch.arange(T, dtype=torch.int32, device="cuda") * 777, torch.arange(T, dtype=torch.int32, device="cuda")

    def append(x):
        cache = _empty_cache(kind, 3, x.shape[2], page, d, rows, byte=0)
        paged, codes = ip.make_paged(cache[0], tokens=T, dtype=torch.bfloat16, K_new=x[:, 0]), ip.make_codes(cache[0], cache[2])
        kw = {}
        if rot:
            rope = ip.make_rope(x[:, 0], rot=rot, layout=layout)
            kw = dict(rope=rope, positions=positions, turns=ip.rope_turns(rope))
        assert ip.ccd_paged_append_codes(paged, codes, x[:, 0], x[:, 1], slots, *cache, **kw) == ip.CCD_OK
        return cache
    all_of_them = append(new)
    for h in range(Hkv):
        for a, b in zip(all_of_them, append(new[:, :, h: h + 1])):
            assert torch.equal(a.view(torch.uint8)[:, h], b.view(torch.uint8)[:, 0])
    x = C.decode(_bytes(all_of_them[1]), all_of_them[3].cpu().numpy().astype(np.float64), kind, rows).transpose(0, 2, 1, 3).reshape(-1, Hkv, d)[:T]
    step = np.repeat(all_of_them[3].cpu().numpy(), rows, axis=2).transpose(0, 2, 1).reshape(-1, Hkv, 1)[:T].astype(np.float64)
    y = _f64(new[:, 1])
    assert (np.abs(x - y) <= (step / 2 if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * step)) * (1 + 2.0 ** -20)).all()


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 1), ("e4m3", 8)])
def test_append_of_what_is_no_number(kind, rows):
    """Infinities and NaN: int8, the row's scale is NaN; e4m3, the element's code is, and its neighbours and their scale are as without it."""
    d, T = 64, 16
    new = torch.randn((T, 2, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    for t, v in ((3, float("nan")), (5, float("inf")), (9, float("-inf"))):
        new[t, 1, 7] = v
    new[11, 0] = float("nan")
    K, V, Ks, Vs = _empty_cache(kind, 2, 2, 8, d, rows)
    bits, scales = _bytes(K), Ks.cpu().numpy()
    paged, codes = ip.make_paged(K, tokens=T, dtype=torch.bfloat16, K_new=new), ip.make_codes(K, Ks)
    slots = np.arange(T, dtype=np.int32)
    ip.ccd_paged_append_codes(paged, codes, new, new, _dev(slots), K, V, Ks, Vs)
    torch.cuda.synchronize()
    C.append(_f64(new), slots, bits, scales, kind, rows)
    np.testing.assert_array_equal(Ks.cpu().numpy(), scales)
    got = C.decode(_bytes(K), Ks.cpu().numpy(), kind, rows)
    want = C.decode(bits, scales, kind, rows)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(got[~np.isnan(got)], want[~np.isnan(got)])
    assert np.isnan(got).any() and np.isnan(_f64(_read(kind, K, V, Ks, Vs, np.array([[0, 1]]), [0, T], [T], torch.float32)[0])).any()


@pytest.mark.parametrize("rows", [4, 16])
def test_blocks_that_grow_token_by_token(rows):
    """Tokens of growing size, one a call: scales rise, what stands before is rounded again; small ones leave the scale; a first row begins anew."""
    d, page, Hkv = 128, 32, 3
    g = torch.Generator(device="cuda").manual_seed(rows)
    K, V, Ks, Vs = _empty_cache("e4m3", 2, Hkv, page, d, rows, byte=0x7F, scale=float("nan"))
    want = [(_bytes(K), Ks.cpu().numpy()) for _ in range(2)]
    for round_no in range(2):
        for t in range(page):
            x = torch.randn((1, 2, Hkv, d), generator=g, device="cuda") * float(2.0 ** ((t * 5) % 13 - 6)) * (0.01 if round_no else 1.0)
            x = x.bfloat16()
            slots = np.array([page + t], np.int32)
            paged, codes = ip.make_paged(K, tokens=1, dtype=torch.bfloat16, K_new=x[:, 0]), ip.make_codes(K, Ks)
            ip.ccd_paged_append_codes(paged, codes, x[:, 0], x[:, 1], _dev(slots), K, V, Ks, Vs)
            for j in range(2):
                C.append(_f64(x[:, j]), slots, *want[j], "e4m3", rows)
        torch.cuda.synchronize()
        for (bits, scales), X, S in zip(want, (K, V), (Ks, Vs)):
            np.testing.assert_array_equal(S.cpu().numpy(), scales)
            np.testing.assert_array_equal(_bytes(X), bits)


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 8)])
@pytest.mark.parametrize("layout", [0, 1])
def test_append_turned_the_other_way_and_longer(kind, rows, layout):
    """inverse and amplitude of the descriptor; a token without a position is not written."""
    T, Hkv, d, page, rot = 24, 3, 128, 8, 96
    new = torch.randn((T, Hkv, d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    positions = np.arange(T, dtype=np.int32) * 1000
    positions[-1] = -1
    K, V, Ks, Vs = _empty_cache(kind, 3, Hkv, page, d, rows, byte=0)
    rope = ip.make_rope(new, rot=rot, layout=layout, amplitude=1.5, inverse=True)
    paged, codes = ip.make_paged(K, tokens=T, dtype=torch.float32, K_new=new), ip.make_codes(K, Ks)
    ip.ccd_paged_append_codes(paged, codes, new, new, torch.arange(T, dtype=torch.int32, device="cuda"), K, V, Ks, Vs, rope=rope, positions=_dev(positions), turns=ip.rope_turns(rope))
    torch.cuda.synchronize()
    x = _f64(new)
    y = O.rope(x, positions, O.frequencies(rot, 10000.0), half=layout == 0, inverse=True, amplitude=1.5)
    scales = Ks.cpu().numpy().astype(np.float64)
    got = C.decode(_bytes(K), scales, kind, rows).transpose(0, 2, 1, 3).reshape(T, Hkv, d)
    step = np.repeat(scales, rows, axis=2).transpose(0, 2, 1).reshape(T, Hkv, 1)
    half = step / 2 if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * step)
    assert (np.abs(got - y) <= half * (1 + 2.0 ** -20) + 2.0 ** -20 * 1.5 * np.abs(x).max())[:-1].all()
    assert (_bytes(K)[-1, :, -1] == 0).all() and (_bytes(V)[-1, :, -1] == 0).all()


def test_append_of_more_tokens_than_a_workgroup_each():
    """2^24 tokens in blocks of two (rows of the new tensors overlap): the first, last and some in between."""
    T, Hkv, d, page = (1 << 24) + 6, 8, 64, 1 << 12
    n_pages = -(-T // page)
    flat = torch.randn(((T + Hkv) * d,), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda", dtype=torch.float32).bfloat16()
    new = flat.as_strided((T, Hkv, d), (d, d, 1))
    K, V = (torch.zeros((n_pages, Hkv, page, d), dtype=torch.uint8, device="cuda").view(CODE["e4m3"]) for _ in range(2))
    Ks, Vs = (torch.zeros((n_pages, Hkv, page // 2), device="cuda") for _ in range(2))
    paged, codes = ip.make_paged(K, tokens=T, dtype=torch.bfloat16, K_new=new), ip.make_codes(K, Ks)
    assert ip.ccd_paged_append_codes(paged, codes, new, new, torch.arange(T, dtype=torch.int32, device="cuda"), K, V, Ks, Vs) == ip.CCD_OK
    torch.cuda.synchronize()
    for t in (0, 2, 12346, (1 << 23) + 4, T - 2):
        bits, scales = np.zeros((1, Hkv, 2, d), np.uint8), np.zeros((1, Hkv, 1), np.float32)
        C.append(_f64(new[t: t + 2]), np.arange(2), bits, scales, "e4m3", 2)
        p, r = t // page, t % page
        for x, s in ((K, Ks), (V, Vs)):
            np.testing.assert_array_equal(x.view(torch.uint8)[p, :, r: r + 2].cpu().numpy(), bits[0])
            np.testing.assert_array_equal(s[p, :, r // 2].cpu().numpy(), scales[0, :, 0])


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 4)])
def test_append_of_a_batch_with_heads_before_tokens(kind, rows):
    """K_new [B, Hkv, m, d] as a memory pot is given its chunks."""
    B, Hkv, m, d, page = 3, 2, 21, 64, 32
    x = torch.randn((B, Hkv, m, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    slots = np.concatenate([np.arange(m) + b * page + 5 for b in range(B)]).astype(np.int32)
    got = []
    for batched in (True, False):
        K, V, Ks, Vs = _empty_cache(kind, B, Hkv, page, d, rows)
        new = x if batched else x.transpose(1, 2).reshape(B * m, Hkv, d)
        paged = ip.make_paged(K, tokens=B * m, dtype=torch.bfloat16, K_new=new)
        ip.ccd_paged_append_codes(paged, ip.make_codes(K, Ks, K_new=new), new, new, _dev(slots), K, V, Ks, Vs)
        torch.cuda.synchronize()
        got.append([_bytes(K), _bytes(V), Ks.cpu().numpy(), Vs.cpu().numpy()])
    for a, b in zip(*got):
        np.testing.assert_array_equal(a, b)


# ------------------------------------------------------------------------------------------------ read

def _read(kind, K, V, Ks, Vs, table, q_start, lens, dtype, *, pad=0, keys=True, values=True, out=None):
    T = q_start[-1] + pad
    outs = [torch.full((T, K.shape[1], K.shape[3]), 5.0, dtype=dtype, device="cuda") if x else None for x in (keys, values)] if out is None else out
    table, q_start, lens = _dev(np.asarray(table, np.int32)), _dev(np.asarray(q_start, np.int32)), _dev(np.asarray(lens, np.int32))
    paged = ip.make_paged(K, tokens=T, dtype=dtype, block_table=table, out=outs[0] if outs[0] is not None else outs[1])
    assert ip.ccd_paged_read_codes(paged, ip.make_codes(K, Ks), K if keys else None, V if values else None, Ks if keys else None, Vs if values else None, table, q_start, lens,
                                   *outs) == ip.CCD_OK
    torch.cuda.synchronize()
    return outs


def _random_cache(kind, n_pages, Hkv, page, d, rows, seed, *, rows_first=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    K, V, Ks, Vs = _empty_cache(kind, n_pages, Hkv, page, d, rows, rows_first=rows_first)
    for x in (K, V):
        c = torch.randint(0, 256, x.shape, generator=g, device="cuda")
        if kind == "e4m3":
            c = torch.where(c % 128 == 127, 0, c)
            c = torch.where((c & 120) > 72, c - 40, c)             # numbers up to 7.5 or so
        x.view(torch.uint8).copy_(c.to(torch.uint8))
    for s in (Ks, Vs):
        u = torch.rand(s.shape, generator=g, device="cuda")
        s.copy_(torch.exp2(torch.floor(4.0 * u) - 4.0) if kind == "e4m3" else (0.5 + u) / 64.0)
    return K, V, Ks, Vs


def _paged_problem(seed, kind, rows, dtype, lens, news, Hq, Hkv, d, page, *, W=None, pad=0, rows_first=False, holes=0.0, gain=1.0):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    W = W or max(1, max(-(-max(0, n) // page) for n in lens))
    held = [min(W, -(-max(0, n) // page)) for n in lens]
    n_pages = sum(held) + 2
    ids, at = rng.permutation(n_pages).astype(np.int32), 0
    table = np.full((len(lens), W), -1, np.int32)
    for b, h in enumerate(held):
        table[b, :h] = ids[at: at + h]
        at += h
    K, V, Ks, Vs = _random_cache(kind, n_pages, Hkv, page, d, rows, seed, rows_first=rows_first)
    Ks.mul_(gain)
    # what no sequence holds is not a number: pages of nobody, rows behind the last token, scales of blocks without a token
    used = np.zeros((n_pages, page), bool)
    for b, n in enumerate(lens):
        for c in range(held[b]):
            used[table[b, c], :max(0, min(page, n - c * page))] = True
    dead = torch.from_numpy(~used).cuda()[:, None, :, None].expand(K.shape)
    blocks = torch.from_numpy(~used.reshape(n_pages, page // rows, rows).any(2)).cuda()[:, None].expand(Ks.shape)
    for x, s in ((K, Ks), (V, Vs)):
        x.view(torch.uint8).masked_fill_(dead, 0x7F)
        s.masked_fill_(blocks, float("nan"))
    if holes:
        hit = rng.random(table.shape) < holes
        table[hit] = rng.choice([-1, n_pages, -(1 << 31), (1 << 31) - 1], hit.sum())
    T = sum(news)
    Q = torch.randn((T + pad, Hq, d), generator=g, device="cuda").to(DT[dtype])
    q_start = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    return dict(Q=Q, K=K, V=V, Ks=Ks, Vs=Vs, kind=kind, rows=rows, table=table, q_start=q_start, lens=np.array(lens, np.int32), T=T, pad=pad)


def _numbers(p):
    return [C.decode(_bytes(p[x]), p[x + "s"].cpu().numpy(), p["kind"], p["rows"]) for x in "KV"]


KINDS = [("int8", 1, 1), ("e4m3", 1, 1), ("e4m3", 4, 4), ("e4m3", 16, 16)]          # kind, rows, what divides the page


@pytest.mark.parametrize("kind,rows,unit", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,news,Hkv,d,page,pad", [
    ([1], [1], 1, 64, 16, 0), ([40, 0, 7], [40, 0, 3], 3, 128, 16, 2), ([100, 5, 33], [20, 9, 33], 5, 64, 48, 1), ([700], [650], 8, 128, 64, 0), ([3] * 130, [2] * 130, 2, 64, 16, 3),
    ([3, 0, 50], [7, 2, 20], 2, 128, 16, 1),                                       # more rows than tokens: 0 in front
])
def test_read(kind, rows, unit, dtype, lens, news, Hkv, d, page, pad):
    p = _paged_problem(len(lens) + d, kind, rows, dtype, lens, news, Hkv, Hkv, d, page, rows_first=d == 64, holes=0.2 if len(lens) == 130 else 0.0)
    K_out, V_out = _read(kind, p["K"], p["V"], p["Ks"], p["Vs"], p["table"], p["q_start"], lens, DT[dtype], pad=pad)
    for out, x in zip((K_out, V_out), _numbers(p)):
        want = C.read(x, p["table"], p["q_start"], p["lens"])
        got = _f64(out)
        assert (got[p["T"]:] == 5.0).all()
        assert (np.abs(got[: p["T"]] - want) <= np.abs(want) * (2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0))).all()
    only, none = _read(kind, p["K"], p["V"], p["Ks"], p["Vs"], p["table"], p["q_start"], lens, DT[dtype], pad=pad, values=False)
    assert none is None and torch.equal(only, K_out)
    none, only = _read(kind, p["K"], p["V"], p["Ks"], p["Vs"], p["table"], p["q_start"], lens, DT[dtype], pad=pad, keys=False)
    assert none is None and torch.equal(only, V_out)


def test_read_of_whole_pots_with_heads_before_tokens():
    B, Hkv, n, d = 3, 2, 300, 128
    K, V, Ks, Vs = _random_cache("int8", B, Hkv, n, d, 1, 3)
    outs = [torch.zeros((B, Hkv, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = np.arange(B)[:, None]
    paged = ip.make_paged(K, tokens=B * n, dtype=torch.bfloat16, block_table=_dev(table.astype(np.int32)), out=outs[0])
    ip.ccd_paged_read_codes(paged, ip.make_codes(K, Ks), K, V, Ks, Vs, _dev(table.astype(np.int32)), _dev(np.arange(B + 1, dtype=np.int32) * n), _dev(np.full(B, n, np.int32)), *outs)
    torch.cuda.synchronize()
    for out, X, S in zip(outs, (K, V), (Ks, Vs)):
        assert torch.equal(out, (X.float() * S[..., None]).bfloat16())


# ------------------------------------------------------------------------------------------------ attention

def _check_attend(p, out, lse, dtype, *, window=0, behind=False, scale=0.0, sentinel=5.0):
    K, V = (np.nan_to_num(x, nan=0.0) for x in _numbers(p))
    want, want_lse, size, logit = O.attend(_f64(p["Q"]), K, V, p["table"], p["q_start"], p["lens"], window=window, behind=behind, scale=scale)
    got, T, d = _f64(out), p["T"], p["Q"].shape[-1]
    assert (got[T:] == sentinel).all()
    e = (3 * d + 12) * 2.0 ** -24 * logit
    n = np.maximum(1, p["lens"].max()) * 2.0 ** -24
    tol = size * (2 * e[..., None] + 6 * n + 2.0 ** -20) + 1e-30
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
    paged = ip.make_paged(p["K"], tokens=Q.shape[0], dtype=Q.dtype, block_table=table, Q=Q, out=out, lse=lse, window=window, behind=behind, scale=scale,
                          max_new=int(news.max()) if max_new is None else max_new, max_len=int(p["lens"].max()) if max_len is None else max_len)
    codes = ip.make_codes(p["K"], p["Ks"])
    ws = ip.alloc_codes_workspace(paged, codes)
    ws.fill_(0xFF)                                       # scratch may start at any value
    torch.cuda.synchronize()
    assert ip.ccd_paged_attend_codes(paged, codes, Q, p["K"], p["V"], p["Ks"], p["Vs"], table, q_start, lens, out, lse, ws, stream=stream) == ip.CCD_OK
    torch.cuda.synchronize()
    return out, lse


# lengths, new tokens, Hq, Hkv, d, page (a multiple of the kind's block where it is one)
ATTEND = [
    ([1], [1], 1, 1, 64, 16), ([1], [1], 4, 1, 128, 16), ([2, 0, 5], [1, 0, 5], 4, 2, 128, 16), ([33], [1], 8, 1, 128, 16), ([64, 65, 63, 31, 32], [1] * 5, 32, 8, 128, 16),
    ([129, 1000, 7], [1, 1, 1], 12, 3, 64, 48), ([700], [1], 16, 1, 128, 64), ([700], [1], 34, 2, 64, 64), ([5000], [1], 4, 4, 128, 256), ([3001, 17, 2500], [1, 1, 1], 8, 2, 128, 112),
    ([40], [40], 4, 2, 128, 16), ([130], [129], 2, 2, 64, 16), ([257, 31], [5, 31], 8, 4, 128, 32), ([90, 200, 1], [3, 64, 1], 9, 3, 64, 48),
    ([513], [257], 3, 1, 128, 4096), ([1000, 600, 5, 0, 90], [130, 1, 5, 0, 33], 8, 2, 128, 64), ([20], [33], 4, 2, 64, 16), ([0, 3], [2, 7], 4, 2, 128, 16), ([600], [200], 16, 2, 64, 80),
    ([2100], [16], 8, 8, 128, 128), ([2100], [17], 10, 2, 64, 128), ([999], [4], 96, 4, 128, 32),
]


@pytest.mark.parametrize("case", range(len(ATTEND)))
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("option", ["plain", "window", "behind", "behind_window", "holes"])
def test_attend(case, dtype, option):
    lens, news, Hq, Hkv, d, page = ATTEND[case]
    kind, rows, _ = KINDS[(case + len(option)) % 4]
    print("attend codes", ATTEND[case], kind, rows, dtype, option, flush=True)
    p = _paged_problem(case, kind, rows, dtype, lens, news, Hq, Hkv, d, page, pad=case % 3, rows_first=case % 2 == 1, holes=0.3 if option == "holes" else 0.0,
                       gain=3.0 if case % 4 == 0 else 1.0)
    # a window of a few tokens, that leaves rows behind the cache empty, or one about as long as the cache
    window = 0 if "window" not in option else (5, max(1, max(lens) - 3), 70)[case % 3]
    behind = option.startswith("behind")
    out, lse = _run_attend(p, window=window, behind=behind, with_lse=case % 5 != 4)
    _check_attend(p, out, lse, dtype, window=window, behind=behind)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,news,page", [([300, 41], [1, 1], 37), ([600], [200], 37), ([250, 90], [100, 7], 1), ([130], [128], 100)])
def test_attend_over_odd_pages(kind, dtype, lens, news, page):
    p = _paged_problem(31, kind, 4 if kind == "e4m3" and page == 100 else 1, dtype, lens, news, 8, 2, 128, page)
    out, lse = _run_attend(p)
    _check_attend(p, out, lse, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("max_new,max_len", [(0, 0), (1, 1), (3, 100000), (1000, 64)])
def test_hints_change_no_result(dtype, max_new, max_len):
    p = _paged_problem(5, "int8" if max_new % 2 else "e4m3", 1 if max_new % 2 else 16, dtype, [800, 1, 333, 2000], [40, 1, 333, 2], 8, 2, 128, 16, pad=2)
    out, lse = _run_attend(p, max_new=max_new, max_len=max_len)
    _check_attend(p, out, lse, dtype)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 60), ("fp32", 1), ("fp32", 60)])
def test_attend_with_a_length_that_the_table_cannot_hold(dtype, new):
    p = _paged_problem(8, "int8", 1, dtype, [96], [new], 4, 2, 64, 16, pad=1)
    p["lens"] = np.array([1 << 30], np.int32)
    out, lse = _run_attend(p, max_len=96)
    _check_attend({**p, "lens": np.array([96], np.int32)}, out, lse, dtype)
    p = _paged_problem(8, "e4m3", 4, dtype, [96], [new + 5], 4, 2, 64, 16)
    p["Q"], p["T"] = p["Q"][:new].contiguous(), new
    out, lse = _run_attend(p)
    _check_attend(p, out, lse, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("new", [1, 50])
def test_attend_scale_and_large_logits(kind, dtype, new):
    """Logits of hundreds that grow along the sequence: the running reference rises again and again."""
    p = _paged_problem(9, kind, 1, dtype, [700], [new], 4, 2, 128, 16, gain=4.0)
    for c in range(44):
        p["Ks"][int(p["table"][0, c])] *= 0.1 + 0.2 * c if kind == "int8" else 2.0 ** (c // 8 - 3)
    for _ in range(2):
        out, lse = _run_attend(p, scale=0.3)
        _check_attend(p, out, lse, dtype, scale=0.3)
        p["Q"].neg_()


def _spoil(p, b, pos, kind, what):
    """Token `pos` of sequence b is no number: its scales (int8), or codes (e4m3)."""
    page, row = int(p["table"][b, pos // p["K"].shape[2]]), pos % p["K"].shape[2]
    for x in what:
        if kind == "int8":
            p[x + "s"][page, :, row] = float("nan")
        else:
            p[x].view(torch.uint8)[page, :, row] = 0x7F


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 1), ("e4m3", 16)])
@pytest.mark.parametrize("new,window", [(3, 0), (8, 0), (70, 0), (200, 0), (40, 25), (1, 30)])
@pytest.mark.parametrize("what", ["KV", "V"])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, kind, rows, new, window, what):
    """Keys and values of a token are no numbers: rows before it, and rows whose window has passed it, are as if it were not there."""
    p = _paged_problem(12, kind, rows, dtype, [330, 90], [new, 1], 4, 2, 64, 16)
    first = 330 - new
    for pos in (first - 40, first + new // 2, first + new - 1) if window else (first + new // 2, first + new - 1):
        _spoil(p, 0, pos, kind, what)
    out, lse = _run_attend(p, window=window)
    K, V = _numbers(p)
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.attend(_f64(p["Q"]), K, V, p["table"], p["q_start"], p["lens"], window=window)
    got, got_lse = _f64(out), _f64(lse)
    np.testing.assert_array_equal(np.isnan(got_lse), np.isnan(want_lse))
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want_lse)
    assert ok[:new // 2].all()
    assert (np.abs(got_lse[ok] - want_lse[ok]) <= 1e-4).all()
    fin = np.isfinite(want)
    assert (np.abs(got[fin] - want[fin]) <= (2.0 ** -6 if dtype == "bf16" else 2.0 ** -15) * np.nanmax(np.abs(V))).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("new", [[3, 3, 2], [3, 40, 2], [16, 2, 1]])
def test_what_a_row_does_not_see_in_long_caches(dtype, kind, new):
    """The same where sequences share workgroups and rows are joined from many stretches, among chunks too."""
    lens = [20000, 700, 5000]
    p = _paged_problem(13, kind, 1, dtype, lens, new, 4, 2, 64, 16)
    for b, n in enumerate(lens):
        _spoil(p, b, n - 1, kind, "KV")
    out, lse = _run_attend(p)
    K, V = _numbers(p)
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.attend(_f64(p["Q"]), K, V, p["table"], p["q_start"], p["lens"])
    got, got_lse = _f64(out), _f64(lse)
    seen = np.isnan(want_lse)
    last = np.zeros(sum(new), dtype=bool)
    last[np.cumsum(new) - 1] = True
    assert (seen == last[:, None]).all()                            # the last rows alone see the last tokens
    assert np.isnan(got[seen]).all() and np.isnan(got_lse[seen]).all()
    assert (np.abs(got_lse[~seen] - want_lse[~seen]) <= 1e-4).all()
    assert (np.abs(got[~seen] - want[~seen]) <= (2.0 ** -6 if dtype == "bf16" else 2.0 ** -15) * np.nanmax(np.abs(V))).all()


def _same(a, b):
    return torch.equal(a, b)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 70), ("fp32", 1), ("fp32", 70)])
def test_attend_is_repeatable_on_other_streams_and_in_replayed_graphs(dtype, new):
    """The same bits on every run; a captured call replayed with other inputs in its buffers, eager work and other calls on the same
    workspace in between; the workspace of two captured graphs shared."""
    p = _paged_problem(11, "int8", 1, dtype, [900, 333], [new, new], 8, 2, 128, 16)
    first, first_lse = _run_attend(p)
    side = torch.cuda.Stream()
    out, lse = _run_attend(p, stream=side)
    assert torch.equal(out, first) and torch.equal(lse, first_lse)
    table, q_start, lens = (_dev(p[x]) for x in ("table", "q_start", "lens"))
    Q2 = p["Q"].flip(0).contiguous()
    outs = [torch.empty_like(p["Q"]) for _ in range(2)]
    lses = [torch.empty(p["Q"].shape[:2], device="cuda") for _ in range(2)]
    paged, codes = ip.make_paged(p["K"], tokens=p["T"], dtype=DT[dtype], block_table=table, Q=Q2, out=outs[0], lse=lses[0], max_new=new, max_len=900), ip.make_codes(p["K"], p["Ks"])
    ws = ip.alloc_codes_workspace(paged, codes)
    q_in = Q2.clone()
    graphs = []
    for o, l in zip(outs, lses):
        def call():
            ip.ccd_paged_attend_codes(paged, codes, q_in, p["K"], p["V"], p["Ks"], p["Vs"], table, q_start, lens, o, l, ws)
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
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


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_offsets_that_pass_32_bits(kind):
    """A cache of more than 2^32 bytes: pages at both ends of it; write, read back, attend."""
    d, page, Hkv = 128, 512, 8
    n_pages = (1 << 32) // (d * page * Hkv) + 6
    K = torch.empty((n_pages, Hkv, page, d), dtype=torch.uint8, device="cuda").view(CODE[kind])
    V, Ks = torch.empty_like(K), torch.ones((n_pages, Hkv, page), device="cuda")
    Vs = torch.ones_like(Ks)
    ids = [n_pages - 1, 0, n_pages // 2 + 1]
    T = 1100
    g = torch.Generator(device="cuda").manual_seed(2)
    new = torch.randn((T, 2, Hkv, d), generator=g, device="cuda").bfloat16()
    t = np.arange(T)
    slots = (np.array(ids)[t // page] * page + t % page).astype(np.int32)
    paged = ip.make_paged(K, tokens=T, dtype=torch.bfloat16, K_new=new[:, 0])
    assert ip.ccd_paged_append_codes(paged, ip.make_codes(K, Ks), new[:, 0], new[:, 1], _dev(slots), K, V, Ks, Vs) == ip.CCD_OK
    torch.cuda.synchronize()
    small = {n: torch.stack([x.view(torch.uint8)[i] for i in ids]).view(CODE[kind]) for n, x in (("K", K), ("V", V))}
    small.update({n: torch.stack([x[i] for i in ids]) for n, x in (("Ks", Ks), ("Vs", Vs))})
    for x, j in (("K", 0), ("V", 1)):
        bits, scales = np.zeros((3, Hkv, page, d), np.uint8), np.ones((3, Hkv, page), np.float32)
        C.append(_f64(new[:, j]), t, bits, scales, kind, 1)
        rows = _bytes(small[x]).transpose(0, 2, 1, 3).reshape(-1, Hkv, d)[:T]
        np.testing.assert_array_equal(rows, bits.transpose(0, 2, 1, 3).reshape(-1, Hkv, d)[:T])
    table = np.array([ids], np.int32)
    out = _read(kind, K, V, Ks, Vs, table, [0, T], [T], torch.bfloat16)
    want = _read(kind, *(small[x] for x in ("K", "V", "Ks", "Vs")), np.array([[0, 1, 2]]), [0, T], [T], torch.bfloat16)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    for n_new in (1, 40):
        Q = torch.randn((n_new, 16, d), generator=g, device="cuda").bfloat16()
        p = dict(Q=Q, K=K, V=V, Ks=Ks, Vs=Vs, kind=kind, rows=1, table=table, q_start=np.array([0, n_new], np.int32), lens=np.array([T], np.int32), T=n_new)
        o, lse = _run_attend(p)
        _check_attend({**p, **small, "table": np.array([[0, 1, 2]])}, o, lse, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", [(4, 2), (40, 1)])
@pytest.mark.parametrize("option", ["plain", "window", "behind", "max_new"])
def test_chunks_among_many_sequences(dtype, heads, option):
    """More than 64 sequences of very different numbers of new tokens, none among them.  max_new: fewer expected than there are."""
    rng = np.random.default_rng(14)
    news = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 9, 17, 40], 150)]
    news[70], news[149], news[0] = 300, 70, 129
    lens = [n + int(rng.integers(0, 260)) for n in news]
    lens[3] = 0
    p = _paged_problem(15, *(("int8", 1) if heads[0] == 4 else ("e4m3", 16)), dtype, lens, news, heads[0], heads[1], 64, 16, pad=9)
    kw = dict(window=50) if option == "window" else dict(behind=True) if option == "behind" else {}
    out, lse = _run_attend(p, max_new=33 if option == "max_new" else None, **kw)
    _check_attend(p, out, lse, dtype, **kw)


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 16)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decoding_of_many_sequences_cut_evenly(dtype, kind, rows):
    rng = np.random.default_rng(16)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(3000), 90))]
    p = _paged_problem(16, kind, rows, dtype, lens, [1] * 90, 8, 2, 128, 64)
    out, lse = _run_attend(p)
    _check_attend(p, out, lse, dtype)


# ------------------------------------------------------------------------------------------------ compaction

@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("pots,Hkv,page,d,k", [(1, 1, 1, 64, 1), (2, 3, 37, 64, 11), (3, 2, 300, 128, 299), (1, 8, 1000, 128, 500), (5, 1, 64, 128, 64), (2, 2, 5000, 64, 1), (2, 2, 4096, 128, 2048)])
@pytest.mark.parametrize("novelty", [False, True])
def test_compact(kind, pots, Hkv, page, d, k, novelty):
    rng = np.random.default_rng(page)
    K, V, Ks, Vs = _random_cache(kind, pots, Hkv, page, d, 1, page, rows_first=page == 300)
    nov = torch.rand((pots, Hkv, page), device="cuda") if novelty else None
    keep = np.stack([np.sort(rng.permutation(page)[:k]) for _ in range(pots * Hkv)]).reshape(pots, Hkv, k).astype(np.int32)
    want = [C.compact(_bytes(x), keep) for x in (K, V)] + [C.compact(x.cpu().numpy(), keep) for x in ((Ks, Vs, nov) if novelty else (Ks, Vs))]
    paged = ip.make_paged(K, tokens=0, dtype=torch.bfloat16)
    assert ip.ccd_paged_compact_codes(paged, ip.make_codes(K, Ks), K, V, Ks, Vs, _dev(keep), novelty=nov) == ip.CCD_OK
    torch.cuda.synchronize()
    got = [_bytes(K), _bytes(V), Ks.cpu().numpy(), Vs.cpu().numpy()] + ([nov.cpu().numpy()] if novelty else [])
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g, w)


@pytest.mark.parametrize("pots,Hkv,page,d,k", [(32, 8, 300, 128, 131), (129, 1, 1000, 128, 513), (40, 4, 128, 128, 128), (150, 1, 700, 64, 257)])
def test_compact_of_many_pots(pots, Hkv, page, d, k):
    """Whole rows by one workgroup, scales with strides of their own, kept rows side by side and far apart."""
    rng = np.random.default_rng(k)
    K, V, Ks, Vs = _random_cache("int8", pots, Hkv, page, d, 1, k)
    wide = torch.zeros((2, pots, 3, Hkv, page + 5), device="cuda")
    for w, s in zip(wide, (Ks, Vs)):
        w[:, 1, :, :page] = s
    Ks, Vs = (w[:, 1, :, :page] for w in wide)
    nov = torch.rand((pots, Hkv, page), device="cuda")
    keep = np.stack([np.sort(rng.permutation(page)[:k]) if u % 3 else np.arange(page - k, page) for u in range(pots * Hkv)]).reshape(pots, Hkv, k).astype(np.int32)
    want = [C.compact(_bytes(x), keep) for x in (K, V)] + [C.compact(x.cpu().numpy(), keep) for x in (Ks, Vs, nov)]
    paged = ip.make_paged(K, tokens=0, dtype=torch.bfloat16)
    assert ip.ccd_paged_compact_codes(paged, ip.make_codes(K, Ks), K, V, Ks, Vs, _dev(keep), novelty=nov) == ip.CCD_OK
    torch.cuda.synchronize()
    for g, w in zip([_bytes(K), _bytes(V), Ks.cpu().numpy(), Vs.cpu().numpy(), nov.cpu().numpy()], want):
        np.testing.assert_array_equal(g, w)
    assert (wide[:, :, 0] == 0).all() and (wide[:, :, 2] == 0).all() and (wide[..., page:] == 0).all()


def test_compact_leaves_rows_whose_entry_is_outside_the_page():
    K, V, Ks, Vs = _random_cache("int8", 1, 1, 64, 64, 1, 1)
    keep = np.array([[[0, 5, 64, 9, -1, 2 ** 31 - 1, 40]]], np.int32)
    want = _bytes(K)
    for j, i in enumerate(keep[0, 0]):
        if 0 <= i < 64:
            want[0, 0, j] = _bytes(K)[0, 0, i]
    ip.ccd_paged_compact_codes(ip.make_paged(K, tokens=0, dtype=torch.bfloat16), ip.make_codes(K, Ks), K, V, Ks, Vs, _dev(keep))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(_bytes(K), want)


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 1), ("e4m3", 8)])
def test_a_captured_step_on_another_stream(kind, rows):
    """Append, attention, reading back and (where rows have their own scales) compaction in one graph, replayed with other tokens at other places, eager work and synchronisations
    in between: the same bits as the calls by themselves."""
    B, Hq, Hkv, d, page, m = 3, 8, 2, 64, 32, 5
    g0 = torch.Generator(device="cuda").manual_seed(17)
    rand = lambda *shape: torch.randn(shape, generator=g0, device="cuda").bfloat16()           # noqa: E731
    table = torch.tensor([[4, 1], [0, 5], [2, 3]], dtype=torch.int32, device="cuda")
    q_start = torch.arange(B + 1, dtype=torch.int32, device="cuda") * m
    keep = torch.sort(torch.rand((6, Hkv, page), generator=g0, device="cuda").argsort(-1)[..., :16])[0].int().contiguous()
    buffers = dict(new=rand(B * m, 2, Hkv, d), Q=rand(B * m, Hq, d), slots=torch.zeros(B * m, dtype=torch.int32, device="cuda"),
                   positions=torch.zeros(B * m, dtype=torch.int32, device="cuda"), lens=torch.zeros(B, dtype=torch.int32, device="cuda"))

    def state():
        return _empty_cache(kind, 6, Hkv, page, d, rows, byte=0x11, scale=2.0 ** -6), torch.empty((B * m, Hq, d), dtype=torch.bfloat16, device="cuda"), \
            torch.empty((B * m, Hq), device="cuda"), torch.empty((B * m, Hkv, d), dtype=torch.bfloat16, device="cuda"), torch.ones((6, Hkv, page), device="cuda")

    def step(b, s, ws, turns, rope):
        cache, out, lse, back, novelty = s
        K_new, V_new = b["new"][:, 0], b["new"][:, 1]
        codes = ip.make_codes(cache[0], cache[2])
        ip.ccd_paged_append_codes(ip.make_paged(cache[0], tokens=B * m, dtype=torch.bfloat16, K_new=K_new), codes, K_new, V_new, b["slots"], *cache, rope=rope,
                                  positions=b["positions"], turns=turns)
        paged = ip.make_paged(cache[0], tokens=B * m, dtype=torch.bfloat16, block_table=table, Q=b["Q"], out=out, lse=lse)
        ws = ip.alloc_codes_workspace(paged, codes) if ws is None else ws
        ip.ccd_paged_attend_codes(paged, codes, b["Q"], *cache, table, q_start, b["lens"], out, lse, ws)
        ip.ccd_paged_read_codes(ip.make_paged(cache[0], tokens=B * m, dtype=torch.bfloat16, block_table=table, out=back), codes, *cache, table, q_start, b["lens"], back, None)
        if rows == 1:
            ip.ccd_paged_compact_codes(ip.make_paged(cache[0], tokens=0, dtype=torch.bfloat16), codes, *cache, keep, novelty=novelty)
        return ws

    def fill(round_no):
        held = [3 + 5 * round_no, 20 + round_no, 31 + 2 * round_no]
        tokens = [(b, t) for b in range(B) for t in range(held[b], held[b] + m)]
        places = table.cpu().numpy()
        buffers["slots"].copy_(torch.tensor([int(places[b, t // page]) * page + t % page for b, t in tokens], dtype=torch.int32))
        buffers["positions"].copy_(torch.tensor([t for _, t in tokens], dtype=torch.int32))
        buffers["lens"].copy_(torch.tensor([n + m for n in held], dtype=torch.int32))
        buffers["new"].copy_(rand(B * m, 2, Hkv, d) * 2.0 ** round_no)
        buffers["Q"].copy_(rand(B * m, Hq, d))

    rope = ip.make_rope(buffers["new"][:, 0], rot=32)
    turns = ip.rope_turns(rope)
    fill(0)
    captured, eager = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = step(buffers, state(), None, turns, rope)                   # (once outside: allocations and lazy loading)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(buffers, captured, ws, turns, rope)
    for round_no in range(4):
        fill(round_no)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        side.synchronize()
        step(buffers, eager, None, turns, rope)
        torch.cuda.synchronize()
        flat = lambda s: [x.view(torch.uint8) for x in (*s[0], *s[1:])]  # noqa: E731
        for a, b in zip(flat(captured), flat(eager)):
            assert torch.equal(a, b)
