"""The cache in 8 bits at its edges: elements that are no numbers beside ones that are not turned, blocks quantised elsewhere, weights of 0 in fp32, stretches of more than
64 tiles, odd pages of long caches.  Tolerances as in test_gpu_codes; codes and scales bit for bit wherever nothing is rotated.
"""
import numpy as np
import pytest
import torch

from oracle import codes_oracle as C
from oracle import paged_oracle as O
from paper_2410_01518_amd import infinipot as ip
from tests.test_gpu_codes import _bytes, _check_attend, _empty_cache, _numbers, _paged_problem, _run_attend
from tests.test_gpu_paged import DT, _dev, _f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 1), ("e4m3", 8)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", [ip.CCD_ROPE_HALF, ip.CCD_ROPE_PAIRS])
@pytest.mark.parametrize("d,rot", [(64, 32), (128, 12), (128, 96)])
def test_append_beside_what_is_no_number(kind, rows, dtype, layout, d, rot):
    """Infinities and NaN among the elements that are not turned are the codes of those elements alone; what is not turned keeps its sign, zeros too.  The largest elements stand there,
    so scales and codes of the elements that are not turned are known bit for bit."""
    T, Hkv, page = 16, 3, 8
    new = torch.randn((T, Hkv, d), generator=torch.Generator(device="cuda").manual_seed(rot), device="cuda").to(DT[dtype])
    new[..., rot:] *= 16.0
    new[..., rot + 4] = 50.0
    new[..., rot + 6], new[..., rot + 7] = -0.0, 1.0
    new[3, 0, rot], new[3, 1, rot + 1] = float("inf"), float("-inf")
    new[5, 2, d - 1], new[6, 2, d - 2] = float("nan"), float("inf")
    K, V, Ks, Vs = _empty_cache(kind, 2, Hkv, page, d, rows)
    bits, scales = _bytes(K), Ks.cpu().numpy()
    rope = ip.make_rope(new, rot=rot, layout=layout)
    slots, positions = np.arange(T, dtype=np.int32), np.arange(T, dtype=np.int32) * 1001
    paged, codes = ip.make_paged(K, tokens=T, dtype=DT[dtype], K_new=new), ip.make_codes(K, Ks)
    ip.ccd_paged_append_codes(paged, codes, new, new, _dev(slots), K, V, Ks, Vs, rope=rope, positions=_dev(positions), turns=ip.rope_turns(rope))
    torch.cuda.synchronize()
    C.append(O.rope(_f64(new), positions, O.frequencies(rot, 10000.0), half=layout == ip.CCD_ROPE_HALF), slots, bits, scales, kind, rows)
    np.testing.assert_array_equal(Ks.cpu().numpy(), scales)
    got = _bytes(K)
    known = np.broadcast_to(np.isfinite(np.repeat(scales, rows, axis=2))[..., None], got.shape)[..., rot:]      # (int8: rows that are no numbers have no codes to speak of)
    np.testing.assert_array_equal(got[..., rot:][known], bits[..., rot:][known])
    assert known.sum() < known.size if kind == "int8" else (bits[..., rot:] == 0x7F).sum() == 4
    np.testing.assert_array_equal(np.isnan(C.decode(got, scales, kind, rows)), np.isnan(C.decode(bits, scales, kind, rows)))


@pytest.mark.parametrize("rows,first", [(8, 3), (32, 17)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_into_blocks_quantised_elsewhere(rows, first, dtype):
    """A block's own scale may be any number: the rows before the new ones are rounded again from what they read as, to a scale that is a power of two."""
    d, page, Hkv = 64, 32, 1
    held = np.array([3.0, 0.75, 1.0 / 3.0, 5e-7, 1e-40, 0.0, 2.0 ** 120, 1.5 * 2.0 ** 120, 2.0 ** 127, 3.4e38, np.inf, np.nan, 2.0 ** -9, 1.0 + 2.0 ** -23, 2.0 - 2.0 ** -23], np.float32)
    n = len(held)
    g = torch.Generator(device="cuda").manual_seed(rows)
    K, V, Ks, Vs = _empty_cache("e4m3", n, Hkv, page, d, rows)
    for x in (K, V):
        x.view(torch.uint8).copy_(torch.randint(0, 256, x.shape, generator=g, device="cuda").to(torch.uint8))
    for s in (Ks, Vs):
        s.copy_(_dev(held)[:, None, None].expand(s.shape))
    new = (torch.randn((2 * n, 2, Hkv, d), generator=g, device="cuda") * 0.01).to(DT[dtype])
    slots = np.concatenate([[p * page + first, p * page + first + 1] for p in range(n)]).astype(np.int32)
    want = [(_bytes(x), s.cpu().numpy()) for x, s in ((K, Ks), (V, Vs))]
    paged, codes = ip.make_paged(K, tokens=2 * n, dtype=DT[dtype], K_new=new[:, 0]), ip.make_codes(K, Ks)
    assert ip.ccd_paged_append_codes(paged, codes, new[:, 0], new[:, 1], _dev(slots), K, V, Ks, Vs) == ip.CCD_OK
    torch.cuda.synchronize()
    for j, (x, s) in enumerate(((K, Ks), (V, Vs))):
        C.append(_f64(new[:, j]), slots, *want[j], "e4m3", rows)
        np.testing.assert_array_equal(s.cpu().numpy(), want[j][1])
        got, bits = (C.E4M3[b] for b in (_bytes(x), want[j][0]))           # (a code that is no number has two signs)
        np.testing.assert_array_equal(got, bits)
        fin = np.isfinite(bits)
        np.testing.assert_array_equal(_bytes(x)[fin], want[j][0][fin])


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pos", [10, 40, 66])
@pytest.mark.parametrize("news", [[1], [3], [40], [1, 40], [2, 1, 1]])
@pytest.mark.parametrize("length,max_len", [(70, None), (70 + 32 * 40, None), (70 + 32 * 40, 64)])
def test_a_value_that_is_no_number_and_is_seen(kind, dtype, pos, news, length, max_len):
    """A row that sees such a value has it, whatever is left of its weight: here 0 in fp32, in tiles that are seen whole and in others, however the call is cut."""
    lens = [length] * len(news)
    p = _paged_problem(21, kind, 1, dtype, lens, news, 4, 2, 64, 16)
    at = length - 70 + pos
    p["Q"].copy_(p["Q"].abs() + 1.0)
    for b in range(len(news)):
        page, row = int(p["table"][b, at // 16]), at % 16
        if kind == "int8":                                                     # the key: a logit far below all others, about -127 * 64 * 1.8 * 8 / 8
            p["K"].view(torch.uint8)[page, :, row] = 0x81
            p["Ks"][page, :, row] = 8.0
            p["Vs"][page, :, row] = float("nan")
        else:
            p["K"].view(torch.uint8)[page, :, row] = 0xFE
            p["Ks"][page, :, row] = 8.0
            p["V"].view(torch.uint8)[page, 0, row, 5] = 0x7F
            p["V"].view(torch.uint8)[page, 1, row] = 0x7F
    out, lse = _run_attend(p, max_len=max_len)
    K, V = _numbers(p)
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.attend(_f64(p["Q"]), K, V, p["table"], p["q_start"], p["lens"])
    np.testing.assert_array_equal(np.isnan(_f64(out)), np.isnan(want))
    assert np.isnan(want).any() and np.isfinite(want_lse).all()
    for b in range(len(news)):
        K[int(p["table"][b, at // 16]), :, at % 16] = 0.0                      # (the sizes of the logits that have weights)
    logit = O.attend(_f64(p["Q"]), K, np.zeros_like(V), p["table"], p["q_start"], p["lens"])[3]
    assert (np.abs(_f64(lse) - want_lse) <= (3 * 64 + 12) * 2.0 ** -24 * logit + length * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 16)])
@pytest.mark.parametrize("dtype,length,new,page,d,max_len", [
    ("bf16", 9200, 9, 16, 128, 64), ("bf16", 9200, 17, 48, 64, 64), ("bf16", 9200, 10, 4096, 128, 64), ("fp32", 9200, 9, 16, 64, 64),      # a stretch of 144 tiles
    ("bf16", 24000, 9, 64, 64, 1100), ("bf16", 9200, 9, 16, 128, None),                # stretches of 75 tiles or more, without the sums of rounded weights; many short ones
])
def test_stretches_of_more_than_64_tiles(kind, rows, dtype, length, new, page, d, max_len):
    """Shuffled pages, by few stretches (the hint says so): pages are looked up for 64 tiles at once."""
    p = _paged_problem(23, kind, rows, dtype, [length], [new], 4, 1, d, page)
    out, lse = _run_attend(p, max_len=max_len)
    _check_attend(p, out, lse, dtype)


@pytest.mark.parametrize("kind,rows", [("int8", 1), ("e4m3", 1), ("e4m3", 4)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,news,page", [([1800, 1300], [9, 17], 37), ([2500], [17], 100), ([4300], [9], 100)])
def test_chunks_over_odd_pages_of_long_caches(kind, rows, d, lens, news, page):
    p = _paged_problem(29, kind, rows if page % rows == 0 else 1, "bf16", lens, news, 8, 2, d, page)
    out, lse = _run_attend(p)
    _check_attend(p, out, lse, "bf16")
