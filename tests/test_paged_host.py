"""The paged cache's entry points on the host: descriptors, frequencies, refusals (all decided before any launch), and the
reference's own pins."""
import ctypes
import math
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2410_01518_amd import infinipot as ip

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000  # a fake, aligned, non-null device address: never dereferenced because every case below fails on the host
P2 = 0x100000


def test_struct_layouts_match_the_header():
    fields = {"ccd_paged_t": ("scale", "page_stride", "new_stride_t", "q_stride_b", "o_stride_b", "lse_stride_h"),
              "ccd_rope_t": ("amplitude", "x_stride_t", "scaling", "context", "base", "high")}
    lines = "".join(f'printf("%zu {" ".join(["%zu"] * len(f))}\\n", sizeof({s}), {", ".join(f"offsetof({s}, {x})" for x in f)});' for s, f in fields.items())
    prog = "#include <stdio.h>\n#include <stddef.h>\n#include \"infinipot.h\"\nint main(void){" + lines + \
        'printf("%d %d %d %d %d %d\\n", CCD_ROPE_HALF, CCD_ROPE_PAIRS, CCD_ROPE_PLAIN, CCD_ROPE_LINEAR, CCD_ROPE_NTK, CCD_ROPE_PARTS); return 0; }'
    with tempfile.TemporaryDirectory() as td:
        open(os.path.join(td, "t.c"), "w").write(prog)
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), os.path.join(td, "t.c"), "-o", os.path.join(td, "t")], check=True)
        out = subprocess.run([os.path.join(td, "t")], capture_output=True, text=True, check=True).stdout.splitlines()
    for line, (name, f) in zip(out, fields.items()):
        S = getattr(ip, name)
        assert [int(v) for v in line.split()] == [ctypes.sizeof(S)] + [getattr(S, x).offset for x in f]
    assert [int(v) for v in out[2].split()] == [ip.CCD_ROPE_HALF, ip.CCD_ROPE_PAIRS, ip.CCD_ROPE_PLAIN, ip.CCD_ROPE_LINEAR, ip.CCD_ROPE_NTK, ip.CCD_ROPE_PARTS]


def _paged(**kw):
    base = dict(B=2, tokens=6, Hq=8, Hkv=2, d=128, dtype=ip.CCD_BF16, page=16, n_pages=10, table_width=4, page_stride=2 * 16 * 128, head_stride=16 * 128,
                row_stride=128, new_stride_t=256, new_stride_h=128, q_stride_t=1024, q_stride_h=128, o_stride_t=1024, o_stride_h=128, lse_stride_t=8,
                lse_stride_h=1)
    base.update(kw)
    return ip.ccd_paged_t(**base)


def _attend(c, Q=P, K=P2, V=2 * P2, table=P, q_start=P, kv_len=P, out=3 * P2, lse=P, ws=0x10000, ws_bytes=1 << 40):
    return ip.lib().ccd_paged_attend(ctypes.byref(c), Q, K, V, table, q_start, kv_len, out, lse, ws, ws_bytes, None)


def _append(c, rope=None, K_new=P, V_new=P, slots=P, positions=P, turns=P, K=P2, V=2 * P2):
    return ip.lib().ccd_paged_append(ctypes.byref(c), None if rope is None else ctypes.byref(rope), K_new, V_new, slots, positions, turns, K, V, None)


def _plan(c, **kw):
    names = ("before", "after", "table", "table_next", "ring", "cursor", "cursor_next", "q_start", "slots", "positions")
    return ip.lib().ccd_paged_plan(ctypes.byref(c), *[kw.get(n, P) for n in names], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), ip.CCD_EINVAL), (dict(page=0), ip.CCD_EINVAL), (dict(n_pages=0), ip.CCD_EINVAL), (dict(tokens=-1), ip.CCD_EINVAL),
    (dict(table_width=0), ip.CCD_EINVAL), (dict(page=1 << 20, n_pages=1 << 11), ip.CCD_EINVAL), (dict(page=1 << 20, table_width=1 << 11, n_pages=1), ip.CCD_EINVAL),
    (dict(B=1 << 12, table_width=1 << 19, page=1), ip.CCD_EINVAL), (dict(Hq=7), ip.CCD_EINVAL), (dict(Hkv=0), ip.CCD_EINVAL), (dict(window=-1), ip.CCD_EINVAL),
    (dict(behind=2), ip.CCD_EINVAL), (dict(max_new=-1), ip.CCD_EINVAL), (dict(scale=-1.0), ip.CCD_EINVAL), (dict(scale=float("nan")), ip.CCD_EINVAL),
    (dict(d=96), ip.CCD_EUNSUPPORTED), (dict(dtype=2), ip.CCD_EUNSUPPORTED), (dict(row_stride=64), ip.CCD_EINVAL), (dict(page_stride=4), ip.CCD_EINVAL),
    (dict(head_stride=16 * 128 + 4), ip.CCD_EALIGN), (dict(q_stride_t=1028), ip.CCD_EALIGN), (dict(o_stride_h=130), ip.CCD_EALIGN),
    (dict(q_stride_b=-128), ip.CCD_EINVAL), (dict(lse_stride_h=0), ip.CCD_EINVAL),
])
def test_bad_descriptors_of_attention_are_refused(kw, code):
    assert _attend(_paged(**kw)) == code
    assert ip.ccd_paged_workspace_bytes(_paged(**kw)) == 0


def test_bad_pointers_and_workspaces_of_attention_are_refused():
    c = _paged()
    need = ip.ccd_paged_workspace_bytes(c)
    assert need >= 256
    for name in ("Q", "K", "V", "table", "q_start", "kv_len", "out"):
        assert _attend(c, **{name: None}) == ip.CCD_EINVAL
    for name in ("Q", "K", "V", "out"):
        assert _attend(c, **{name: 5 * P2 + 8}) == ip.CCD_EALIGN
    assert _attend(c, out=P) == ip.CCD_EINVAL                     # out over Q
    assert _attend(c, ws=None) == ip.CCD_EWORKSPACE
    assert _attend(c, ws=0x10010) == ip.CCD_EWORKSPACE
    assert _attend(c, ws_bytes=need - 1) == ip.CCD_EWORKSPACE
    assert _attend(_paged(tokens=0), Q=None, out=None, ws=None) == ip.CCD_OK         # an empty step: nothing to do
    assert ip.lib().ccd_paged_attend(None, P, P, P, P, P, P, P, P, P, 256, None) == ip.CCD_EINVAL
    assert ip.lib().ccd_paged_workspace_bytes(None) == 0


def test_bad_plans_are_refused():
    assert _plan(_paged(B=4097)) == ip.CCD_EUNSUPPORTED
    for kw in (dict(B=0), dict(page=0), dict(n_pages=0), dict(table_width=0), dict(tokens=-1), dict(page=1 << 30, n_pages=2)):
        assert _plan(_paged(**kw)) == ip.CCD_EINVAL
    for name in ("before", "after", "table", "table_next", "ring", "cursor", "cursor_next", "q_start", "slots", "positions"):
        assert _plan(_paged(), **{name: None}) == ip.CCD_EINVAL
    assert ip.lib().ccd_paged_plan(None, *[P] * 10, None) == ip.CCD_EINVAL


def _rope(**kw):
    base = dict(tokens=4, heads=3, d=128, rot=128, dtype=ip.CCD_BF16, x_stride_t=384, x_stride_h=128, y_stride_t=384, y_stride_h=128, base=10000.0, factor=2.0,
                context=100, low=1.0, high=4.0)
    base.update(kw)
    return ip.ccd_rope_t(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), ip.CCD_EINVAL), (dict(heads=0), ip.CCD_EINVAL), (dict(rot=0), ip.CCD_EINVAL), (dict(rot=7), ip.CCD_EINVAL), (dict(rot=130), ip.CCD_EINVAL),
    (dict(layout=2), ip.CCD_EINVAL), (dict(inverse=2), ip.CCD_EINVAL), (dict(amplitude=float("inf")), ip.CCD_EINVAL), (dict(dtype=7), ip.CCD_EUNSUPPORTED),
    (dict(d=132, rot=4), ip.CCD_EUNSUPPORTED), (dict(d=2048), ip.CCD_EUNSUPPORTED), (dict(x_stride_h=64), ip.CCD_EINVAL), (dict(y_stride_t=386), ip.CCD_EALIGN),
])
def test_bad_rotations_are_refused(kw, code):
    assert ip.lib().ccd_rope(ctypes.byref(_rope(**kw)), P, P, P, P2, None) == code


def test_bad_pointers_of_rotations_and_appends_are_refused():
    L, r = ip.lib(), _rope()
    assert L.ccd_rope(None, P, P, P, P2, None) == ip.CCD_EINVAL
    for args in ((None, P, P, P2), (P, None, P, P2), (P, P, None, P2), (P, P, P, None)):
        assert L.ccd_rope(ctypes.byref(r), *args, None) == ip.CCD_EINVAL
    assert L.ccd_rope(ctypes.byref(r), P + 8, P, P, P2, None) == ip.CCD_EALIGN
    assert L.ccd_rope(ctypes.byref(_rope(y_stride_t=512)), P, P, P, P, None) == ip.CCD_EINVAL       # in place, other strides
    assert L.ccd_rope(ctypes.byref(_rope(tokens=0)), None, None, None, None, None) == ip.CCD_OK
    c = _paged()
    for name in ("K_new", "V_new", "slots", "K", "V"):
        assert _append(c, **{name: None}) == ip.CCD_EINVAL
    for name in ("positions", "turns"):
        assert _append(c, _rope(), **{name: None}) == ip.CCD_EINVAL
    assert _append(c, K=P2, V=P2) == ip.CCD_EINVAL
    assert _append(c, K_new=P + 4) == ip.CCD_EALIGN
    assert _append(c, _rope(rot=200)) == ip.CCD_EINVAL
    assert _append(_paged(new_stride_t=100)) == ip.CCD_EINVAL
    assert _append(_paged(new_stride_h=132)) == ip.CCD_EALIGN
    assert _append(_paged(tokens=0), K_new=None, V_new=None) == ip.CCD_OK
    assert ip.lib().ccd_paged_append(None, None, P, P, P, P, P, P, P2, None) == ip.CCD_EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(rot=3), ip.CCD_EINVAL), (dict(base=1.0), ip.CCD_EINVAL), (dict(base=float("nan")), ip.CCD_EINVAL), (dict(scaling=4), ip.CCD_EUNSUPPORTED),
    (dict(scaling=ip.CCD_ROPE_LINEAR, factor=0.5), ip.CCD_EINVAL), (dict(scaling=ip.CCD_ROPE_PARTS, context=0), ip.CCD_EINVAL),
    (dict(scaling=ip.CCD_ROPE_PARTS, low=4.0), ip.CCD_EINVAL), (dict(scaling=ip.CCD_ROPE_NTK, factor=float("inf")), ip.CCD_EINVAL),
])
def test_bad_frequencies_are_refused(kw, code):
    out = (ctypes.c_uint64 * 64)()
    assert ip.lib().ccd_rope_turns(ctypes.byref(_rope(**kw)), ctypes.cast(out, ctypes.c_void_p)) == code


@pytest.mark.parametrize("name", ["plain", "linear", "ntk", "parts"])
@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (90, 1000000.0)])
def test_frequencies_are_fractions_of_a_turn(name, rot, base):
    """Within 2^-52 of the frequency (the reference is in 64-bit floats: powers within a few units of 2^-53) plus half of 2^-64."""
    kind = {"plain": ip.CCD_ROPE_PLAIN, "linear": ip.CCD_ROPE_LINEAR, "ntk": ip.CCD_ROPE_NTK, "parts": ip.CCD_ROPE_PARTS}[name]
    got = ip.rope_turns(_rope(rot=rot, base=base, scaling=kind, factor=8.0, context=8192), device="cpu").numpy().view(np.uint64)
    want = O.frequencies(rot, base, name, 8.0, 8192) / (2 * math.pi) * 2.0 ** 64
    assert len(got) == rot // 2
    np.testing.assert_allclose(got.astype(np.float64), want, rtol=2.0 ** -48, atol=1.0)


def test_reference_attention_pins():
    """Equal keys: the mean of the values and log n + the logit; one visible token: its value; torch's attention on a causal block."""
    rng = np.random.default_rng(0)
    K, V = np.zeros((2, 1, 4, 8)), rng.standard_normal((2, 1, 4, 8))
    out, lse, _, _ = O.attend(np.ones((1, 2, 8)), K, V, np.array([[1, 0]]), [0, 1], [7])
    flat = np.concatenate([V[1, 0], V[0, 0]])[:7]
    np.testing.assert_allclose(out[0, 0], flat.mean(0))
    np.testing.assert_allclose(lse, math.log(7))
    out, _, _, _ = O.attend(np.ones((3, 2, 8)), K, V, np.array([[1, 0]]), [0, 3], [3])
    np.testing.assert_allclose(out[0, 0], V[1, 0, 0])
    q, k, v = (torch.from_numpy(rng.standard_normal((2, 5, 8))) for _ in range(3))
    want = torch.nn.functional.scaled_dot_product_attention(q, k, v, is_causal=True)
    pages = [x.numpy().reshape(1, 2, 5, 8) for x in (k, v)]
    out, _, _, _ = O.attend(q.transpose(0, 1).numpy(), *pages, np.array([[0]]), [0, 5], [5])
    np.testing.assert_allclose(out, want.transpose(0, 1).numpy(), rtol=1e-12)


def test_reference_plan_worked_by_hand():
    """Pages of 4, a ring of 6 that starts at place 4: sequence 0 grows from 3 to 9 tokens (pages 2, 5), 1 is done (gives 1, 0 back), 2 starts."""
    table = np.array([[7, -1, -1], [1, 0, -1], [-1, -1, -1]], np.int32)
    ring = np.array([3, -1, -1, -1, 2, 5, 4, 6], np.int32)                         # place 4 on: 2 5 4 6 3
    nxt, ring2, cur, q_start, slots, pos = O.plan([3, 6, 0], [9, 0, 2], table, ring, [4, 5, 0, 0], page=4, n_pages=8, tokens=10)
    assert nxt.tolist() == [[7, 2, 5], [-1, -1, -1], [4, -1, -1]]
    assert ring2.tolist() == [3, 1, 0, -1, 2, 5, 4, 6] and cur.tolist() == [7, 4, 0, 0]
    assert q_start.tolist() == [0, 6, 6, 8]
    assert slots.tolist() == [31, 8, 9, 10, 11, 20, 16, 17, -1, -1] and pos.tolist() == [3, 4, 5, 6, 7, 8, 0, 1, -1, -1]


def test_reference_rope_pins():
    """A quarter turn, both layouts; turning back; lengths stay."""
    f, x = np.array([math.pi / 2, 0.0]), np.arange(1.0, 7.0).reshape(1, 1, 6)
    np.testing.assert_allclose(O.rope(x, [1], f, half=True)[0, 0], [-3, 2, 1, 4, 5, 6], atol=1e-12)
    np.testing.assert_allclose(O.rope(x, [1], f, half=False)[0, 0], [-2, 1, 3, 4, 5, 6], atol=1e-12)
    y = O.rope(x, [12345], O.frequencies(6, 10000.0), half=False)
    np.testing.assert_allclose(np.linalg.norm(y), np.linalg.norm(x))
    np.testing.assert_allclose(O.rope(y, [12345], O.frequencies(6, 10000.0), half=False, inverse=True), x)


def test_calls_of_more_threads_than_a_launch_has_are_refused():
    for kw in (dict(B=1 << 20, table_width=1, Hkv=4, Hq=4), dict(B=1 << 20, table_width=1, Hkv=1 << 12, Hq=1 << 12), dict(tokens=(1 << 25) + 1)):
        assert _attend(_paged(**kw)) == ip.CCD_EUNSUPPORTED
        assert ip.ccd_paged_workspace_bytes(_paged(**kw)) == 0
    assert ip.ccd_paged_workspace_bytes(_paged(B=1 << 20, table_width=1)) > 0 and ip.ccd_paged_workspace_bytes(_paged(tokens=1 << 25)) > 0
    assert _append(_paged(tokens=(1 << 25) + 1)) == ip.CCD_EUNSUPPORTED
    assert ip.lib().ccd_rope(ctypes.byref(_rope(tokens=(1 << 25) + 1)), P, P, P, P2, None) == ip.CCD_EUNSUPPORTED


def test_the_binding_refuses_index_tensors_that_are_too_short():
    i = lambda n: torch.zeros(n, dtype=torch.int32)                            # noqa: E731
    c = _paged()
    good = dict(len_before=i(2), len_after=i(2), block_table=i(8), block_table_next=i(8), free_pages=i(10), cursor=i(4), cursor_next=i(4), q_start=i(3),
                slots=i(6), positions=i(6))
    for name, t in good.items():
        with pytest.raises(AssertionError, match="needed"):
            ip.ccd_paged_plan(c, **{**good, name: t[:-1]})
        with pytest.raises(AssertionError, match="int32"):
            ip.ccd_paged_plan(c, **{**good, name: t.float()})
    K = torch.zeros((10, 2, 16, 128), dtype=torch.bfloat16)
    Q, K_new = torch.zeros((6, 8, 128), dtype=torch.bfloat16), torch.zeros((6, 2, 128), dtype=torch.bfloat16)
    attend = dict(block_table=i(8), q_start=i(3), kv_len=i(2))
    for name, t in attend.items():
        with pytest.raises(AssertionError, match="needed"):
            ip.ccd_paged_attend(c, Q, K, K.clone(), out=Q.clone(), lse=None, workspace=None, **{**attend, name: t[:-1]})
    with pytest.raises(AssertionError):
        ip.ccd_paged_attend(c, Q.float(), K, K.clone(), out=Q.clone(), lse=None, workspace=None, **attend)
    rope = ip.make_rope(K_new, rot=64)
    with pytest.raises(AssertionError, match="needed"):
        ip.ccd_paged_append(c, K_new, K_new.clone(), i(5), K, K.clone())
    with pytest.raises(AssertionError, match="needed"):
        ip.ccd_paged_append(c, K_new, K_new.clone(), i(6), K, K.clone(), rope=rope, positions=i(5), turns=torch.zeros(32, dtype=torch.int64))
    with pytest.raises(AssertionError, match="turns"):
        ip.ccd_paged_append(c, K_new, K_new.clone(), i(6), K, K.clone(), rope=rope, positions=i(6), turns=torch.zeros(31, dtype=torch.int64))
    with pytest.raises(AssertionError):
        ip.ccd_paged_append(c, K_new, K_new.float(), i(6), K, K.clone())
    with pytest.raises(AssertionError, match="turns"):
        ip.ccd_rope(rope, K_new, i(6), torch.zeros(32, dtype=torch.int32), K_new)


def test_positions_that_int32_could_not_count_are_refused():
    """Repeated pages make a table of 2^30 tokens small; beyond that a tile would be counted past 2^31."""
    big = dict(page=1 << 20, n_pages=1, page_stride=1 << 28, head_stride=1 << 27)
    assert ip.ccd_paged_workspace_bytes(_paged(table_width=1 << 10, **big)) > 0
    c = _paged(table_width=(1 << 10) + 1, **big)
    assert _attend(c) == _plan(c) == ip.CCD_EINVAL and ip.ccd_paged_workspace_bytes(c) == 0
