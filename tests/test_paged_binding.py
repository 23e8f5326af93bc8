"""What the binding of the paged calls refuses before anything is launched: a tensor that is elsewhere, one that the descriptor reaches past, another type.
Host tensors stand for those of the current device here, and the library for one that only counts its calls."""
import pytest
import torch

from paper_2410_01518_amd import infinipot as ip

B, TOKENS, HQ, HKV, D, PAGE, N_PAGES, W = 3, 6, 8, 2, 64, 16, 10, 4


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 5


class Counting:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


@pytest.fixture
def launches(monkeypatch):
    L = Counting()
    monkeypatch.setattr(ip, "lib", lambda: L)
    monkeypatch.setattr(ip, "_get_device", lambda: -1)               # (where host tensors say they are)
    monkeypatch.setattr(ip, "_raw_stream", lambda device: 0)
    return L


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _plan():
    t = dict(len_before=_ints(B), len_after=_ints(B), block_table=_ints(B, W), block_table_next=_ints(B, W), free_pages=_ints(N_PAGES), cursor=_ints(4), cursor_next=_ints(4),
             q_start=_ints(B + 1), slots=_ints(TOKENS), positions=_ints(TOKENS))
    paged = ip.make_plan(t["block_table"], tokens=TOKENS, page=PAGE, n_pages=N_PAGES)
    return t, lambda t: ip.ccd_paged_plan(paged, **t)


def _rope():
    t = dict(X=_bf16(TOKENS, HQ, D), positions=_ints(TOKENS), turns=torch.zeros(D // 2, dtype=torch.int64), Y=_bf16(TOKENS, HQ, D))
    rope = ip.make_rope(t["X"], t["Y"])
    return t, lambda t: ip.ccd_rope(rope, **t)


def _append(embedded):
    t = dict(K_new=_bf16(TOKENS, HKV, D), V_new=_bf16(TOKENS, HKV, D), slots=_ints(TOKENS), K_pages=_bf16(N_PAGES, HKV, PAGE, D), V_pages=_bf16(N_PAGES, HKV, PAGE, D))
    paged = ip.make_paged(t["K_pages"], tokens=TOKENS, K_new=t["K_new"])
    rope = None
    if embedded:
        t.update(positions=_ints(TOKENS), turns=torch.zeros(D // 2, dtype=torch.int64))
        rope = ip.make_rope(t["K_new"])
    return t, lambda t: ip.ccd_paged_append(paged, rope=rope, **t)


def _attend(batched=False):
    Q = _bf16(B, HQ, TOKENS // B, D) if batched else _bf16(TOKENS, HQ, D)
    t = dict(Q=Q, K_pages=_bf16(N_PAGES, HKV, PAGE, D), V_pages=_bf16(N_PAGES, HKV, PAGE, D), block_table=_ints(B, W), q_start=_ints(B + 1), kv_len=_ints(B), out=Q.clone(),
             lse=torch.zeros(Q.shape[:-1]), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    paged = ip.make_paged(t["K_pages"], tokens=TOKENS, block_table=t["block_table"], Q=Q, out=t["out"], lse=t["lse"])
    return t, lambda t: ip.ccd_paged_attend(paged, **t)


CALLS = {"plan": _plan, "rope": _rope, "append": lambda: _append(False), "append embedded": lambda: _append(True), "attend": _attend, "attend batched": lambda: _attend(True)}


@pytest.mark.parametrize("name", CALLS)
def test_every_tensor_has_to_be_on_the_current_device(launches, name):
    t, call = CALLS[name]()
    assert call(t) == ip.CCD_OK and launches.calls == 1
    for x in t:
        with pytest.raises(ValueError, match="current device"):
            call({**t, x: t[x].as_subclass(Elsewhere)})
    assert launches.calls == 1


@pytest.mark.parametrize("name", CALLS)
def test_no_tensor_may_end_before_what_the_descriptor_reaches(launches, name):
    """One row, head or page less, or strides that go further."""
    t, call = CALLS[name]()
    for x in t:
        if x == "workspace":                                           # (the library looks at its size)
            continue
        for axis in range(t[x].dim()):
            if t[x].dtype is torch.int32 and t[x].dim() > 1:
                short = t[x][:-1]
            else:
                short = t[x].narrow(axis, 0, t[x].shape[axis] - 1).clone()
            pair = {"K_new": "V_new", "V_new": "K_new", "K_pages": "V_pages", "V_pages": "K_pages"}.get(x)
            with pytest.raises(AssertionError):
                call({**t, x: short, **({pair: short.clone()} if pair else {})})
            if pair:
                with pytest.raises(AssertionError, match="differ"):
                    call({**t, x: short})
    assert launches.calls == 0


def test_strides_of_a_longer_tensor(launches):
    """A descriptor of rows that lie apart, and a tensor whose rows do not."""
    wide = _bf16(TOKENS, HQ + 4, D)
    Q, t = wide[:, 2: HQ + 2], _attend()[0]
    paged = ip.make_paged(t["K_pages"], tokens=TOKENS, block_table=t["block_table"], Q=Q, out=t["out"], lse=t["lse"])
    assert ip.ccd_paged_attend(paged, **{**t, "Q": Q}) == ip.CCD_OK
    assert ip.ccd_paged_attend(paged, **{**t, "Q": wide[:, 4:]}) == ip.CCD_OK            # other heads of the same rows
    with pytest.raises(AssertionError):
        ip.ccd_paged_attend(paged, **{**t, "Q": Q.contiguous()})
    with pytest.raises(AssertionError):
        ip.ccd_paged_attend(paged, **{**t, "Q": Q[1:]})
    assert launches.calls == 2


def test_more_rows_than_the_descriptor_has_are_fine(launches):
    for name in ("rope", "append embedded", "attend"):
        t, call = CALLS[name]()
        rows = {k: torch.cat([v, v[-1:]]) for k, v in t.items() if k in ("X", "Y", "positions", "K_new", "V_new", "slots", "Q", "out", "lse")}
        assert call({**t, **rows}) == ip.CCD_OK
    t, call = _attend()
    assert call({**t, "lse": None}) == ip.CCD_OK and call({**t, "workspace": None}) == ip.CCD_OK
    empty = ip.make_paged(t["K_pages"], tokens=0, block_table=t["block_table"], Q=t["Q"][:0])
    assert ip.ccd_paged_attend(empty, **{**t, "Q": t["Q"][:0], "out": t["out"][:0], "lse": None}) == ip.CCD_OK


@pytest.mark.parametrize("name,tensors", [("rope", ("X",)), ("rope", ("Y",)), ("rope", ("X", "Y")), ("append", ("K_new", "V_new")), ("append", ("K_new", "V_new", "K_pages", "V_pages")),
                                          ("attend", ("Q",)), ("attend", ("out",)), ("attend", ("lse",)), ("attend", ("Q", "out", "K_pages", "V_pages"))])
def test_types_that_are_not_the_descriptors(launches, name, tensors):
    t, call = CALLS[name]()
    with pytest.raises(AssertionError, match="type"):
        call({**t, **{x: t[x].to(torch.bfloat16 if t[x].dtype is torch.float32 else torch.float32) for x in tensors}})
    assert launches.calls == 0
