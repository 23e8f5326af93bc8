"""The memory pot of Continual Context Distillation (paper Sec. 3.2) as a thin driver around ccd_compress.

A pot holds at most n_cap cached tokens per (layer, KV head).  New context is appended until the pot is
full; then the catalyst-prompt queries of that moment score the cache and ccd_compress keeps k entries per
head in place, after which appending continues behind them.  Novelty is carried per head, because after
the first distillation heads no longer hold the same tokens in the same slots (Sec. 3.3.1).

Only buffer bookkeeping happens here; appending, attention, scoring, selection and compaction all run in the library's kernels
(the append stands in for the model forward that would write new keys and values).

`MemoryPot` is one pot per sequence, all filled alike.  `PagedPots` serves sequences of different lengths from one pool of pages; where a
page is a whole pot, a sequence's pot is distilled as soon as it is full, whatever the others hold.

Either holds its cache in 8 bits if it is given a type of code (`codes`: torch.int8 or torch.float8_e4m3fn): half of a bf16 pot's memory and of the bytes that
decoding reads.  Keys and values are quantised as they are appended, attention reads the codes; a distillation reads keys back into a buffer of its own for their
scores, and moves codes and scales of what it keeps.  The buffer has the keys of about 256 heads at a time, however many sequences and layers there are (32 layers of 8
heads, 4096 tokens of 128 in bf16: 256 MiB, while one distillation runs, next to 264 MiB of codes and scales for every sequence).
"""
from __future__ import annotations

import torch

from . import infinipot as ip


class _Kept:
    """What calls of one stream keep for the next ones: nothing says that another stream's are done with it, or have written it."""

    MOST = 16               # of rows: the oldest leaves (chunks of ever other lengths)

    def __init__(self):
        self.ws, self.rows, self.kv_len, self.held = None, {}, None, None      # rows: (pages, tokens) -> block table, q_start; held: the number in kv_len

    def workspace(self, paged, device, codes=None):
        """A graph that is being captured has one of its own, which nobody frees or uses between its replays."""
        if torch.cuda.is_current_stream_capturing():
            return self._new(paged, device, codes)
        if self.ws is None or self.ws.numel() < (ip.ccd_paged_workspace_bytes(paged) if codes is None else ip.ccd_codes_workspace_bytes(paged, codes)):
            self.ws = self._new(paged, device, codes)
        return self.ws

    @staticmethod
    def _new(paged, device, codes):
        return ip.alloc_paged_workspace(paged, device) if codes is None else ip.alloc_codes_workspace(paged, codes, device)


def _kept(by_stream):
    return by_stream.setdefault(torch.cuda.current_stream().cuda_stream, _Kept())


def _described(held, kind, geometry, make):
    """The descriptor of the last call of this kind, if this one's geometry is the same (a step's layers, a chunk's), or a new one: making and
    checking one takes longer on the host than a call."""
    last = held.get(kind)
    if last is None or last[0] != geometry:
        last = held[kind] = (geometry, make())
    return last[1]


def _geometry(*tensors):
    return [(t.shape, t.stride()) for t in tensors]


def _pool(shape, dtype, codes, scale_rows, device):
    """Keys, values, and over codes their scales (else None): shape [..., tokens, d]."""
    if codes is None:
        K = torch.zeros(shape, dtype=dtype, device=device)
        return K, torch.zeros_like(K), None, None
    if codes not in ip.CODE_TYPES:
        raise TypeError(f"unsupported code type {codes}")
    if scale_rows < 1 or scale_rows & (scale_rows - 1) or shape[-2] % scale_rows or (scale_rows > 1 and codes is not torch.float8_e4m3fn):
        raise ValueError("scale_rows is a power of two that divides the page, and 1 with codes of torch.int8")
    K = torch.zeros(shape, dtype=torch.uint8, device=device).view(codes)
    scales = torch.zeros((*shape[:-2], shape[-2] // scale_rows), dtype=torch.float32, device=device)
    return K, torch.zeros_like(K.view(torch.uint8)).view(codes), scales, torch.zeros_like(scales)


# Units (pots and heads) of which a distillation over codes reads the keys back at a time: about one for every compute unit, so that the score kernels take no longer than over all at
# once.  8 heads, 4096 tokens of 128, us: 4 sequences of 32 layers 1095 over all 1024 units, 1065 by 256, 1249 by 128, 1551 by 64; one of 48 layers 459 at once, 431 by 192; but 36 layers 351 and 420 by 144.
READ_UNITS = 256


def _read_groups(B, L, Hkv):
    """(b0, b1, l0, l1): sequences and layers whose keys are read back at a time, side by side in memory."""
    parts = (L * Hkv + READ_UNITS // 2) // READ_UNITS       # of a sequence's layers
    if parts > 1:
        each = -(-L // parts)
        return [(b, b + 1, l, min(L, l + each)) for b in range(B) for l in range(0, L, each)]
    each = max(1, READ_UNITS // (L * Hkv))
    return [(b, min(B, b + each), 0, L) for b in range(0, B, each)]


def _distil_codes(K, V, K_scales, V_scales, Q_cat, novelty, keep_idx, workspace, *, dtype, n_valid, k, T, pool_w, pool_mode, scores=None, lse=None) -> int:
    """ccd_compress (ccd_compress_lse with lse) over codes K, V [B, L, Hkv, n_cap, d]: the keys are read back for their scores.  workspace: of ccd_score, or None."""
    B, L, Hkv, n_cap, d = K.shape
    if n_valid < n_cap or n_valid <= k:
        return ip.CCD_NOOP
    # (carried per head, as the shape has it: compacted, with rows of its own for every head)
    carried = novelty if novelty is not None and novelty.dim() == 4 and (novelty.stride(1) or novelty.stride(2)) else None
    if carried is not None and any(step == 0 and size > 1 for step, size in zip(carried.stride(), carried.shape)):
        raise AssertionError("novelty that is carried per head and shared by some of them")
    device, groups = K.device, _read_groups(B, L, Hkv)
    most = max((b1 - b0) * (l1 - l0) for b0, b1, l0, l1 in groups)
    buffer = torch.empty((most, Hkv, n_cap, d), dtype=dtype, device=device)
    table = torch.arange(B * L, dtype=torch.int32, device=device)[:, None]
    q_start, kv_len = torch.arange(most + 1, dtype=torch.int32, device=device) * n_cap, torch.full((most,), n_cap, dtype=torch.int32, device=device)
    flat = [x.flatten(0, 1) for x in (K, V, K_scales, V_scales)]
    codes = ip.make_codes(flat[0], flat[2])
    scores = torch.empty((B, L, Hkv, n_valid), dtype=torch.float32, device=device) if scores is None else scores
    for b0, b1, l0, l1 in groups:
        numbers, own, queries, sums, new, into = buffer, table, Q_cat, lse, novelty, scores
        if len(groups) > 1:
            pots, first = (b1 - b0) * (l1 - l0), b0 * L + l0
            numbers, own, queries, into = buffer[:pots], table[first: first + pots], Q_cat[b0:b1, l0:l1], scores[b0:b1, l0:l1]
            new = None if novelty is None else novelty[b0:b1] if novelty.dim() == 2 else novelty[b0:b1, l0:l1]
            if lse is not None:
                sums = lse[b0:b1, l0:l1]
                sums = sums if sums.data_ptr() % 16 == 0 else sums.clone()
        paged = ip.make_paged(flat[0], tokens=own.shape[0] * n_cap, dtype=dtype, block_table=own, out=numbers)
        ip.ccd_paged_read_codes(paged, codes, flat[0], None, flat[2], None, own, q_start, kv_len, numbers, None)
        numbers = numbers.view(b1 - b0, l1 - l0, Hkv, n_cap, d)
        shape = ip.make_shape(queries, numbers, new, k=k, T=T, pool_w=pool_w, pool_mode=pool_mode, n_valid=n_valid)
        if workspace is None or (len(groups) > 1 and workspace.numel() < ip.ccd_workspace_bytes(shape)):
            workspace = ip.alloc_workspace(shape, device)
        if lse is None:
            ip.ccd_score(shape, queries, numbers, new, into, workspace)
        else:
            ip.ccd_score_lse(shape, queries, numbers, sums, new, into, workspace)
    shape.B, shape.L = B, L                                 # of all: what the selection reads
    ip.ccd_select(shape, scores, keep_idx)
    # (compacted where it stands if it is dense, else by way of a copy)
    dense = carried if carried is None else carried.contiguous()
    rc = ip.ccd_paged_compact_codes(paged, codes, *flat, keep_idx, novelty=dense)
    if dense is not carried:
        carried[..., :k].copy_(dense[..., :k])
    return rc


class MemoryPot:
    def __init__(self, B, L, Hkv, d, n_cap, k, T, *, dtype=torch.bfloat16, pool_w=7, pool_mode=ip.CCD_POOL_MAX,
                 device="cuda", codes=None):
        self.B, self.L, self.Hkv, self.d, self.n_cap, self.k, self.T = B, L, Hkv, d, n_cap, k, T
        self.pool_w, self.pool_mode = pool_w, pool_mode
        self.dtype, self.codes = dtype, codes
        self.K, self.V, self.K_scales, self.V_scales = _pool((B, L, Hkv, n_cap, d), dtype, codes, 1, device)
        self.novelty = torch.zeros((B, L, Hkv, n_cap), dtype=torch.float32, device=device)
        self.keep_idx = torch.empty((B, L, Hkv, k), dtype=torch.int32, device=device)
        self.n_valid = 0
        self.calls = 0
        self._ws = None
        self._attn = {}                         # stream -> _Kept
        self._held = {}                         # descriptors (_described)

    @property
    def room(self) -> int:
        return self.n_cap - self.n_valid

    def append(self, K_new, V_new, novelty_new) -> None:
        """K_new, V_new [B, L, Hkv, m, d]; novelty_new [B, m] (one value per token, copied to every head)."""
        m = K_new.shape[3]
        assert m <= self.room, "pot overflow: distill first"
        if self.codes is not None:
            return self._append_codes(K_new, V_new, novelty_new, m)
        shape = ip.make_shape(None, self.K, self.novelty, k=1, n_valid=self.n_valid)
        rc = ip.ccd_append(shape, self.K, self.V, self.novelty, K_new, V_new, novelty_new)
        assert rc == ip.CCD_OK, rc
        self.n_valid += m

    def _append_codes(self, K_new, V_new, novelty_new, m):
        pages = self.B * self.L
        K, V, Ks, Vs = (x.flatten(0, 1) for x in (self.K, self.V, self.K_scales, self.V_scales))
        new, values = K_new.reshape(pages, self.Hkv, m, self.d), V_new.reshape(pages, self.Hkv, m, self.d)
        paged, codes = _described(self._held, "append", _geometry(new), lambda: (
            ip.make_paged(K, tokens=pages * m, dtype=self.dtype, K_new=new), ip.make_codes(K, Ks, K_new=new)))
        rows = torch.arange(self.n_valid, self.n_valid + m, dtype=torch.int32, device=K.device)
        slots = (torch.arange(pages, dtype=torch.int32, device=K.device)[:, None] * self.n_cap + rows).reshape(-1)
        rc = ip.ccd_paged_append_codes(paged, codes, new, values, slots, K, V, Ks, Vs)
        assert rc == ip.CCD_OK, rc
        self.novelty[..., self.n_valid: self.n_valid + m] = novelty_new[:, None, None]
        self.n_valid += m

    def attend(self, Q, *, layer=None, behind=False, window=0, K=None, out=None, lse=None):
        """Attention of m query tokens over the pot: Q [B, L, Hq, m, d], or [B, Hq, m, d] of one layer.  The tokens are the pot's last m (already
        appended: each sees what stands before it and itself) or, with `behind`, stand behind it and see all of it (the catalyst prompt).
        K: other keys than the stored ones (the embedded ones of CR-RoPE; over codes a pair of codes and scales).  Returns (out, lse) like Q and Q without its last axis; the
        catalyst prompt's lse is what `distill` can take."""
        coded, one = self.codes is not None, layer is not None
        K, K_scales = (self.K, self.K_scales) if K is None else K if coded else (K, None)
        keys, values = (K[:, layer], self.V[:, layer]) if one else (K.view(-1, *K.shape[2:]), self.V.view(-1, *K.shape[2:]))
        pages, (Hq, m) = keys.shape[0], Q.shape[-3:-1]
        q = Q if one else Q.reshape(-1, *Q.shape[2:])
        out = torch.empty_like(Q, memory_format=torch.contiguous_format) if out is None else out
        lse = torch.empty(Q.shape[:-1], dtype=torch.float32, device=Q.device) if lse is None else lse
        table, q_start, kv_len = self._attn_index(pages, m, Q.device)
        o, s = (out, lse) if one else (out.view(-1, *out.shape[2:]), lse.view(-1, *lse.shape[2:]))
        paged = _described(self._held, "attend", (window, behind, self.n_valid, _geometry(keys, q, o, s)), lambda: ip.make_paged(
            keys, tokens=pages * m, dtype=self.dtype, block_table=table, Q=q, out=o, lse=s, window=window, behind=behind, max_new=m, max_len=max(1, self.n_valid)))
        if coded:
            ks, vs = (K_scales[:, layer], self.V_scales[:, layer]) if one else (K_scales.view(-1, *K_scales.shape[2:]), self.V_scales.view(-1, *K_scales.shape[2:]))
            codes = _described(self._held, "codes", _geometry(keys, ks), lambda: ip.make_codes(keys, ks))
            ws = _kept(self._attn).workspace(paged, Q.device, codes)
            rc = ip.ccd_paged_attend_codes(paged, codes, q, keys, values, ks, vs, table, q_start, kv_len, o, s, ws)
        else:
            ws = _kept(self._attn).workspace(paged, Q.device)
            rc = ip.ccd_paged_attend(paged, q, keys, values, table, q_start, kv_len, o, s, ws)
        assert rc == ip.CCD_OK, rc
        return out, lse

    def _attn_index(self, pages, m, device):
        """Block table, q_start and kv_len of `pages` pots of m query tokens each."""
        def rows():
            return (torch.arange(pages, dtype=torch.int32, device=device)[:, None].contiguous(),
                    torch.arange(pages + 1, dtype=torch.int32, device=device) * m)
        if torch.cuda.is_current_stream_capturing():        # a graph keeps its own: nothing is written before it is replayed
            return *rows(), torch.full((pages,), self.n_valid, dtype=torch.int32, device=device)
        kept = _kept(self._attn)
        if (pages, m) not in kept.rows:
            if len(kept.rows) == _Kept.MOST:
                del kept.rows[next(iter(kept.rows))]            # (the stream's own memory: what still runs is before what takes it next)
            kept.rows[pages, m] = rows()
        if kept.kv_len is None:
            kept.kv_len = torch.empty(self.B * self.L, dtype=torch.int32, device=device)
        if kept.held != self.n_valid:
            kept.kv_len.fill_(self.n_valid)
            kept.held = self.n_valid
        return *kept.rows[pages, m], kept.kv_len[:pages]

    def distill(self, Q_cat, scores=None, lse=None) -> int:
        """One CCD compression if the pot is full; returns the library's code (CCD_OK or CCD_NOOP).  lse: the catalyst rows' log-sum-exps, as
        `attend` returns them (one pass over the keys instead of two)."""
        if self.codes is not None:
            rc = _distil_codes(self.K, self.V, self.K_scales, self.V_scales, Q_cat, self.novelty, self.keep_idx, None, dtype=self.dtype, n_valid=self.n_valid, k=self.k, T=self.T,
                               pool_w=self.pool_w, pool_mode=self.pool_mode, scores=scores, lse=lse)
            if rc == ip.CCD_OK:
                self.n_valid = self.k
                self.calls += 1
            return rc
        shape = ip.make_shape(Q_cat, self.K, self.novelty, k=self.k, T=self.T, pool_w=self.pool_w,
                              pool_mode=self.pool_mode, n_valid=self.n_valid)
        if self._ws is None:
            full = ip.make_shape(Q_cat, self.K, self.novelty, k=self.k, T=self.T, pool_w=self.pool_w,
                                 pool_mode=self.pool_mode, n_valid=self.n_cap)
            self._ws = ip.alloc_workspace(full)
        if lse is not None:
            rc = ip.ccd_compress_lse(shape, Q_cat, self.K, self.V, lse, self.novelty, self.keep_idx, self._ws, scores=scores)
        else:
            rc = ip.ccd_compress(shape, Q_cat, self.K, self.V, self.novelty, self.keep_idx, self._ws, scores=scores)
        if rc == ip.CCD_OK:
            self.n_valid = self.k
            self.calls += 1
        return rc


class PagedPots:
    """Sequences of different lengths over one pool of pages, for all layers.

    A step of a serving loop: `step(lengths)` says how many tokens every sequence holds after it (one that shrinks gives pages back, 0 ends it)
    and plans where the new ones go; then, in every layer, `append` writes their keys and values and `attend` lets them attend.  The new
    tokens are numbered sequence after sequence; tensors may have more rows than that, which are left alone.  A pool whose pages
    are as long as the longest sequence is a pool of memory pots: `distill` compresses the pot of one sequence.
    scale_rows: tokens that share a scale, with codes of torch.float8_e4m3fn (pots to be distilled have a scale per token).
    """

    def __init__(self, sequences, n_pages, page, max_len, step_tokens, L, Hq, Hkv, d, *, dtype=torch.bfloat16, window=0, device="cuda", codes=None, scale_rows=1):
        self.page, self.L, self.Hq, self.window, self.step_tokens = page, L, Hq, window, step_tokens
        self.dtype, self.codes = dtype, codes
        self.K, self.V, self.K_scales, self.V_scales = _pool((n_pages, L, Hkv, page, d), dtype, codes, scale_rows, device)
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)            # noqa: E731
        self.table = torch.full((sequences, -(-max_len // page)), -1, dtype=torch.int32, device=device)
        self.free_pages = torch.arange(n_pages, dtype=torch.int32, device=device)
        self.cursor = torch.tensor([0, n_pages, 0, 0], dtype=torch.int32, device=device)
        self.before, self.after, self.q_start = ints(sequences), ints(sequences), ints(sequences + 1)
        self.slots, self.positions = ints(step_tokens), ints(step_tokens)
        self.lengths = [0] * sequences                  # on the host, as of the last step
        self.new = [0] * sequences
        self._plan = ip.make_plan(self.table, tokens=step_tokens, page=page, n_pages=n_pages)
        self._attn = {}                                 # stream -> _Kept
        self._held = {}                                 # descriptors (_described)
        self._hints()

    def _hints(self):
        self._most = max(1, *self.new), max(1, *self.lengths)

    def pages(self, length) -> int:
        return -(-length // self.page)

    def step(self, lengths) -> int:
        """Plans the step that leaves sequence b with lengths[b] tokens; returns the number of new ones.  The lengths come from the host: a step is
        not captured into a graph, its `append` and `attend` may be (for steps of the same number of rows)."""
        lengths = [int(n) for n in lengths]
        new = [max(0, n - o) for o, n in zip(self.lengths, lengths)]
        if len(lengths) != len(self.lengths) or min(lengths) < 0 or self.pages(max(lengths)) > self.table.shape[1] or sum(new) > self.step_tokens:
            raise ValueError("a length, or the number of new tokens, beyond what the pool was made for")
        held = sum(map(self.pages, self.lengths))
        if held + sum(max(0, self.pages(n) - self.pages(o)) for o, n in zip(self.lengths, lengths)) > self.K.shape[0]:
            raise ValueError("not enough free pages (those given back in a step are free from the next one on)")
        both = torch.tensor([self.lengths, lengths], dtype=torch.int32).to(self.table.device)
        self.before.copy_(both[0])
        self.after.copy_(both[1])
        rc = ip.ccd_paged_plan(self._plan, self.before, self.after, self.table, self.table, self.free_pages, self.cursor, self.cursor, self.q_start,
                               self.slots, self.positions)
        assert rc == ip.CCD_OK, rc
        self.lengths, self.new = lengths, new
        self._hints()
        return sum(new)

    def append(self, layer, K_new, V_new, rope=None, turns=None) -> None:
        """Keys and values of the step's new tokens, [rows, Hkv, d]; rope and turns (as of rope_turns): the keys are embedded at their positions."""
        rows, K, V = K_new.shape[0], self.K[:, layer], self.V[:, layer]
        if self.codes is not None:
            Ks, Vs = self.K_scales[:, layer], self.V_scales[:, layer]
            paged, codes = _described(self._held, "append", _geometry(K_new), lambda: (ip.make_paged(K, tokens=rows, dtype=self.dtype, K_new=K_new), ip.make_codes(K, Ks)))
            rc = ip.ccd_paged_append_codes(paged, codes, K_new, V_new, self.slots[:rows], K, V, Ks, Vs, rope=rope, positions=None if rope is None else self.positions[:rows],
                                           turns=turns)
            assert rc == ip.CCD_OK, rc
            return
        paged = _described(self._held, "append", _geometry(K_new), lambda: ip.make_paged(K, tokens=rows, K_new=K_new))
        rc = ip.ccd_paged_append(paged, K_new, V_new, self.slots[:rows], K, V, rope=rope, positions=None if rope is None else self.positions[:rows], turns=turns)
        assert rc == ip.CCD_OK, rc

    def attend(self, layer, Q, out=None, lse=None):
        """Q [rows, Hq, d] of the step's new tokens, their keys and values appended; returns (out, lse)."""
        out = torch.empty_like(Q, memory_format=torch.contiguous_format) if out is None else out
        lse = torch.empty(Q.shape[:2], dtype=torch.float32, device=Q.device) if lse is None else lse
        K, V = self.K[:, layer], self.V[:, layer]
        paged = _described(self._held, "attend", (self.window, self._most, _geometry(Q, out, lse)), lambda: ip.make_paged(
            K, tokens=Q.shape[0], dtype=self.dtype, block_table=self.table, Q=Q, out=out, lse=lse, window=self.window, max_new=self._most[0], max_len=self._most[1]))
        if self.codes is not None:
            Ks, Vs = self.K_scales[:, layer], self.V_scales[:, layer]
            codes = _described(self._held, "codes", None, lambda: ip.make_codes(K, Ks))
            ws = _kept(self._attn).workspace(paged, Q.device, codes)
            rc = ip.ccd_paged_attend_codes(paged, codes, Q, K, V, Ks, Vs, self.table, self.q_start, self.after, out, lse, ws)
        else:
            ws = _kept(self._attn).workspace(paged, Q.device)
            rc = ip.ccd_paged_attend(paged, Q, K, V, self.table, self.q_start, self.after, out, lse, ws)
        assert rc == ip.CCD_OK, rc
        return out, lse

    def distill(self, b, page_id, Q_cat, novelty, keep_idx, workspace, *, k, T, pool_w=7, pool_mode=ip.CCD_POOL_MAX, lse=None) -> int:
        """Compresses the pot of sequence b, the page page_id that it holds (one page per sequence), if it is full: Q_cat [1, L, Hq, P, d], novelty
        [1, page] or [1, L, Hkv, page], keep_idx [1, L, Hkv, k].  Returns the library's code; after CCD_OK the sequence has k tokens, as of the
        next step."""
        assert self.table.shape[1] == 1, "distillation needs pages that are whole pots"
        assert self.codes is None or self.K_scales.shape[-1] == self.page, "distillation needs a scale per token"
        K, V = self.K[page_id: page_id + 1], self.V[page_id: page_id + 1]
        if self.codes is not None:
            rc = _distil_codes(K, V, self.K_scales[page_id: page_id + 1], self.V_scales[page_id: page_id + 1], Q_cat, novelty, keep_idx, workspace, dtype=self.dtype,
                               n_valid=self.lengths[b], k=k, T=T, pool_w=pool_w, pool_mode=pool_mode, lse=lse)
        else:
            shape = ip.make_shape(Q_cat, K, novelty, k=k, T=T, pool_w=pool_w, pool_mode=pool_mode, n_valid=max(1, self.lengths[b]))
            if lse is not None:
                rc = ip.ccd_compress_lse(shape, Q_cat, K, V, lse, novelty, keep_idx, workspace)
            else:
                rc = ip.ccd_compress(shape, Q_cat, K, V, novelty, keep_idx, workspace)
        if rc == ip.CCD_OK:
            self.lengths[b] = k
            self._hints()
        return rc
