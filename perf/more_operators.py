"""The operators of a paged key/value cache that is held in 8 bits, as cases that can be timed and compared with their plain forms.

A cache in 8 bits has half the bytes of a bf16 one, which is what decoding reads and what a memory pot occupies.  New keys and values
are quantised as they are written, keys embedded on the way (`append`; the pass reads back what it wrote, and with it what it rescaled); cached
tokens are read back as numbers for what does not take codes, such as the catalyst prompt's scores (`read`); new tokens attend
over codes and scales (`attend`); a distillation keeps some rows of every pot, in place (`compact`).

int8: a scale per token and head, s = max(|x| / 127, 2^-120), code = x / s rounded, halves to even.  e4m3: a scale per block of `rows` tokens and head, the
smallest power of two s >= 2^-120 with |x| <= 448 s; a block whose row 0 is written begins anew, otherwise its scale can only grow, and
the rows before the new ones are taken to the new scale.

With `own` false, `run` computes a case in elementary torch operations, in 32 bits (rotations and what is rounded to a code in 64); with `own`
true it makes the library's calls.  Lengths are a function of the case (`mix` seeds them), values of the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

SHARED = 0.8        # share of a query's variance that all queries of its head have in common
LEAST = 2.0 ** -120
BASE = 500000.0     # of the rotary frequencies


def _tokens(op, name, B, Hq, Hkv, d, page, shortest, longest, new, mix, *, code="int8", rows=1, dtype="bf16", window=0, behind=False, pad=0, rope=False,
            keys=False, heads=False):
    """Sequences of shortest .. longest cached tokens, the new ones among them; `new` tokens each, or 1 .. -new where negative."""
    return dict(name=name, op=op, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, shortest=shortest, longest=longest, new=new, mix=mix, code=code, rows=rows, dtype=dtype,
                window=window, behind=behind, pad=pad, rope=rope, keys=keys, heads=heads)


def _compact(name, pots, Hkv, d, page, k, *, code="int8", novelty=True):
    return dict(name=name, op="compact", B=pots, Hkv=Hkv, d=d, page=page, k=k, code=code, rows=1, novelty=novelty)


def listed():
    return [
        # one decoding step of a batch: a token each into blocks that hold earlier ones, keys embedded
        _tokens("append", "append_decode", 64, 32, 8, 128, 64, 200, 2000, 1, 1, code="e4m3", rows=16, rope=True),
        # chunks of several prompts, a scale per token
        _tokens("append", "append_chunk", 4, 32, 8, 128, 64, 6000, 8192, 4096, 2, rope=True, pad=100),
        # a few ragged chunks of an fp32 model, odd pages, keys as they are
        _tokens("append", "append_ragged_fp32", 7, 3, 3, 64, 37, 100, 900, -300, 3, dtype="fp32", pad=5),
        # the keys of a layer stack's full pots, for the scores of the catalyst prompt
        _tokens("read", "read_pot_keys", 32, 32, 8, 128, 4096, 4096, 4096, 4096, 4, keys=True, heads=True),
        # sequences handed on as fp32 tensors
        _tokens("read", "read_ragged_fp32", 5, 3, 3, 64, 100, 300, 3001, -2500, 5, code="e4m3", rows=4, dtype="fp32", pad=11),
        # a decoding step over short caches
        _tokens("attend", "attend_decode_short", 4, 32, 8, 128, 16, 200, 500, 1, 6),
        # a decoding step of a batch of uneven sequences, blocks of 16 tokens
        _tokens("attend", "attend_decode_batch", 64, 32, 8, 128, 64, 500, 8192, 1, 7, code="e4m3", rows=16),
        # a decoding step of one long sequence
        _tokens("attend", "attend_decode_long", 1, 32, 8, 128, 256, 131072, 131072, 1, 8),
        # a chunk of 2048 tokens that fills a memory pot of 4096: the pot is the page
        _tokens("attend", "attend_pot", 1, 32, 8, 128, 4096, 4096, 4096, 2048, 9),
        # ragged chunks, single tokens among them, a sliding window, an fp32 model
        _tokens("attend", "attend_ragged_fp32", 5, 12, 3, 64, 100, 300, 3001, -701, 10, code="e4m3", rows=4, dtype="fp32", window=1024, pad=11),
        # distillation of one layer's pots
        _compact("compact_layer", 1, 8, 128, 2048, 1024, novelty=False),
        # ... of a whole model's
        _compact("compact_stack", 32, 8, 128, 4096, 2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(("attend", "append", "read", "compact"), (50, 20, 15, 15))[0]
    code, dtype = rng.choice(("int8", "e4m3")), rng.choices(("bf16", "fp32"), (75, 25))[0]
    d, Hkv, G = rng.choice((64, 128, 128)), rng.choice((1, 2, 3, 4, 8, 8)), rng.choice((1, 2, 3, 4, 4, 8))
    page = rng.choice((16, 32, 37, 64, 100, 256, 4096))
    rows = rng.choice([r for r in (1, 2, 4, 16, 32, 64) if page % r == 0]) if code == "e4m3" else 1
    pad = rng.choice((0, 0, 7))
    if op == "compact":
        n = _log_int(rng, 16, 4096)
        case = _compact("", _log_int(rng, 1, 32), Hkv, d, n, max(1, min(n, int(n * rng.uniform(0.1, 1.0)))), code=code, novelty=rng.random() < 0.5)
    elif op == "attend":
        while True:
            decode = rng.random() < 0.45
            B, longest = _log_int(rng, 1, 64 if decode else 8), _log_int(rng, 100, 131072 if decode else 32768)
            new = rng.choice((1, 1, 1, 2, 5, -8)) if decode else rng.choice((-1, 1)) * _log_int(rng, 16, 2048)
            gathered, scores = B * longest * Hkv * d, B * longest * Hkv * G * abs(new)
            if gathered <= 64 * 8192 * 8 * 128 and scores <= (4096 * 32 * 2048 if dtype == "bf16" else 1 << 28) and abs(new) <= longest:
                break
        case = _tokens(op, "", B, Hkv * G, Hkv, d, page, max(1, int(longest * rng.random())), longest, new, rng.randrange(1 << 30), code=code, rows=rows, dtype=dtype,
                       window=_log_int(rng, 32, longest + 32) if rng.random() < 0.25 else 0, behind=rng.random() < 0.15, pad=pad)
    else:
        while True:
            B, longest = _log_int(rng, 1, 128), _log_int(rng, 20, 8192)
            new = rng.choice((-1, 1)) * _log_int(rng, 1, 4096)
            if B * longest <= 65536 and B * abs(new) <= 16384 and abs(new) <= longest:
                break
        rope = op == "append" and dtype == "bf16" and rng.random() < 0.7
        case = _tokens(op, "", B, Hkv * G, Hkv, d, page, max(1, int(longest * rng.random())), longest, new, rng.randrange(1 << 30), code=code, rows=rows, dtype=dtype, pad=pad,
                       rope=rope, keys=op == "read" and rng.random() < 0.5)
    del case["name"]
    return case


_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _lengths(case):
    """Cached tokens of every sequence, and how many of them are new (with `behind`: how many queries stand behind them)."""
    rng = random.Random(case["mix"])
    lens = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(case["B"])]
    lens[0] = case["longest"]
    new = [case["new"] if case["new"] > 0 else rng.choice((1, rng.randint(1, -case["new"]))) for _ in lens]
    return lens, [m if case["behind"] else min(m, n) for m, n in zip(new, lens)]


def _read_lengths(case):
    """How many of a sequence's last tokens a pass reads: the new ones, and with them what stands in the first one's block."""
    lens, new = _lengths(case)
    return [n - (n - m) // case["rows"] * case["rows"] for n, m in zip(lens, new)] if case["op"] == "append" else new


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(counts):
    c = torch.tensor([0] + counts, device="cuda")
    return torch.cumsum(c, 0).to(torch.int32)


def _power_of_two(top):
    """The smallest power of two s >= LEAST with top <= 448 s."""
    m, e = torch.frexp(top)                    # top = m 2^e, 1/2 <= m < 1, and 448 = 7/8 of 2^9
    return torch.ldexp(torch.ones_like(top), (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-120)).clamp(min=LEAST)


def _scales(code, top):
    return _power_of_two(top.float()) if code == "e4m3" else (top.double() / 127.0).float().clamp(min=LEAST)


def _to_codes(code, x, s):
    """x / s as codes; x and s in 64 bits."""
    y = x / s
    return y.float().to(torch.float8_e4m3fn).view(torch.int8) if code == "e4m3" else torch.round(y).to(torch.int8)


def _numbers(code, bits):
    return bits.view(torch.float8_e4m3fn).float() if code == "e4m3" else bits.float()


def _quantised(case, x):
    """Codes (as bytes) and scales of whole pages x [n_pages, Hkv, page, d]."""
    n, H, page, d = x.shape
    rows = case["rows"]
    s = _scales(case["code"], x.abs().reshape(n, H, page // rows, rows * d).amax(-1))
    return _to_codes(case["code"], x.float(), s.repeat_interleave(rows, -1)[..., None]), s


def _cache(case, n_pages, g):
    H, page, d = case["Hkv"], case["page"], case["d"]
    x = torch.empty((n_pages, H, page, d), dtype=torch.float32, device="cuda").normal_(generator=g)
    # one token in a hundred is four times as long (attention sinks and other outliers)
    K, Ks = _quantised(case, x * torch.where(torch.rand((n_pages, 1, page, 1), generator=g, device="cuda") < 0.01, 4.0, 1.0))
    V, Vs = _quantised(case, x.normal_(generator=g))
    t = torch.float8_e4m3fn if case["code"] == "e4m3" else torch.int8
    return dict(K=K.view(t), V=V.view(t), Ks=Ks, Vs=Vs)


def _table(case, lens, g):
    """Pages of every sequence, anywhere in the pool; and how many pages the pool has."""
    page, W = case["page"], -(-max(lens) // case["page"])
    held = torch.tensor([-(-n // page) for n in lens], device="cuda")
    n_pages = sum(-(-n // page) for n in lens) + 3
    ids = torch.arange(n_pages, device="cuda") if case["heads"] else torch.randperm(n_pages, generator=g, device="cuda")
    col = torch.arange(W, device="cuda")[None, :]
    first = torch.cumsum(held, 0) - held
    return torch.where(col < held[:, None], ids[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32), n_pages


def _inv_freq(d):
    """Radians per position of the pairs (i, i + d/2), in 64 bits."""
    return BASE ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)


def _prepare_compact(case, g):
    B, H, n, k = case["B"], case["Hkv"], case["page"], case["k"]
    s = _cache(case, B, g)
    s["keep"] = torch.rand((B, H, n), generator=g, device="cuda").topk(k, -1).indices.sort(-1).values.to(torch.int32)
    s["novelty"] = torch.rand((B, H, n), generator=g, device="cuda") if case["novelty"] else None
    return s


def _prepare_tokens(case, g):
    lens, new = _lengths(case)
    read = _read_lengths(case)
    Hq, Hkv, d, page, dt, pad = case["Hq"], case["Hkv"], case["d"], case["page"], _DT[case["dtype"]], case["pad"]
    table, n_pages = _table(case, lens, g)
    s = dict(_cache(case, n_pages, g), table=table, lens=_ints(lens), q_start=_starts(new), read_start=_starts(read), max_len=max(lens), max_new=max(new))
    T, T_read = sum(new), sum(read)
    if case["op"] == "attend":
        head = torch.randn((Hkv, 1, d), generator=g, device="cuda").expand(Hkv, Hq // Hkv, d).reshape(1, Hq, d)
        s["Q"] = (math.sqrt(SHARED) * head + math.sqrt(1.0 - SHARED) * torch.randn((T + pad, Hq, d), generator=g, device="cuda")).to(dt)
        s["out"], s["lse"] = torch.zeros_like(s["Q"]), torch.zeros((T + pad, Hq), dtype=torch.float32, device="cuda")
        return s
    shape = (case["B"], Hkv, case["new"], d) if case["heads"] else (T_read + pad, Hkv, d)
    s["K_out"] = torch.zeros(shape, dtype=dt, device="cuda")
    s["V_out"] = None if case["keys"] else torch.zeros(shape, dtype=dt, device="cuda")
    if case["op"] == "append":
        # tokens differ in length, so that blocks grow; queries, keys and values as one projection leaves them
        x = torch.randn((T + pad, 2 * Hkv + Hq, d), generator=g, device="cuda") * torch.exp(torch.randn((T + pad, 1, 1), generator=g, device="cuda"))
        s["new"] = x.to(dt)
        i = torch.arange(T, device="cuda")
        b = torch.searchsorted(s["q_start"][1:].contiguous(), i.to(torch.int32), right=True)
        pos = (s["lens"].long() - s["q_start"][1:].long())[b] + i
        slots = table[b, pos // page].long() * page + pos % page
        s["slots"], s["positions"] = (torch.cat([v, v.new_full((pad,), -1)]).to(torch.int32) for v in (slots, pos))
        s["inv"] = _inv_freq(d)
    return s


def _handles(case, s):
    """What a program keeps for its calls: descriptors, frequencies, workspace."""
    from paper_2410_01518_amd import infinipot as ip
    s["codes"] = ip.make_codes(s["K"], s["Ks"])
    if case["op"] == "compact":
        s["paged"] = ip.make_paged(s["K"], tokens=0, dtype=torch.bfloat16)
        return
    dt = _DT[case["dtype"]]
    if case["op"] == "attend":
        s["paged"] = ip.make_paged(s["K"], tokens=s["Q"].shape[0], dtype=dt, block_table=s["table"], Q=s["Q"], out=s["out"], lse=s["lse"], window=case["window"],
                                   behind=case["behind"], max_new=s["max_new"], max_len=s["max_len"])
        s["ws"] = ip.alloc_codes_workspace(s["paged"], s["codes"])
        return
    s["back"] = ip.make_paged(s["K"], tokens=case["B"] * case["new"] if case["heads"] else s["K_out"].shape[0], dtype=dt, block_table=s["table"], out=s["K_out"])
    if case["op"] == "append":
        K_new = s["new"][:, case["Hq"]: case["Hq"] + case["Hkv"]]
        s["paged"] = ip.make_paged(s["K"], tokens=K_new.shape[0], dtype=dt, K_new=K_new)
        s["rope"] = ip.make_rope(K_new, base=BASE) if case["rope"] else None
        s["turns"] = ip.rope_turns(s["rope"]) if case["rope"] else None


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = _prepare_compact(case, g) if case["op"] == "compact" else _prepare_tokens(case, g)
    s["case"] = case
    if own:
        _handles(case, s)
    return s


def _gathered(s, X, scales, pages, at):
    """Numbers at rows `at` of `pages` [..., Hkv, d]."""
    case = s["case"]
    bits = s[X].view(torch.int8)[pages, :, at]
    return _numbers(case["code"], bits) * s[scales][pages, :, at // case["rows"]][..., None]


def _plain_write(s, X, scales, x, slots):
    """x [tokens, Hkv, d], in 64 bits, to the rows of `slots`, block by block."""
    case = s["case"]
    code, rows, page = case["code"], case["rows"], case["page"]
    bits = s[X].view(torch.int8)
    n_pages, H, _, d = bits.shape
    blocks, which = torch.unique(slots // rows, return_inverse=True)
    here, block = blocks // (page // rows), blocks % (page // rows)
    row = slots % rows
    new = torch.zeros((blocks.numel(), rows, H, d), dtype=torch.float64, device=x.device)
    written = torch.zeros((blocks.numel(), rows), dtype=torch.bool, device=x.device)
    new[which, row], written[which, row] = x, True
    s1 = _scales(code, new.abs().amax((1, 3)))
    s0 = s[scales][here, :, block]
    anew = written[:, :1]
    grown = torch.where(anew, s1, torch.maximum(s0, s1))                                            # [blocks, Hkv]
    at = block[:, None] * rows + torch.arange(rows, device=x.device)
    old = bits[here[:, None], :, at]                                                                # [blocks, rows, Hkv, d]
    first = torch.where(written, torch.arange(rows, device=x.device), rows).amin(1)
    taken = (grown > s0)[:, None, :, None] & ~anew[:, :, None, None] & (torch.arange(rows, device=x.device) < first[:, None])[..., None, None]
    again = _to_codes(code, _numbers(code, old).double() * s0[:, None, :, None].double(), grown[:, None, :, None].double())
    now = torch.where(written[..., None, None], _to_codes(code, new, grown[:, None, :, None].double()), torch.where(taken, again, old))
    bits[here[:, None], :, at] = now
    s[scales][here, :, block] = grown


def _plain_append(s):
    case = s["case"]
    here = s["slots"] >= 0
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    k, v = s["new"][here][:, Hq: Hq + Hkv].double(), s["new"][here][:, Hq + Hkv:].double()
    if case["rope"]:
        angle = s["positions"][here].double()[:, None] * s["inv"]
        cos, sin = angle.cos()[:, None], angle.sin()[:, None]
        u, w = k[..., : d // 2], k[..., d // 2:]
        k = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    slots = s["slots"][here].long()
    _plain_write(s, "K", "Ks", k, slots)
    _plain_write(s, "V", "Vs", v, slots)


def _plain_read(s):
    case = s["case"]
    start, page = s["read_start"].long(), case["page"]
    i = torch.arange(sum(_read_lengths(case)), device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), i, right=True)
    t = s["lens"].long()[b] - start[1:][b] + i
    pages = s["table"][b, t // page].long()

    def back(X, scales, out):
        x = _gathered(s, X, scales, pages, t % page).to(out.dtype)
        if case["heads"]:
            out.copy_(x.reshape(case["B"], case["new"], case["Hkv"], case["d"]).transpose(1, 2))
        else:
            out[: x.shape[0]] = x

    back("K", "Ks", s["K_out"])
    if not case["keys"]:
        back("V", "Vs", s["V_out"])


def _plain_attend(s):
    case, Q, N, M = s["case"], s["Q"], s["max_len"], s["max_new"]
    T, Hq, d = Q.shape
    page, Hkv, B = case["page"], case["Hkv"], case["B"]
    G = Hq // Hkv
    t = torch.arange(N, device=Q.device)
    pages = s["table"][:, t // page].long().clamp(min=0)                                             # [B, N]
    k = _gathered(s, "K", "Ks", pages, t % page).permute(0, 2, 3, 1).contiguous()                    # [B, Hkv, d, N]
    v = _gathered(s, "V", "Vs", pages, t % page).transpose(1, 2).contiguous()                        # [B, Hkv, N, d]
    start, count = s["q_start"][:-1].long(), (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(M, device=Q.device)
    rows = (start[:, None] + i).clamp(max=T - 1)
    q = Q[rows].float().reshape(B, M, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * M, d).contiguous()
    x = torch.matmul(q, k).reshape(B, Hkv, G, M, N) * (1.0 / math.sqrt(d))
    lens = s["lens"].long()
    pos = (lens if case["behind"] else lens - count)[:, None] + i                                    # [B, M]
    seen = (t <= pos[..., None]) & (t < lens[:, None, None])
    if case["window"] > 0:
        seen &= t > pos[..., None] - case["window"]
    x = x.masked_fill(~seen[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.reshape(B, Hkv, G * M, N), v).reshape(B, Hkv, G, M, d) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(-1)                                                       # an empty row: -inf
    mine = i < count[:, None]
    to = rows[mine]
    s["out"][to] = o.permute(0, 3, 1, 2, 4).reshape(B, M, Hq, d)[mine].to(Q.dtype)
    s["lse"][to] = lse.permute(0, 3, 1, 2).reshape(B, M, Hq)[mine]


def _plain_compact(s):
    k, keep = s["keep"].shape[-1], s["keep"].long()
    p = torch.arange(keep.shape[0], device="cuda")[:, None, None]
    h = torch.arange(keep.shape[1], device="cuda")[None, :, None]
    K, V = s["K"].view(torch.int8), s["V"].view(torch.int8)
    K[:, :, :k], V[:, :, :k] = K[p, h, keep], V[p, h, keep]
    s["Ks"][:, :, :k], s["Vs"][:, :, :k] = s["Ks"][p, h, keep], s["Vs"][p, h, keep]
    if s["novelty"] is not None:
        s["novelty"][:, :, :k] = s["novelty"][p, h, keep]


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "append":
            _plain_append(s)
            _plain_read(s)
        elif op == "read":
            _plain_read(s)
        elif op == "attend":
            _plain_attend(s)
        else:
            _plain_compact(s)
    else:
        from paper_2410_01518_amd import infinipot as ip
        if op == "append":
            Hq, Hkv = case["Hq"], case["Hkv"]
            ip.ccd_paged_append_codes(s["paged"], s["codes"], s["new"][:, Hq: Hq + Hkv], s["new"][:, Hq + Hkv:], s["slots"], s["K"], s["V"], s["Ks"], s["Vs"],
                                      rope=s["rope"], positions=s["positions"], turns=s["turns"])
        if op in ("append", "read"):
            ip.ccd_paged_read_codes(s["back"], s["codes"], s["K"], s["V"], s["Ks"], s["Vs"], s["table"], s["read_start"], s["lens"], s["K_out"], s["V_out"])
        elif op == "attend":
            ip.ccd_paged_attend_codes(s["paged"], s["codes"], s["Q"], s["K"], s["V"], s["Ks"], s["Vs"], s["table"], s["q_start"], s["lens"], s["out"], s["lse"], s["ws"])
        else:
            ip.ccd_paged_compact_codes(s["paged"], s["codes"], s["K"], s["V"], s["Ks"], s["Vs"], s["keep"], novelty=s["novelty"])
    if op == "attend":
        return {"out": s["out"], "lse": s["lse"]}
    if op == "compact":
        # rows are moved, not computed: their bits are compared as whole numbers
        moved = {"K": s["K"].view(torch.int8), "V": s["V"].view(torch.int8), "Ks": s["Ks"].view(torch.int32), "Vs": s["Vs"].view(torch.int32)}
        return moved if s["novelty"] is None else {**moved, "novelty": s["novelty"].view(torch.int32)}
    return {"K": s["K_out"]} if case["keys"] else {"K": s["K_out"], "V": s["V_out"]}


def work(case):
    """append: new rows read, codes, scales and the numbers read back written, rows that stand in front of them in their block read.  read: codes and scales read, numbers written.
    attend: queries and the visible codes and scales read, outputs and log-sum-exps written; two products per visible pair.  compact: kept rows read and written."""
    d, H, R = case["d"], case["Hkv"], case["rows"]
    if case["op"] == "compact":
        return {"bytes": case["B"] * H * case["k"] * (4 * (d + 4) + (8 if case["novelty"] else 0) + 4), "flops": 0}
    lens, new = _lengths(case)
    e = 2 if case["dtype"] == "bf16" else 4
    row = d + 4.0 / R                                    # a code row of one head and its share of a scale
    if case["op"] in ("append", "read"):
        T, T_read, sides = sum(new), sum(_read_lengths(case)), 1 if case["keys"] else 2
        if case["op"] == "read":
            return {"bytes": sides * T * H * (row + e * d), "flops": sides * T * H * d}
        return {"bytes": 2 * H * (T * (e * d + row) + (T_read - T) * row + T_read * e * d) + 8 * T, "flops": 2 * T * H * d * 3}
    pairs, tokens = 0, 0
    for n, m in zip(lens, new):
        p = n if case["behind"] else n - m
        low = 0 if not case["window"] else max(0, min(n, p - case["window"] + 1))
        tokens += max(0, n - low)
        for i in range(m):
            first = max(0, p + i - case["window"] + 1) if case["window"] else 0
            pairs += max(0, min(n, p + i + 1) - first)
    rows = sum(new) * case["Hq"]
    return {"bytes": 2 * tokens * H * row + rows * (2 * e * d + 4), "flops": 4 * d * case["Hq"] * pairs}


def exact(case, seed):
    """In 64 bits, sequence by sequence; a compaction moves rows and has no such value."""
    if case["op"] == "compact":
        return None
    s = prepare(case, seed)
    lens, new = _lengths(case)
    d, page, R, Hq, Hkv = case["d"], case["page"], case["rows"], case["Hq"], case["Hkv"]

    def tokens_of(b, t, X, scales):
        """Numbers of tokens t of sequence b [tokens, Hkv, d]."""
        ids = s["table"][b].long()[t // page]
        c = s[X].view(torch.uint8)[ids, :, t % page]
        if case["code"] == "int8":
            c = torch.where(c > 127, c.double() - 256.0, c.double())
        else:                                             # sign, four bits of exponent (bias 7), three of mantissa
            c = c.long()
            ex, man = (c >> 3) & 15, (c & 7).double()
            c = torch.where(c > 127, -1.0, 1.0) * torch.where(ex == 0, man * 2.0 ** -9, (1.0 + man / 8.0) * torch.exp2(ex.double() - 7.0))
        return c * s[scales].double()[ids, :, t % page // R][..., None]

    def nearest(y, s_):
        """The numbers that codes stand for, nearest to y; s_ the scale."""
        if case["code"] == "int8":
            return torch.round(y / s_) * s_
        z = y / s_
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3.0)
        return torch.round(z / step) * step * s_

    def scale_of(top):
        if case["code"] == "int8":
            return (top / 127.0).float().double().clamp(min=LEAST)
        e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e))
        return torch.exp2(e.clamp(min=-120.0))

    def written(b, a, n, x, X, scales):
        """What tokens a - a % R .. n - 1 of sequence b stand for after the new ones, x [n - a, Hkv, d], are in."""
        t0 = a - a % R
        old = torch.arange(t0, a, device="cuda")
        y = torch.cat([tokens_of(b, old, X, scales), x])
        y = torch.cat([y, y.new_zeros((-y.shape[0] % R, Hkv, d))]).reshape(-1, R, Hkv, d)
        fresh = y.clone()
        fresh[0, : a - t0] = 0.0                          # (those are there: their scale counts, not their size)
        sc = scale_of(fresh.abs().amax((1, 3)))
        if a > t0:
            was = s[scales].double()[int(s["table"][b, t0 // page]), :, t0 % page // R]
            sc[0] = torch.maximum(sc[0], was)
        return nearest(y, sc[:, None, :, None]).reshape(-1, Hkv, d)[: n - t0]

    if case["op"] in ("append", "read"):
        found = []
        row = 0
        for b, (n, m) in enumerate(zip(lens, new)):
            if case["op"] == "read":
                t = torch.arange(n - m, n, device="cuda")
                found.append([tokens_of(b, t, X, sc) for X, sc in (("K", "Ks"), ("V", "Vs"))])
                continue
            k, v = s["new"][row: row + m, Hq: Hq + Hkv].double(), s["new"][row: row + m, Hq + Hkv:].double()
            if case["rope"]:
                inv = BASE ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
                z = torch.complex(k[..., : d // 2], k[..., d // 2:]) * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.arange(
                    n - m, n, dtype=torch.float64, device="cuda")[:, None] * inv)[:, None]
                k = torch.cat([z.real, z.imag], -1)
            found.append([written(b, n - m, n, k, "K", "Ks"), written(b, n - m, n, v, "V", "Vs")])
            row += m
        sides = []
        for j in range(1 if case["keys"] else 2):
            x = torch.cat([f[j] for f in found])
            if case["heads"]:
                x = x.reshape(case["B"], case["new"], Hkv, d).transpose(1, 2)
            else:
                x = torch.cat([x, x.new_zeros((case["pad"], Hkv, d))])
            sides.append(x)
        return dict(zip(("K", "V"), sides))
    if sum(n * m for n, m in zip(lens, new)) * Hq * d > 3e11:
        return None
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        t = torch.arange(n, device="cuda")
        p = (n if case["behind"] else n - m) + torch.arange(m, device="cuda")
        hidden = t[None, :] > p[:, None]
        if case["window"]:
            hidden |= t[None, :] <= p[:, None] - case["window"]
        k, v = tokens_of(b, t, "K", "Ks"), tokens_of(b, t, "V", "Vs")
        for h in range(Hkv):
            kt, vh = k[:, h].t().contiguous(), v[:, h].contiguous()
            for j in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                x = torch.mm(s["Q"][row: row + m, j].double().contiguous(), kt) / math.sqrt(d)
                x[hidden] = float("-inf")
                L = torch.logsumexp(x, -1)
                w = torch.exp(x - torch.where(torch.isinf(L), 0.0, L)[:, None])
                out[row: row + m, j], lse[row: row + m, j] = torch.mm(w, vh), L
        row += m
    return {"out": out, "lse": lse}
