"""The operators around a paged key/value cache, as cases that can be timed and compared with their plain forms.

A program that serves several sequences at once keeps their keys and values in pages.  Before a step it plans: which
sequences grow, which page every new token's key and value go to (`plan`).  In every layer it embeds the positions of the
step's queries and keys (`rope`), writes keys and values into the pages (`append`) and lets the new tokens attend to what
their sequence has cached (`attend`).  A memory pot is such a cache with one page per sequence.

With `own` false, `run` computes a case in elementary torch operations, in 32 bits (angles in 64); with `own` true it makes
the library's calls.  Lengths are a function of the case (`mix` seeds them), values of the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

SHARED = 0.8        # share of a query's variance that all queries of its head have in common


def _plan(name, B, page, W, mix, *, kind="mixed", longest=0, pad=0, tight=False):
    return dict(name=name, op="plan", B=B, page=page, W=W, mix=mix, kind=kind, longest=longest or page * W, pad=pad, tight=tight)


def _rope(name, tokens, Hq, Hkv, d, *, rot=0, layout="half", dtype="bf16", base=10000.0, scaling="plain", factor=1.0, context=8192,
          far=8192, inverse=False, pad=0):
    return dict(name=name, op="rope", tokens=tokens, Hq=Hq, Hkv=Hkv, d=d, rot=rot or d, layout=layout, dtype=dtype, base=base, scaling=scaling,
                factor=factor, context=context, far=far, inverse=inverse, pad=pad)


def _append(name, tokens, Hkv, d, page, n_pages, *, dtype="bf16", rope=True, rot=0, layout="half", pad=0, runs=1):
    return dict(name=name, op="append", tokens=tokens, Hkv=Hkv, d=d, page=page, n_pages=n_pages, dtype=dtype, rope=rope, rot=rot or d, layout=layout,
                base=500000.0, scaling="parts", factor=8.0, context=8192, far=131072, inverse=False, pad=pad, runs=runs)


def _attend(name, B, Hq, Hkv, d, page, shortest, longest, new, mix, *, dtype="bf16", window=0, behind=False, pad=0):
    """Sequences of shortest .. longest cached tokens, the new ones among them; `new` tokens each, or 1 .. -new where negative."""
    return dict(name=name, op="attend", B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, shortest=shortest, longest=longest, new=new, mix=mix, dtype=dtype,
                window=window, behind=behind, pad=pad)


def listed():
    return [
        # one decoding step of a few sequences: launch and host latency only
        _plan("plan_decode", 8, 16, 256, 1, kind="decode"),
        # a full scheduler step: chunks of prompts, decoding, finished, compressed and idle sequences side by side
        _plan("plan_step", 512, 64, 512, 2, kind="mixed", pad=37),
        # queries and keys of a decoding step
        _rope("rope_decode", 16, 32, 8, 128),
        # ... of a long chunk far into a long context, frequencies scaled by parts, neighbouring pairs
        _rope("rope_chunk", 8192, 32, 8, 128, layout="pairs", base=500000.0, scaling="parts", factor=8.0, context=8192, far=1000000),
        # one token per sequence of a batch, fp32 cache, part of the head embedded
        _append("append_decode_fp32", 67, 3, 64, 16, 900, dtype="fp32", rot=32, layout="pairs", runs=67),
        # a chunk of prompt tokens of several sequences
        _append("append_chunk", 16384, 8, 128, 64, 1024, pad=100, runs=5),
        # a decoding step over short caches
        _attend("attend_decode_short", 4, 32, 8, 128, 16, 200, 500, 1, 3),
        # a decoding step of a batch of uneven sequences
        _attend("attend_decode_batch", 64, 32, 8, 128, 64, 500, 8192, 1, 4),
        # a decoding step of one long sequence
        _attend("attend_decode_long", 1, 32, 8, 128, 256, 131072, 131072, 1, 5),
        # a chunk of 2048 tokens that fills a memory pot of 4096: the pot is the page
        _attend("attend_pot", 1, 32, 8, 128, 4096, 4096, 4096, 2048, 6),
        # a chunk deep into a long prompt
        _attend("attend_long_chunk", 1, 32, 8, 128, 128, 32768, 32768, 2048, 7),
        # ragged chunks, single tokens among them, odd pages, a sliding window, fp32
        _attend("attend_ragged_fp32", 5, 12, 3, 64, 37, 300, 3001, -701, 8, dtype="fp32", window=1024, pad=11),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(("attend", "rope", "append", "plan"), (55, 15, 15, 15))[0]
    dtype = rng.choices(("bf16", "fp32"), (75, 25))[0]
    d, Hkv, G = rng.choice((64, 128, 128)), rng.choice((1, 2, 3, 4, 8, 8)), rng.choice((1, 2, 3, 4, 4, 8))
    freq = dict(layout=rng.choice(("half", "pairs")), base=rng.choice((10000.0, 500000.0)), scaling=rng.choice(("plain", "linear", "ntk", "parts")),
                factor=rng.choice((2.0, 4.0, 8.0)), far=_log_int(rng, 4096, 1000000))
    rot = rng.choice((d, d, d // 2, d // 4, d - 2 * rng.randrange(1, 12)))
    if op == "plan":
        page = rng.choice((1, 16, 32, 64, 100, 256))
        W = _log_int(rng, 2, 512)
        case = _plan("", _log_int(rng, 1, 512), page, W, rng.randrange(1 << 30), kind=rng.choice(("decode", "mixed", "mixed")), longest=min(page * W, 32768),
                     pad=rng.choice((0, 0, 5, 300)), tight=rng.random() < 0.2)
    elif op == "rope":
        case = _rope("", _log_int(rng, 1, 8192), Hkv * G, Hkv, d, rot=rot, dtype=dtype if Hkv * G <= 16 else "bf16", inverse=rng.random() < 0.3,
                     pad=rng.choice((0, 0, 9)), **freq)
    elif op == "append":
        tokens, page = _log_int(rng, 1, 16384), rng.choice((16, 32, 64, 100, 256, 1000))
        case = _append("", tokens, Hkv, d, page, tokens // page + rng.randrange(tokens // 8 + 40) // page * 8 + 70, dtype=dtype if Hkv <= 4 else "bf16",
                       rope=rng.random() < 0.7, rot=rot, pad=rng.choice((0, 0, 33)), runs=rng.randrange(1, 33))
        case.update(freq)
    else:
        while True:
            decode = rng.random() < 0.45
            B, longest = _log_int(rng, 1, 64 if decode else 8), _log_int(rng, 100, 131072 if decode else 32768)
            new = rng.choice((1, 1, 1, 2, 5, -8)) if decode else rng.choice((-1, 1)) * _log_int(rng, 16, 2048)
            gathered, scores = B * longest * Hkv * d, B * longest * Hkv * G * abs(new)
            if gathered <= 64 * 8192 * 8 * 128 and scores <= (32768 * 32 * 2048 if dtype == "bf16" else 1 << 28) and abs(new) <= longest:
                break
        case = _attend("", B, Hkv * G, Hkv, d, rng.choice((16, 32, 37, 64, 100, 256, 4096)), max(1, int(longest * rng.random())), longest, new,
                       rng.randrange(1 << 30), dtype=dtype, window=_log_int(rng, 32, longest + 32) if rng.random() < 0.25 else 0,
                       behind=rng.random() < 0.15, pad=rng.choice((0, 0, 7)))
    del case["name"]
    return case


_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _plan_lengths(case):
    """Lengths before and after the step, and the pages of the pool."""
    rng = random.Random(case["mix"])
    before, after = [], []
    for _ in range(case["B"]):
        n = min(case["longest"] - 1, _log_int(rng, 1, case["longest"]))
        what = "decode" if case["kind"] == "decode" else rng.choice(("decode", "decode", "prompt", "chunk", "done", "shrunk", "idle"))
        m = {"decode": n + 1, "prompt": min(case["longest"], n), "chunk": min(case["longest"], n + _log_int(rng, 2, 512)), "done": 0,
             "shrunk": (n + 1) // 2, "idle": n}[what]
        before.append(0 if what == "prompt" else n)
        after.append(m)
    pages = lambda n: -(-n // case["page"])                                                   # noqa: E731
    held, need = sum(map(pages, before)), sum(max(0, pages(m) - pages(n)) for n, m in zip(before, after))
    return before, after, held + (need // 2 if case["tight"] else need + 3 * case["B"] + 7)


def _attend_lengths(case):
    """Cached tokens of every sequence, and how many of them are new (with `behind`: how many queries stand behind them)."""
    rng = random.Random(case["mix"])
    lens = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(case["B"])]
    lens[0] = case["longest"]
    new = [case["new"] if case["new"] > 0 else rng.choice((1, rng.randint(1, -case["new"]))) for _ in lens]
    return lens, [m if case["behind"] else min(m, n) for m, n in zip(new, lens)]


def _inv_freq(case):
    """Radians per position of the pairs, in 64 bits."""
    rot, base = case["rot"], case["base"]
    if case["scaling"] == "ntk" and rot > 2:
        base *= case["factor"] ** (rot / (rot - 2))
    f = base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "parts":          # pairs that turn often within the trained context keep their angle, slow ones are stretched
        keep = ((case["context"] * f / (2.0 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / case["factor"])
    return f


def _descriptor(ip, case, X, Y=None):
    return ip.make_rope(X, Y, rot=case["rot"], layout={"half": ip.CCD_ROPE_HALF, "pairs": ip.CCD_ROPE_PAIRS}[case["layout"]], base=case["base"],
                        scaling={"plain": ip.CCD_ROPE_PLAIN, "linear": ip.CCD_ROPE_LINEAR, "ntk": ip.CCD_ROPE_NTK, "parts": ip.CCD_ROPE_PARTS}[case["scaling"]],
                        factor=case["factor"], context=case["context"], low=1.0, high=4.0, inverse=case["inverse"])


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _prepare_plan(case, g):
    before, after, n_pages = _plan_lengths(case)
    B, page, W = case["B"], case["page"], case["W"]
    held = torch.tensor([-(-n // page) for n in before], device="cuda")
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    first = torch.cumsum(held, 0) - held
    col = torch.arange(W, device="cuda")[None, :]
    table = torch.where(col < held[:, None], ids[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32)
    used = int(held.sum())
    head = int(torch.randint(0, n_pages, (1,), generator=g, device="cuda"))
    ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(n_pages - used, device="cuda")) % n_pages] = ids[used:]
    tokens = sum(max(0, m - n) for n, m in zip(before, after)) + case["pad"]
    tokens = max(1, tokens)
    s = dict(before=_ints(before), after=_ints(after), table=table, ring=ring, cursor=_ints([head, n_pages - used, 0, 0]), page=page, n_pages=n_pages,
             table_next=torch.full_like(table, -7), cursor_next=_ints([0, 0, 0, 0]), q_start=_ints([0] * (B + 1)),
             slots=torch.zeros(tokens, dtype=torch.int32, device="cuda"), positions=torch.zeros(tokens, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2410_01518_amd import infinipot as ip
        s["paged"] = ip.make_plan(table, tokens=tokens, page=page, n_pages=n_pages)
    return s


def _positions(case, g):
    """Runs of neighbouring positions that start anywhere below `far`; the padding behind the step's tokens has -1."""
    tokens, runs = case["tokens"], case.get("runs", 3)
    i = torch.arange(tokens, device="cuda")
    start = torch.randint(0, max(1, case["far"] - tokens), (runs,), generator=g, device="cuda")
    pos = start[i * runs // tokens] + i - (i * runs // tokens * tokens + runs - 1) // runs
    return torch.cat([pos, pos.new_full((case["pad"],), -1)]).to(torch.int32)


def _prepare_rope(case, g):
    H, d, rows = case["Hq"] + case["Hkv"], case["d"], case["tokens"] + case["pad"]
    # queries, keys and values as one projection leaves them: the first Hq + Hkv heads of a token are embedded
    packed = torch.empty((rows, H + case["Hkv"], d), dtype=_DT[case["dtype"]], device="cuda").normal_(generator=g)
    s = dict(X=packed[:, :H], positions=_positions(case, g), Y=torch.zeros((rows, H, d), dtype=_DT[case["dtype"]], device="cuda"),
             inv=_inv_freq(case).cuda(), rot=case["rot"], layout=case["layout"], inverse=case["inverse"])
    if own:
        from paper_2410_01518_amd import infinipot as ip
        s["rope"] = _descriptor(ip, case, s["X"], s["Y"])
        s["turns"] = ip.rope_turns(s["rope"])
    return s


def _prepare_append(case, g):
    Hkv, d, page, n_pages, T = case["Hkv"], case["d"], case["page"], case["n_pages"], case["tokens"]
    dt = _DT[case["dtype"]]
    new = torch.empty((T + case["pad"], 2, Hkv, d), dtype=dt, device="cuda").normal_(generator=g)
    # neighbouring tokens stand in neighbouring rows of a page, runs of them anywhere
    runs = min(case["runs"], T)
    i = torch.arange(T, device="cuda")
    run = i * runs // T
    off = i - (run * T + runs - 1) // runs
    per = -(-(-(-T // runs)) // page) + 1
    total = max(n_pages, runs * per)
    ids = torch.randperm(total, generator=g, device="cuda")
    at = off + torch.randint(0, page, (runs,), generator=g, device="cuda")[run]
    slots = ids[run * per + at // page] * page + at % page
    s = dict(K_new=new[:, 0], V_new=new[:, 1], slots=torch.cat([slots, slots.new_full((case["pad"],), -1)]).to(torch.int32),
             positions=_positions(case, g), K=torch.zeros((total, Hkv, page, d), dtype=dt, device="cuda"), inv=_inv_freq(case).cuda(),
             V=torch.zeros((total, Hkv, page, d), dtype=dt, device="cuda"), rope=case["rope"], rot=case["rot"], layout=case["layout"], inverse=False)
    if own:
        from paper_2410_01518_amd import infinipot as ip
        s["paged"] = ip.make_paged(s["K"], tokens=T + case["pad"], K_new=s["K_new"])
        s["descriptor"] = _descriptor(ip, case, s["K_new"]) if case["rope"] else None
        s["turns"] = ip.rope_turns(s["descriptor"]) if case["rope"] else None
    return s


def _prepare_attend(case, g):
    lens, new = _attend_lengths(case)
    B, Hq, Hkv, d, page = case["B"], case["Hq"], case["Hkv"], case["d"], case["page"]
    dt, T = _DT[case["dtype"]], sum(new)
    W = -(-max(lens) // page)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    held = torch.tensor(need, device="cuda")
    col = torch.arange(W, device="cuda")[None, :]
    first = torch.cumsum(held, 0) - held
    table = torch.where(col < held[:, None], ids[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32)
    K = torch.empty((n_pages, Hkv, page, d), dtype=dt, device="cuda").normal_(generator=g)
    # one key in a hundred is four times as long (attention sinks and other outliers)
    K *= torch.where(torch.rand((n_pages, 1, page, 1), generator=g, device="cuda") < 0.01, 4.0, 1.0).to(dt)
    V = torch.empty_like(K).normal_(generator=g)
    head = torch.randn((Hkv, 1, d), generator=g, device="cuda").expand(Hkv, Hq // Hkv, d).reshape(1, Hq, d)
    Q = (math.sqrt(SHARED) * head + math.sqrt(1.0 - SHARED) * torch.randn((T + case["pad"], Hq, d), generator=g, device="cuda")).to(dt)
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    s = dict(Q=Q, K=K, V=V, table=table, q_start=_ints(starts), lens=_ints(lens), out=torch.zeros_like(Q), page=page, max_len=max(lens), max_new=max(new),
             lse=torch.zeros((T + case["pad"], Hq), dtype=torch.float32, device="cuda"), window=case["window"], behind=case["behind"])
    if own:
        from paper_2410_01518_amd import infinipot as ip
        s["paged"] = ip.make_paged(K, tokens=T + case["pad"], block_table=table, Q=Q, out=s["out"], lse=s["lse"], window=case["window"],
                                   behind=case["behind"], max_new=max(new), max_len=max(lens))
        s["ws"] = ip.alloc_paged_workspace(s["paged"])
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"plan": _prepare_plan, "rope": _prepare_rope, "append": _prepare_append, "attend": _prepare_attend}[case["op"]](case, g)
    s["op"] = case["op"]
    return s


def _plain_plan(s):
    page, n_pages, table = s["page"], s["n_pages"], s["table"].long()
    W = table.shape[1]
    before, after = s["before"].long().clamp(min=0), s["after"].long().clamp(min=0)
    head, count = s["cursor"][0].long(), s["cursor"][1].long()
    p0 = ((before + page - 1) // page).clamp(max=W)
    wanted = (after + page - 1) // page
    p1 = wanted.clamp(max=W)
    need = (p1 - p0).clamp(min=0)
    col = torch.arange(W, device=table.device)[None, :]
    rank = (torch.cumsum(need, 0) - need)[:, None] + col - p0[:, None]
    kept = torch.where(col < torch.minimum(p0, p1)[:, None], table, -1)
    got = (col >= p0[:, None]) & (col < p1[:, None]) & (rank < count)
    nxt = torch.where(got, s["ring"].long()[(head + rank) % n_pages], kept)
    gone = table[(col >= p1[:, None]) & (col < p0[:, None]) & (table >= 0) & (table < n_pages)]
    ring = s["ring"].clone()
    ring[(head + count + torch.arange(gone.numel(), device=table.device)) % n_pages] = gone.to(torch.int32)
    taken = torch.minimum(need.sum(), count)
    short = need.sum() - taken + (wanted - p1).sum()
    cursor = torch.stack([(head + taken) % n_pages, count - taken + gone.numel(), short, torch.zeros_like(short)])
    added = (after - before).clamp(min=0)
    ends = torch.cumsum(added, 0)
    i = torch.arange(s["slots"].numel(), device=table.device)
    b = torch.searchsorted(ends, i, right=True).clamp(max=table.shape[0] - 1)
    pos = before[b] + i - (ends - added)[b]
    inside = i < ends[-1]
    where = pos // page
    page_id = nxt[b, where.clamp(max=W - 1)]
    there = inside & (where < W) & (page_id >= 0) & (page_id < n_pages)
    slots = torch.where(there, page_id * page + pos % page, -1)
    q_start = torch.cat([torch.zeros_like(ends[:1]), ends])
    return [x.to(torch.int32) for x in (nxt, ring, cursor, q_start, slots, torch.where(inside, pos, -1))]


def _plain_rotation(s, X):
    """X [tokens, heads, d] with the first `rot` elements turned by their position, in 32 bits."""
    x, rot = X.float(), s["rot"]
    angle = s["positions"].double()[:, None] * s["inv"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if s["inverse"]:
        sin = -sin
    if s["layout"] == "half":
        u, v = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    else:
        u, v = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope(s):
    here = (s["positions"] >= 0)[:, None, None]
    s["Y"].copy_(torch.where(here, _plain_rotation(s, s["X"]).to(s["Y"].dtype), s["Y"]))
    return s["Y"]


def _plain_append(s):
    here = s["slots"] >= 0
    slots, page = s["slots"][here].long(), s["K"].shape[2]
    keys = _plain_rotation(s, s["K_new"]).to(s["K"].dtype) if s["rope"] else s["K_new"]
    s["K"][slots // page, :, slots % page] = keys[here]
    s["V"][slots // page, :, slots % page] = s["V_new"][here]


def _plain_attend(s):
    Q, page, N, M = s["Q"], s["page"], s["max_len"], s["max_new"]
    T, Hq, d = Q.shape
    Hkv = s["K"].shape[1]
    B, dev = s["lens"].numel(), Q.device
    t = torch.arange(N, device=dev)
    pages = s["table"][:, t // page].long().clamp(min=0)                                             # [B, N]
    k = s["K"][pages, :, t % page].float().permute(0, 2, 3, 1).contiguous()                          # [B, Hkv, d, N]
    v = s["V"][pages, :, t % page].float().transpose(1, 2).contiguous()                              # [B, Hkv, N, d]
    start, count = s["q_start"][:-1].long(), (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(M, device=dev)
    rows = (start[:, None] + i).clamp(max=T - 1)
    q = Q[rows].float().reshape(B, M, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * M, d).contiguous()
    x = torch.matmul(q, k).reshape(B, Hkv, Hq // Hkv, M, N) * (1.0 / math.sqrt(d))
    lens = s["lens"].long()
    pos = (lens if s["behind"] else lens - count)[:, None] + i                                       # [B, M]
    seen = (t <= pos[..., None]) & (t < lens[:, None, None])
    if s["window"] > 0:
        seen &= t > pos[..., None] - s["window"]
    x = x.masked_fill(~seen[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.reshape(B, Hkv, Hq // Hkv * M, N), v).reshape(B, Hkv, Hq // Hkv, M, d) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(-1)                                                       # an empty row: -inf
    mine = i < count[:, None]
    to = rows[mine]
    s["out"][to] = o.permute(0, 3, 1, 2, 4).reshape(B, M, Hq, d)[mine].to(Q.dtype)
    s["lse"][to] = lse.permute(0, 3, 1, 2).reshape(B, M, Hq)[mine]


def _bits(t):
    """Values are copied: their bit patterns are compared as whole numbers."""
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


def run(s):
    op = s["op"]
    if not own:
        if op == "plan":
            return dict(zip(("table", "ring", "cursor", "q_start", "slots", "positions"), _plain_plan(s)))
        if op == "rope":
            return _plain_rope(s)
        if op == "append":
            _plain_append(s)
        else:
            _plain_attend(s)
    else:
        from paper_2410_01518_amd import infinipot as ip
        if op == "plan":
            ip.ccd_paged_plan(s["paged"], s["before"], s["after"], s["table"], s["table_next"], s["ring"], s["cursor"], s["cursor_next"], s["q_start"],
                              s["slots"], s["positions"])
            return {"table": s["table_next"], "ring": s["ring"], "cursor": s["cursor_next"], "q_start": s["q_start"], "slots": s["slots"],
                    "positions": s["positions"]}
        if op == "rope":
            ip.ccd_rope(s["rope"], s["X"], s["positions"], s["turns"], s["Y"])
            return s["Y"]
        if op == "append":
            ip.ccd_paged_append(s["paged"], s["K_new"], s["V_new"], s["slots"], s["K"], s["V"], rope=s["descriptor"], positions=s["positions"],
                                turns=s["turns"])
        else:
            ip.ccd_paged_attend(s["paged"], s["Q"], s["K"], s["V"], s["table"], s["q_start"], s["lens"], s["out"], s["lse"], s["ws"])
    if op == "append":
        return {"K": s["K"] if s["rope"] else _bits(s["K"]), "V": _bits(s["V"])}
    return {"out": s["out"], "lse": s["lse"]}


def work(case):
    """plan: lengths and table read, table, slots and positions written.  rope, append: the tokens' rows read and written.  attend: queries and the
    visible keys and values read, outputs and log-sum-exps written; two products per visible pair."""
    if case["op"] == "plan":
        before, after, _ = _plan_lengths(case)
        tokens = sum(max(0, m - n) for n, m in zip(before, after)) + case["pad"]
        return {"bytes": 8 * case["B"] * case["W"] + 12 * case["B"] + 8 * tokens, "flops": 0}
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        elements = case["tokens"] * (case["Hq"] + case["Hkv"]) * case["d"]
        return {"bytes": 2 * e * elements + 4 * case["tokens"], "flops": 3 * elements}
    if case["op"] == "append":
        elements = case["tokens"] * case["Hkv"] * case["d"]
        return {"bytes": 4 * e * elements + 8 * case["tokens"], "flops": 3 * elements if case["rope"] else 0}
    lens, new = _attend_lengths(case)
    pairs, tokens = 0, 0
    for n, m in zip(lens, new):
        p = n if case["behind"] else n - m
        low = 0 if not case["window"] else max(0, min(n, p - case["window"] + 1))
        tokens += max(0, n - low)
        for i in range(m):
            first = max(0, p + i - case["window"] + 1) if case["window"] else 0
            pairs += max(0, min(n, p + i + 1) - first)
    rows = sum(new) * case["Hq"]
    return {"bytes": 2 * e * tokens * case["Hkv"] * case["d"] + rows * (2 * e * case["d"] + 4), "flops": 4 * case["d"] * case["Hq"] * pairs}


def exact(case, seed):
    """In 64 bits, sequence by sequence and head by head; the whole numbers of a plan have no such value."""
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)

    def turned(X):
        rot, dev = case["rot"], X.device
        inv = _inv_freq(case).to(dev)
        z = torch.polar(torch.ones((), dtype=torch.float64, device=dev), (-1.0 if case["inverse"] else 1.0) * s["positions"].double()[:, None] * inv)
        y = X.double()
        first = torch.arange(rot // 2, device=dev) * (2 if case["layout"] == "pairs" else 1)
        second = first + (1 if case["layout"] == "pairs" else rot // 2)
        w = torch.complex(y[..., first], y[..., second]) * z[:, None]
        y = y.clone()
        y[..., first], y[..., second] = w.real, w.imag
        return y

    if case["op"] == "rope":
        y = turned(s["X"])
        y[case["tokens"]:] = 0.0
        return y
    if case["op"] == "append":
        T, page = case["tokens"], case["page"]
        to = s["slots"][:T].long()
        K = None
        if case["rope"]:
            K = torch.zeros(s["K"].shape, dtype=torch.float64, device="cuda")
            K[to // page, :, to % page] = turned(s["K_new"])[:T]
        return {"K": K, "V": None}
    lens, new = _attend_lengths(case)
    if sum(n * m for n, m in zip(lens, new)) * case["Hq"] * case["d"] > 3e11:
        return None
    Hq, Hkv, d, page = case["Hq"], case["Hkv"], case["d"], case["page"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        t = torch.arange(n, device="cuda")
        ids = s["table"][b].long()[t // page]
        p = (n if case["behind"] else n - m) + torch.arange(m, device="cuda")
        hidden = t[None, :] > p[:, None]
        if case["window"]:
            hidden |= t[None, :] <= p[:, None] - case["window"]
        for h in range(Hkv):
            k, v = s["K"][ids, h, t % page].double(), s["V"][ids, h, t % page].double()
            kt = k.t().contiguous()
            for j in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                x = torch.mm(s["Q"][row: row + m, j].double().contiguous(), kt) / math.sqrt(d)
                x[hidden] = float("-inf")
                L = torch.logsumexp(x, -1)
                w = torch.exp(x - torch.where(torch.isinf(L), 0.0, L)[:, None])
                out[row: row + m, j], lse[row: row + m, j] = torch.mm(w, v), L
        row += m
    return {"out": out, "lse": lse}
