"""Plain numpy reference (64 bits) of the paged cache's operators: the plan of a step, rotary positions, writing new rows, attention.

Test infrastructure only; shares no code with the library.  Written from the definitions, one loop per thing that is counted.
"""
import math

import numpy as np


def plan(before, after, table, ring, cursor, *, page, n_pages, tokens):
    """(table, ring, cursor, q_start, slots, positions) after the step; nothing passed in is changed."""
    table, out, ring = table.copy(), np.full_like(table, -1), ring.copy()
    B, W = table.shape
    head, count = int(cursor[0]), int(cursor[1])
    free = [(head + i) % n_pages for i in range(count)]
    next_free, missing, back = 0, 0, []
    q_start, slots, positions = [0], np.full(tokens, -1, np.int32), np.full(tokens, -1, np.int32)
    for b in range(B):
        l0, l1 = max(0, int(before[b])), max(0, int(after[b]))
        want = -(-l1 // page)
        p0, p1 = min(W, -(-l0 // page)), min(W, want)
        missing += want - p1
        out[b, :min(p0, p1)] = table[b, :min(p0, p1)]
        for c in range(p0, p1):
            if next_free < count:
                out[b, c] = ring[free[next_free]]
                next_free += 1
            else:
                missing += 1
        back += [int(x) for x in table[b, p1:p0] if 0 <= x < n_pages]
        for pos in range(l0, l1):
            i = q_start[-1] + pos - l0
            if i < tokens:
                c = pos // page
                page_id = out[b, c] if c < W else -1
                positions[i] = pos
                slots[i] = page_id * page + pos % page if 0 <= page_id < n_pages else -1
        q_start.append(q_start[-1] + max(0, l1 - l0))
    for i, page_id in enumerate(back):
        ring[(head + count + i) % n_pages] = page_id
    moved = [(head + next_free) % n_pages, count - next_free + len(back), missing, 0]
    return out, ring, np.array(moved, np.int32), np.array(q_start, np.int32), slots, positions


def frequencies(rot, base, scaling="plain", factor=1.0, context=0, low=1.0, high=4.0):
    """Radians per position of every pair."""
    f = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" and rot > 2 else base
        w = b ** (-2.0 * i / rot)
        if scaling == "linear":
            w /= factor
        if scaling == "parts":
            turns = context * w / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            w = w * keep + w / factor * (1.0 - keep)
        f.append(w)
    return np.array(f)


def rope(x, positions, f, *, half, inverse=False, amplitude=1.0):
    """x [tokens, heads, d] in 64 bits; the first 2 len(f) elements are turned."""
    y, n = x.astype(np.float64).copy(), len(f)
    for t, p in enumerate(positions):
        ang = float(p) * f * (-1.0 if inverse else 1.0)
        c, s = np.cos(ang), np.sin(ang)
        one, two = (np.arange(n), np.arange(n) + n) if half else (2 * np.arange(n), 2 * np.arange(n) + 1)
        u, v = x[t][:, one].astype(np.float64), x[t][:, two].astype(np.float64)
        y[t][:, one] = amplitude * (u * c - v * s)
        y[t][:, two] = amplitude * (v * c + u * s)
    return y


def attend(q, K, V, table, q_start, kv_len, *, window=0, behind=False, scale=0.0):
    """q [tokens, Hq, d], K and V [n_pages, Hkv, page, d], all in 64 bits.  Returns (out, lse, size, logit_size): `size` is
    sum_t w_t |v_t| / sum_t w_t, `logit_size` the largest scale * sum_e |q_e k_te| of the row's visible tokens; rows of no sequence NaN."""
    T, Hq, d = q.shape
    n_pages, Hkv, page, _ = K.shape
    scale = scale or 1.0 / math.sqrt(d)
    out, size = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, logit_size = np.full((T, Hq), np.nan), np.full((T, Hq), np.nan)
    for b in range(len(kv_len)):
        m = int(q_start[b + 1]) - int(q_start[b])
        n = min(max(0, int(kv_len[b])), table.shape[1] * page)
        t = np.arange(n)
        ids = table[b][t // page] if n else np.zeros(0, int)
        there = (ids >= 0) & (ids < n_pages)
        t, ids = t[there], ids[there]
        for i in range(m):
            r = int(q_start[b]) + i
            if r >= T:
                continue
            p = (n if behind else n - m) + i
            see = (t <= p) & ((t > p - window) if window else True)
            for h in range(Hq):
                k, v = K[ids[see], h // (Hq // Hkv), t[see] % page], V[ids[see], h // (Hq // Hkv), t[see] % page]
                if not len(k):
                    out[r, h], size[r, h], lse[r, h], logit_size[r, h] = 0.0, 0.0, -np.inf, 0.0
                    continue
                x = scale * (k @ q[r, h])
                top = x.max()
                w = np.exp(x - top)
                out[r, h], size[r, h] = w @ v / w.sum(), w @ np.abs(v) / w.sum()
                lse[r, h] = top + math.log(w.sum())
                logit_size[r, h] = (scale * (np.abs(k) @ np.abs(q[r, h]))).max()
    return out, lse, size, logit_size
