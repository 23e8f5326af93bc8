"""Plain numpy reference (64 bits) of the caches in 8 bits: what codes stand for, scales, writing with blocks that grow, reading back, compaction.

Test infrastructure only; shares no code with the library.  Codes are uint8 arrays [n_pages, Hkv, page, d], scales [n_pages, Hkv, page / rows].
"""
import math

import numpy as np

LEAST = 2.0 ** -120

# the numbers that the 256 codes of either kind stand for
INT8 = np.array([c - 256 if c > 127 else c for c in range(256)], np.float64)
E4M3 = np.array([(-1.0 if c > 127 else 1.0) * (math.nan if c & 127 == 127 else (c & 7) * 2.0 ** -9 if c & 120 == 0 else
                                               (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10)) for c in range(256)])
NUMBERS = {"int8": INT8, "e4m3": E4M3}


def decode(codes, scales, kind, rows):
    with np.errstate(invalid="ignore"):
        return NUMBERS[kind][codes] * np.repeat(scales.astype(np.float64), rows, axis=2)[..., None]


def scale_for(x, kind):
    """Of all finite elements of x."""
    x = np.abs(x[np.isfinite(x)])
    top = x.max() if x.size else 0.0
    if kind == "int8":
        return max(float(np.float32(top / 127.0)), LEAST)
    s = LEAST
    while 448.0 * s < top:
        s *= 2.0
    return s


def encode(x, scale, kind):
    """Nearest code, halves to even ones; an element that is no finite number: NaN (e4m3), 0 (int8)."""
    x = np.asarray(x, np.float64)
    y = np.where(np.isfinite(x), x, 0.0) / scale
    if kind == "int8":
        return np.rint(y).astype(np.int64).astype(np.uint8)
    # between two neighbouring numbers: the nearer one, or the one whose code is even
    pos = E4M3[:127]                                      # 0 .. 448, ascending
    a = np.minimum(np.abs(y), 448.0)
    lo = np.clip(np.searchsorted(pos, a, side="right") - 1, 0, 125)
    up = a - pos[lo] > pos[lo + 1] - a
    tie = a - pos[lo] == pos[lo + 1] - a
    c = lo + np.where(tie, lo % 2, up)
    c = np.where(a == pos[lo], lo, c)
    return np.where(np.isfinite(x), c + np.where(np.signbit(y), 128, 0), 0x7F).astype(np.uint8)


def own_scale(s):
    """A block's scale as it was found: the power of two at or above it, 2^120 at most; 0 where it is negative or no number."""
    return min(2.0 ** math.ceil(math.log2(s)), 2.0 ** 120) if math.isfinite(s) and s > 0.0 else 0.0


def append(x, slots, codes, scales, kind, rows):
    """x [tokens, Hkv, d] (64 bits) to the rows of slots (negative or outside: not written), changing codes and scales.  Returns nothing."""
    n_pages, Hkv, page, _ = codes.shape
    blocks = {}
    for t, s in enumerate(slots):
        if 0 <= s < page * n_pages:
            blocks.setdefault(int(s) // rows, []).append((int(s) % rows, t))
    for block, new in blocks.items():
        p, j = block // (page // rows), block % (page // rows)
        first = min(r for r, _ in new)
        for h in range(Hkv):
            fresh = np.stack([x[t, h] for _, t in new])
            need, old = scale_for(fresh, kind), scales[p, h, j]
            s = need if first == 0 else max(own_scale(float(old)), need)
            if first > 0 and s != old:
                r = slice(j * rows, j * rows + first)
                with np.errstate(over="ignore", invalid="ignore"):
                    was = NUMBERS[kind][codes[p, h, r]].astype(np.float32) * old            # (what the rows read as, in fp32)
                codes[p, h, r] = encode(was, s, kind)
            for r, t in new:
                codes[p, h, j * rows + r] = encode(x[t, h], s, kind)
            scales[p, h, j] = math.nan if kind == "int8" and not np.isfinite(fresh).all() else s


def read(values, table, q_start, kv_len):
    """The last q_start[b + 1] - q_start[b] tokens of every sequence, values [n_pages, Hkv, page, d]; 0 where there is none.  Rows of no sequence: NaN."""
    n_pages, Hkv, page, d = values.shape
    out = np.full((int(q_start[-1]), Hkv, d), np.nan)
    for b in range(len(kv_len)):
        m = int(q_start[b + 1]) - int(q_start[b])
        n = min(max(0, int(kv_len[b])), table.shape[1] * page)
        for i in range(m):
            t = n - m + i
            p = table[b, t // page] if t >= 0 else -1
            out[int(q_start[b]) + i] = values[p, :, t % page] if 0 <= p < n_pages else 0.0
    return out


def compact(x, keep):
    """Rows keep[page, head] to the front of x [n_pages, Hkv, page, ...]; returns the result."""
    y = x.copy()
    for p in range(x.shape[0]):
        for h in range(x.shape[1]):
            y[p, h, : keep.shape[2]] = x[p, h, keep[p, h]]
    return y
