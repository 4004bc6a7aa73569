"""The paged 8-bit cache in plain numpy, 64 bits: rotary positions, growth of the cache, attention over it.

Written from the definitions; shares no code with the kernels or with the other oracles.  Where the definition rounds
(cosines and products of the rotation to fp32, codes to e4m3), so does this; everything else is fp64.
"""
import math

import numpy as np


# ---- e4m3: sign, four bits of exponent (bias 7), three of significand; no infinities; 0x7f and 0xff are NaN
def decode_e4m3(codes):
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c >> 7, -x, x)


_POSITIVE = decode_e4m3(np.arange(127))        # 0 .. 448, rising


def encode_e4m3(x):
    """Nearest code, ties to the even one; |x| <= 448.  NaN and infinities: 0x7f or 0xff."""
    x = np.asarray(x, np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    assert a.max(initial=0.0) <= 448.0
    above = np.minimum(np.searchsorted(_POSITIVE, a), 126)
    below = np.maximum(above - 1, 0)
    up, down = _POSITIVE[above] - a, a - _POSITIVE[below]
    code = np.where(up < down, above, np.where(down < up, below, np.where(above % 2 == 0, above, below)))
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def same_codes(a, b):
    """Equal codes; a NaN code equals either of them."""
    a, b = np.asarray(a, np.uint8), np.asarray(b, np.uint8)
    return (a == b) | ((a & 127 == 127) & (b & 127 == 127))


def scale_for(most):
    """The smallest power of two s >= 2^-100 with most <= 448 s."""
    s = 2.0 ** -100
    while most > 448.0 * s:
        s *= 2.0
    return s


# ---- rotation
def turn(x, positions, inv_freq, axis_of, pairs, backward=False):
    """x [tokens, heads, d] (any float type) turned, as fp32 before the rounding to x's type."""
    x = np.asarray(x, np.float32)
    half = len(inv_freq)
    angle = np.asarray(positions, np.float64)[np.asarray(axis_of)].T * np.asarray(inv_freq, np.float64)    # [tokens, half]
    c, s = np.cos(angle).astype(np.float32)[:, None, :], np.sin(angle).astype(np.float32)[:, None, :]
    if backward:
        s = -s
    one, two = (slice(0, half), slice(half, 2 * half)) if pairs == 0 else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    y = x.copy()
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., one] = x[..., one] * c - x[..., two] * s
        y[..., two] = x[..., two] * c + x[..., one] * s
    return y


# ---- the cache: dict(k, v: codes [pages, heads, page, d] both token by token; ks, vs: scales [pages, heads])
def append(codes, scale, x, table, seq_lens, q_start, max_new=1 << 30):
    """New rows x [tokens, heads, d] (fp32) into codes [pages, heads, page, d] and scale, in place, token group by token group."""
    n_pages, _, page, _ = codes.shape
    for b in range(len(seq_lens)):
        first, rows = int(q_start[b]), int(q_start[b + 1]) - int(q_start[b])
        pos0 = int(seq_lens[b]) - rows
        by_page = {}
        for i in range(min(rows, max_new)):
            if pos0 + i >= 0:
                by_page.setdefault((pos0 + i) // page, []).append(i)
        for index, rows_of in by_page.items():
            pid = int(table[b][index])
            if not 0 <= pid < n_pages:
                continue
            slots = [(pos0 + i) % page for i in rows_of]
            new = np.asarray(x[[first + i for i in rows_of]], np.float64)              # [rows, heads, d]
            for h in range(codes.shape[1]):
                finite = np.abs(new[:, h][np.isfinite(new[:, h])])
                s = scale_for(finite.max(initial=0.0))
                if 0 not in slots:
                    old = float(scale[pid, h])
                    if old >= s:
                        s = old
                    else:
                        codes[pid, h] = encode_e4m3(decode_e4m3(codes[pid, h]) * (old / s))
                scale[pid, h] = s
                codes[pid, h, slots] = encode_e4m3(new[:, h] / s)


def attend(q, kc, vc, ks, vs, table, seq_lens, q_start, causal=True, scale=None):
    """q [tokens, Hq, d]; returns out, lse in fp64 (rows behind the last sequence: NaN), and for error bounds the
    weighted mean of |v|, the largest |v| and the largest sum of |q k| * scale of every row."""
    q = np.asarray(q, np.float64)
    t, hq, d = q.shape
    n_pages, hk, page, _ = kc.shape
    g = hq // hk
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, lse = np.full((t, hq, d), np.nan), np.full((t, hq), np.nan)
    mean_v, most_v, reach = np.zeros((t, hq, d)), np.zeros((t, hq, d)), np.zeros((t, hq))
    for b in range(len(seq_lens)):
        first, rows, n = int(q_start[b]), int(q_start[b + 1]) - int(q_start[b]), int(seq_lens[b])
        tokens = np.array([j for j in range(n) if 0 <= int(table[b][j // page]) < n_pages], dtype=np.int64)
        pids = np.array([int(table[b][j // page]) for j in tokens], dtype=np.int64)
        for h in range(hk):
            k = decode_e4m3(kc[pids, h, tokens % page]) * ks[pids, h][:, None]
            v = decode_e4m3(vc[pids, h, tokens % page]) * vs[pids, h][:, None]
            for i in range(rows):
                seen = tokens <= n - rows + i if causal else np.ones(len(tokens), bool)
                for hh in range(h * g, h * g + g):
                    row = first + i
                    if not seen.any():
                        out[row, hh], lse[row, hh] = 0.0, -np.inf
                        continue
                    s = (k[seen] @ q[row, hh]) * scale
                    top = np.max(s)
                    w = np.exp(s - top)
                    out[row, hh], lse[row, hh] = (w @ v[seen]) / w.sum(), top + math.log(w.sum())
                    mean_v[row, hh], most_v[row, hh] = (w @ np.abs(v[seen])) / w.sum(), np.abs(v[seen]).max(axis=0)
                    reach[row, hh] = (np.abs(k[seen]) @ np.abs(q[row, hh])).max() * scale
    return out, lse, mean_v, most_v, reach
