"""Plain statements, in 64 bits unless a rounding is part of the definition, of the rotation, the page plan, the rows held in 4
bits and the attention over them (test infrastructure; shares nothing with the library)."""
import numpy as np
import torch

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def frequencies(rotary, base=10000.0):
    return base ** (-2.0 * np.arange(rotary // 2) / rotary)


def rotate(x, pos, freq, scale=1.0, layout="halves", inverse=False, single=False):
    """x [..., n, d], pos [..., n].  `single`: cosines, sines, products and sums rounded to fp32 as the library documents it."""
    r = 2 * len(freq)
    ang = np.asarray(pos, np.longdouble)[..., None] * np.asarray(freq, np.longdouble)
    ang = np.remainder(ang, 2 * np.pi * np.ones(1, np.longdouble)) if np.max(np.abs(ang), initial=0) > 1e15 else ang
    t = np.float32 if single else np.float64
    c, s = (np.cos(ang) * scale).astype(t), (np.sin(ang) * (-scale if inverse else scale)).astype(t)
    x = np.asarray(x, t)
    y = x.copy()
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if layout == "halves" else (x[..., 0:r:2], x[..., 1:r:2])
    ya, yb = a * c - b * s, b * c + a * s
    if layout == "halves":
        y[..., :r // 2], y[..., r // 2:r] = ya, yb
    else:
        y[..., 0:r:2], y[..., 1:r:2] = ya, yb
    return y


def scale_value(byte):
    byte = np.asarray(byte, np.int64)
    e, m = byte >> 3, byte & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 15.0), m * 2.0 ** -17)
    return np.where(byte >= 0xf8, np.where(byte == 0xf8, np.inf, np.nan), v)


def nearest_scale(a):
    """Byte of the scale nearest to a / 6 (ties to even), a finite and >= 0."""
    q = (np.minimum(np.asarray(a, np.float32), np.float32(61440)) / np.float32(6)).astype(np.float64)
    all_bytes = np.arange(0xf8)
    values = scale_value(all_bytes)
    hi = np.searchsorted(values, q).clip(1, len(values) - 1)
    lo = hi - 1
    dl, dh = q - values[lo], values[hi] - q
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return pick


def quantise(x):
    """x float64 [..., d] -> (codes [..., d], scale bytes [..., d / 16])."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    nan = np.isnan(g).any(-1)
    a = np.minimum(np.nan_to_num(np.abs(g), nan=0.0, posinf=np.inf), 61440.0).max(-1)
    byte = nearest_scale(a)
    s = scale_value(byte)[..., None]
    y = np.where(s > 0, np.minimum(np.nan_to_num(np.abs(g), nan=0.0, posinf=np.inf), 61440.0) / np.where(s > 0, s, 1), 0)
    hi = np.searchsorted(LEVELS, y).clip(1, 7)
    lo = hi - 1
    dl, dh = y - LEVELS[lo], LEVELS[hi] - y
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = code + 8 * np.signbit(g)
    code = np.where(nan[..., None], 0, code)
    return code.reshape(x.shape), np.where(nan, 0xff, byte)


def value(code, byte):
    sign = np.where(code >= 8, -1.0, 1.0)
    v = sign * LEVELS[code & 7]
    return (v.reshape(*code.shape[:-1], code.shape[-1] // 16, 16) * scale_value(byte)[..., None]).reshape(code.shape)


def row_bytes(d):
    return {64: 80, 128: 144}[d]


def pack(k, v):
    """uint8 [..., row bytes] of float64 k, v [..., d]."""
    d = k.shape[-1]
    parts = []
    scales = []
    for x in (k, v):
        code, byte = quantise(x)
        parts.append((code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8))
        scales.append(byte.astype(np.uint8))
    row = np.concatenate(parts + scales, -1)
    return np.concatenate([row, np.zeros((*row.shape[:-1], row_bytes(d) - row.shape[-1]), np.uint8)], -1)


def unpack(rows, d):
    h, g = d // 2, d // 16
    out = []
    for first, sc in ((0, 2 * h), (h, 2 * h + g)):
        b = rows[..., first:first + h].astype(np.int64)
        code = np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], d)
        out.append(value(code, rows[..., sc:sc + g]))
    return out


def plan(table, length, n_new, free, free_count, page, max_tokens):
    """One request after the other."""
    table = table.copy()
    B, max_pages = table.shape
    cu = [0]
    start, new_length = [], []
    pos, slot = np.full(max_tokens, -1), np.full(max_tokens, -1)
    left = max(0, min(int(free_count), len(free)))
    wanted = 0
    room = left
    for b in range(B):
        n, had = int(n_new[b]), int(length[b])
        at = cu[-1]
        cu.append(at + max(n, 0))
        fits = n >= 0 and had >= 0 and had + n <= max_pages * page and at + n <= max_tokens
        held = -(-had // page)
        need = -(-(had + n) // page) - held if fits else 0
        wanted += need
        if not fits or (need > 0 and wanted > room):
            start.append(-1)
            new_length.append(had)
            continue
        for i in range(need):
            left -= 1
            table[b, held + i] = free[left]
        start.append(had)
        new_length.append(had + n)
        for j in range(n):
            r = had + j
            pos[at + j] = r
            slot[at + j] = table[b, r // page] * page + r % page if table[b, r // page] >= 0 else -1
    return np.array(start), np.array(new_length), left, np.array(cu), pos, slot, table


def attend(q, k, v, seen, bias=0.0):
    """q [V, d], k, v [n, d] float64, seen [V, n] -> (o [V, d], what an output's error is measured by: sum p |v| / sum p [V, d],
    the largest sum |q_i k_i| / sqrt(d) of a vector's rows [V], the largest |v| of a row that is seen [V])."""
    d = q.shape[-1]
    with np.errstate(invalid="ignore", over="ignore"):
        a = q @ k.T / np.sqrt(d) + bias
        a = np.where(seen, a, -np.inf)
        top = np.max(a, -1, keepdims=True, initial=-np.inf)
        p = np.where(seen, np.exp(a - np.where(np.isinf(top), 0, top)), 0.0)
        den = p.sum(-1, keepdims=True)
        o, size = np.zeros(q.shape), np.zeros(q.shape)
        for i in range(len(q)):
            if den[i, 0] != 0 and seen[i].any():
                o[i] = (p[i, seen[i]] / den[i]) @ v[seen[i]]
                size[i] = (p[i, seen[i]] / den[i]) @ np.abs(v[seen[i]])
        reach = np.max(np.where(seen, np.abs(q) @ np.abs(k).T / np.sqrt(d), 0.0), -1, initial=0.0)
        most = np.max(np.where(seen, np.nan_to_num(np.abs(v)).max(-1, initial=0.0), 0.0), -1, initial=0.0)
    return o, size, reach, most


def attend_bound(o, size, reach, most, dtype, n):
    """How far an output may be off.
    A logit: fp32 sums that the matrix instruction cuts instead of rounding (2^-23 of the largest partial sum for each of up to 16
    instructions, whose 16 products are added the same way): 2^-18 reach; with fp32 queries their two fp16 parts add 2^-22.  An error
    of x in the logits moves a ratio of sums by 2 x at most.  Probabilities: exp2 2^-21; in fp16 half a step is 2^-11, in two parts
    2^-22.  fp16's smallest step is 2^-24 and the running reference's own probability is 2^8 (it was some row's, so the denominator is
    at least that): however small a probability is, it is off by at most half of that step, 2^-33 of the denominator, times its value:
    n 2^-33 most in all.  Sums of the values: cut again, 2^-23 for each of n / 16 instructions with bf16 outputs, 2^-24 for each of
    n / 32 + 600 additions and 2^-21 in a tile with fp32 ones.  The output's own rounding: 2^-8 or 2^-24."""
    rel = 2 * 2.0 ** -18 * reach[:, None] + 2.0 ** -20
    if dtype == torch.bfloat16:
        return (rel + 2 * 2.0 ** -11 + n / 16 * 2.0 ** -23) * size + n * 2.0 ** -33 * most[:, None] + 2.0 ** -8 * np.abs(o)
    return (rel + 2 * 2.0 ** -22 + (n / 32 + 600) * 2.0 ** -24 + 2.0 ** -21) * size + n * 2.0 ** -33 * most[:, None] + 2.0 ** -24 * np.abs(o)
