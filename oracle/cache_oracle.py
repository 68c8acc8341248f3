"""Plain 64-bit implementations of the paged cache's operators (vla_cache.h), one environment, row and head at a time."""
import math

import numpy as np

PAGE = 16


def _pages(n):
    return (n + PAGE - 1) // PAGE


def kv_plan(cached, new, table, free, n_pages, max_rows, head=0):
    """The step's outputs by name, and the page table after it (a copy)."""
    table = np.array(table, dtype=np.int64, copy=True)
    n, max_pages = table.shape
    lens, start, refused = [], [0], 0
    pos, env, slot = np.zeros(max_rows, np.int64), np.full(max_rows, -1), np.full(max_rows, -1)
    at = head
    left = len(free) - head if 0 <= head <= len(free) else 0
    asked = taken = rows = 0  # pages asked for by environments that fit, served or not; pages given; rows so far
    for e in range(n):
        c, w = int(cached[e]), int(new[e])
        end = rows + max(w, 0)
        fits = c >= 0 and w >= 0 and c + w <= PAGE * max_pages and end <= max_rows
        need = _pages(c + w) - _pages(c) if fits else 0
        asked += need
        ok = fits and (need == 0 or asked <= left)
        first = at + asked - need
        if ok:
            for i in range(need):
                table[e, _pages(c) + i] = free[first + i]
            taken = max(taken, asked) if need else taken
        for r in range(rows, min(end, max_rows)):
            p = c + r - rows
            pos[r], env[r] = min(max(p, 0), 2 ** 31 - 1), e
            if ok and 0 <= table[e, p // PAGE] < n_pages:
                slot[r] = table[e, p // PAGE] * PAGE + p % PAGE
        lens.append(c + w if ok else max(c, 0))
        refused += not ok
        rows = end
        start.append(min(rows, max_rows))
    return {"lens": np.array(lens, np.int64), "row_start": np.array(start), "row_pos": pos, "row_env": env, "row_slot": slot,
            "stats": np.array([head + taken, start[-1], refused])}, table


def rope_freqs(rot_dim, base=10000.0, scaling="none", factor=1.0, low=1.0, high=4.0, context=8192.0):
    """(radians per position [rot_dim / 2], factor on cos and sin)."""
    if scaling == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    out = []
    for i in range(rot_dim // 2):
        f = 1.0 / base ** (2 * i / rot_dim)
        if scaling == "linear":
            f = f / factor
        elif scaling == "bands":
            turns = context * f / (2 * math.pi)
            if turns <= low:
                f = f / factor
            elif turns < high:
                w = (turns - low) / (high - low)
                f = w * f + (1 - w) * f / factor
        elif scaling == "ramp":
            def index(n):
                return rot_dim / 2 * math.log(context / (2 * math.pi * n)) / math.log(base)
            a, b = max(0, math.floor(index(high))), min(rot_dim - 1, math.ceil(index(low)))
            w = min(1.0, max(0.0, (i - a) / (b - a if b != a else 0.001)))
            f = (1 - w) * f + w * f / factor
        out.append(f)
    return np.array(out), (0.1 * math.log(factor) + 1 if scaling == "ramp" else 1.0)


def _pairs(rot_dim, layout):
    h = rot_dim // 2
    i = np.arange(h)
    return (i, i + h) if layout == "half" else (2 * i, 2 * i + 1)


def turn(x, pos, freqs, layout, scale=1.0, back=False):
    """The rotation of x [rows, heads, head_dim] at pos [rows]; back: its transpose."""
    t = np.asarray(pos, np.float64)[:, None, None] * np.asarray(freqs, np.float64)
    c, s = scale * np.cos(t), scale * np.sin(t) * (-1 if back else 1)
    a, b = _pairs(2 * len(freqs), layout)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def norm_turn(x, gain, eps, pos, freqs, layout, scale=1.0):
    y = np.asarray(x, np.float64)
    if gain is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * gain
    return turn(y, pos, freqs, layout, scale)


def norm_turn_backward(x, gain, eps, pos, freqs, layout, dout, scale=1.0):
    """(dx, dgain) of norm_turn; dgain None without a gain."""
    dy = turn(np.asarray(dout, np.float64), pos, freqs, layout, scale, back=True)
    if gain is None:
        return dy, None
    x = np.asarray(x, np.float64)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = x * r
    gdy = gain * dy
    return r * (gdy - h * (h * gdy).mean(-1, keepdims=True)), (h * dy).sum((0, 1))


def append(k_pages, v_pages, slots, k, v):
    """Copies of the pools with row r's key and value at slots[r] (rows outside the pool passed over)."""
    kp, vp = k_pages.copy(), v_pages.copy()
    for r, s in enumerate(slots):
        if 0 <= s < PAGE * len(kp):
            kp[s // PAGE, :, s % PAGE] = k[r]
            vp[s // PAGE, :, :, s % PAGE] = v[r]
    return kp, vp


def attention(q, keys, values, scale):
    """(out [head_dim], log-sum-exp, sum_j p_j |v_j|, largest sum of |q k| scale) of one head over keys, values [n, head_dim]."""
    if len(keys) == 0:
        return np.zeros(len(q)), -np.inf, np.zeros(len(q)), 0.0
    s = keys @ q * scale
    m = s.max()
    p = np.exp(s - m)
    z = p.sum()
    return p @ values / z, m + math.log(z), p @ np.abs(values) / z, (np.abs(keys) @ np.abs(q)).max() * abs(scale)


def cached(k_pages, v_pages, table_row, n, head):
    """Keys and values [n, head_dim] of one environment and key head."""
    pages = np.asarray(table_row[:_pages(n)], np.int64)
    hd = k_pages.shape[3]
    return k_pages[pages, head].reshape(-1, hd)[:n], v_pages[pages, head].transpose(0, 2, 1).reshape(-1, hd)[:n]


def paged_attention(q, k_pages, v_pages, table, lens, scale):
    """(out, lse, sum_j p_j |v_j| as out, largest sum of |q k| scale as lse) of q [n_env, n_heads, head_dim]."""
    n, H, hd = q.shape
    G = H // k_pages.shape[1]
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, smax = np.zeros((n, H)), np.zeros((n, H))
    for e in range(n):
        for kh in range(H // G):
            keys, values = cached(k_pages, v_pages, table[e], int(lens[e]), kh)
            for h in range(kh * G, kh * G + G):
                out[e, h], lse[e, h], mag[e, h], smax[e, h] = attention(q[e, h], keys, values, scale)
    return out, lse, mag, smax
