"""Rotary tables, rotation at positions, and a paged key / value cache with its attention: numpy fp64, one token and one head at a
time, from the definitions."""
import numpy as np


def rope_table(n, rot, base=10000.0, first=0, factor=1.0, ramp=None, mscale=1.0):
    w = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if ramp is None:
        w = w / factor
    else:
        context, low, high = ramp
        for i in range(rot // 2):
            t = context * w[i] / (2 * np.pi)
            keep = 0.0 if t <= low else 1.0 if t >= high else (t - low) / (high - low)
            w[i] = keep * w[i] + (1 - keep) * w[i] / factor
    a = (first + np.arange(n, dtype=np.float64))[:, None] * w[None, :]
    return mscale * np.cos(a), mscale * np.sin(a)


def rotate(x, cos, sin, interleaved=False, inverse=False):
    """x [.., hd], cos and sin [rot / 2] of its position.  Returns (result, the sum of the two products' magnitudes of each element)."""
    half = len(cos)
    y, mag = x.copy(), np.abs(x)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos[i], -sin[i] if inverse else sin[i]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        mag[..., a] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s)
        mag[..., b] = np.abs(x[..., b] * c) + np.abs(x[..., a] * s)
    return y, mag


def places(cu_q, kv_len, page_table, page_size, n_pages, T):
    """[(token, sequence, position, page, row)] of the tokens that have a place."""
    out = []
    for b in range(len(kv_len)):
        n = cu_q[b + 1] - cu_q[b]
        for i in range(n):
            p = kv_len[b] - n + i
            if 0 <= p < page_table.shape[1] * page_size and 0 <= page_table[b, p // page_size] < n_pages and cu_q[b] + i < T:
                out.append((cu_q[b] + i, b, p, page_table[b, p // page_size], p % page_size))
    return out


def gather(cache, page_table_row, keys):
    """The first `keys` rows [keys, heads, hd] of a sequence; rows of pages that are none are zeros."""
    n_pages, page_size = cache.shape[:2]
    out = np.zeros((keys,) + cache.shape[2:])
    for j in range(keys):
        page = page_table_row[j // page_size]
        if 0 <= page < n_pages:
            out[j] = cache[page, j % page_size]
    return out


def attention_paged(q, k_cache, v_cache, page_table, cu_q, kv_len, H, scale):
    """q [T, H, hd].  Returns o [T, H, hd], lse [T, H] (NaN where a token belongs to nobody), and for error bounds the softmax-weighted
    sum of |v| [T, H, hd] and the largest scaled sum of |q_i k_i| [T, H]."""
    T, hd = q.shape[0], q.shape[2]
    grp = H // k_cache.shape[2]
    capacity = page_table.shape[1] * k_cache.shape[1]
    o, mag = np.full((2, T, H, hd), np.nan)
    lse, dots = np.full((2, T, H), np.nan)
    for b in range(len(kv_len)):
        n = cu_q[b + 1] - cu_q[b]
        if n <= 0:
            continue
        most = min(max(int(kv_len[b]), 0), capacity)
        k, v = gather(k_cache, page_table[b], most), gather(v_cache, page_table[b], most)
        for i in range(n):
            t, keys = cu_q[b] + i, min(max(int(kv_len[b]) - n + i + 1, 0), capacity)
            for h in range(H):
                if keys == 0:
                    o[t, h], mag[t, h], lse[t, h], dots[t, h] = 0, 0, -np.inf, 0
                    continue
                kk, vv = k[:keys, h // grp], v[:keys, h // grp]
                s = scale * (kk @ q[t, h])
                m = s.max()
                p = np.exp(s - m)
                o[t, h], mag[t, h] = (p @ vv) / p.sum(), (p @ np.abs(vv)) / p.sum()
                lse[t, h] = m + np.log(p.sum())
                dots[t, h] = scale * (np.abs(kk) @ np.abs(q[t, h])).max()
    return o, lse, mag, dots
