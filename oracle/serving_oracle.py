"""Serving operators from their definitions: rows as 8-bit integers and their products, beam search's choice, page tables of forked
sequences, compacted pages.  numpy, fp64 and whole numbers, one element, candidate or table entry at a time where that says most."""
import numpy as np


def quant_rows(x):
    """(integers, scales) of the rows of x (fp64)."""
    q, scale = np.zeros(x.shape, dtype=np.int64), np.empty(len(x))
    for t, row in enumerate(x):
        most = np.max(np.abs(row))
        if not np.isfinite(most):
            scale[t] = np.nan
        elif most / 127 > 2.0 ** -126:
            scale[t], q[t] = most / 127, np.rint(127 * row / most)
        else:
            scale[t], q[t] = 2.0 ** -126, np.rint(row * 2.0 ** 126)
    return q, scale


def matmul_q8(a, sa, b, sb):
    return (a.astype(np.int64) @ b.astype(np.int64).T) * sa[:, None] * sb[None, :]


def linear_q8(x, w_down, s_down, w_up, s_up, silu):
    """(z, act(z), its integers and scales, y)"""
    z = matmul_q8(*quant_rows(x), w_down, s_down)
    a = z / (1 + np.exp(-z)) if silu else z
    q, s = quant_rows(a)
    return z, a, q, s, matmul_q8(q, s, w_up, s_up)


def beam_select(logits, score, n, done=None, done_token=0):
    """logits [batch * beams, V], score [batch, beams] -> parent, token, score [batch, n].  By score, then beam; a beam's by logit (logits closer than a last
    place of the score have one score), then token."""
    batch, beams = score.shape
    parent, token, best = (np.full((batch, n), v, dtype=t) for v, t in ((-1, np.int64), (-1, np.int64), (-np.inf, np.float64)))
    for b in range(batch):
        found = []
        for w in range(beams):
            row = logits[b * beams + w]
            if not np.isfinite(score[b, w]):
                continue
            if done is not None and done[b, w]:
                found.append((-score[b, w], w, 0.0, done_token))
                continue
            most = row.max()
            if not np.isfinite(most):
                continue
            lse = most + np.log(np.sum(np.exp(row - most)))
            value = score[b, w] + (row - lse)
            # more than n of a beam are never wanted; equal ones in the order of their tokens
            for v in np.argsort(-row, kind="stable")[:n]:
                if np.isfinite(value[v]):
                    found.append((-value[v], w, -row[v], int(v)))
        for i, (v, w, _, t) in enumerate(sorted(found)[:n]):
            parent[b, i], token[b, i], best[b, i] = b * beams + w, t, -v
    return parent, token, best


def kv_fork(refs, page_size, table, length, parent, grow):
    """Returns (refs, table, length, src, dst, rows, missing)."""
    n_pages, cols, n = len(refs), table.shape[1], len(parent)
    is_page = lambda e: 0 <= e < n_pages
    free = [p for p in range(n_pages) if refs[p] == 0]
    new_refs, out, now = np.array(refs), np.full((n, cols), -1, dtype=np.int32), np.zeros(n, dtype=np.int32)
    src, dst, rows, missing, had = np.full(n, -1, dtype=np.int32), np.full(n, -1, dtype=np.int32), np.zeros(n, dtype=np.int32), 0, set()
    for i in range(n):
        p = parent[i] if 0 <= parent[i] < len(table) else None
        old = 0 if p is None else max(int(length[p]), 0)
        heir = p is not None and p not in had
        had.add(p)
        keys = old + max(int(grow[i]), 0)
        now[i] = min(keys, 2 ** 31 - 1)
        full, part = divmod(old, page_size)
        for c in range(cols):
            e = -1 if p is None else int(table[p, c])
            half = is_page(e) and c == full and part > 0
            if is_page(e) and (c < full or (heir and (not half or refs[e] == 1))):
                out[i, c] = e
            elif c >= full and c * page_size < keys:
                if not free:
                    missing += 1
                    continue
                out[i, c] = free.pop(0)
                if half:
                    src[i], dst[i], rows[i] = e, out[i, c], part
        missing += max(0, -(-keys // page_size) - max(cols, 0))
    for entries, by in ((table, -1), (out, 1)):
        for e in entries.flatten():
            if is_page(e):
                new_refs[e] += by
    return new_refs, out, now, src, dst, rows, min(missing, 2 ** 31 - 1)


def kv_compact(refs, table):
    """Returns (refs, table, src, dst, page_map, n_live)."""
    n = len(refs)
    live = int(np.sum(np.asarray(refs) > 0))
    movers, holes = [p for p in range(live, n) if refs[p] > 0], [p for p in range(live) if refs[p] <= 0]
    page_map = np.array([p if refs[p] > 0 else -1 for p in range(n)], dtype=np.int32)
    page_map[movers] = holes
    src, dst = np.full(n // 2, -1, dtype=np.int32), np.full(n // 2, -1, dtype=np.int32)
    src[:len(movers)], dst[:len(holes)] = movers, holes
    new = np.zeros(n, dtype=np.int32)
    for p in range(n):
        if page_map[p] >= 0:
            new[page_map[p]] = refs[p]
    out = np.array([[page_map[e] if 0 <= e < n else -1 for e in row] for row in table], dtype=np.int32).reshape(table.shape)
    return new, out, src, dst, page_map, live
