"""Operators of answering with beams from a paged cache and with weights held in 8 bits, as cases that can be timed and compared.

Kinds of cases:

  matmul   activations quantised row by row and multiplied with a weight of 8-bit integers, one scale for each token and channel
  layer    the forward of a bottleneck layer whose two weights are held in 8 bits
  select   the candidates of highest score over all beams of a prompt and the whole vocabulary
  fork     the page tables of the next step's sequences from those of their parents (shared, forked, new or ended), with the half
           filled pages copied
  compact  the pages in use moved together to the front of the cache

Sizes are those of the library's benchmark workloads and tests (layers 4096 -> 1024 -> 4096 and 4096 x 11008, 777 and 16384 tokens, 8
key / value heads of 128, pages of 16 and 24 tokens, sequences of 4096 and 8192) and vocabularies of generic size.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # the logits of a decoding step: 16 prompts with 4 beams against a vocabulary of 32000
        {"name": "matmul_logits_64", "kind": "matmul", "M": 64, "K": 4096, "N": 32000, "dtype": "bf16"},
        # a wide projection over the benchmark's batch of prompts, 4 x 4096 tokens
        {"name": "matmul_prompts_16384", "kind": "matmul", "M": 16384, "K": 4096, "N": 11008, "dtype": "bf16"},
        # odd everything, in the precision path
        {"name": "matmul_ragged_f32", "kind": "matmul", "M": 777, "K": 5461, "N": 2047, "dtype": "f32"},
        # the serving layer, one decoding step of 16 sequences
        {"name": "layer_decode_16", "kind": "layer", "T": 16, "d_in": 4096, "r": 1024, "d_out": 4096, "dtype": "bf16", "silu": True},
        # the same layer over prompts
        {"name": "layer_prompts_16384", "kind": "layer", "T": 16384, "d_in": 4096, "r": 1024, "d_out": 4096, "dtype": "bf16", "silu": True},
        # one prompt, 4 beams: latency
        {"name": "select_1x4", "kind": "select", "batch": 1, "beams": 4, "V": 32000, "n": 4, "dtype": "bf16", "done": 0.0, "first": False},
        # a full batch of prompts with 8 beams and a large vocabulary
        {"name": "select_64x8", "kind": "select", "batch": 64, "beams": 8, "V": 131072, "n": 8, "dtype": "bf16", "done": 0.0, "first": False},
        # twice as many candidates as beams, some of which have ended; odd vocabulary, fp32 logits
        {"name": "select_16x5_f32", "kind": "select", "batch": 16, "beams": 5, "V": 50257, "n": 10, "dtype": "f32", "done": 0.2, "first": False},
        # a decoding step of 48 sequences: six end, as many prompts of up to 777 tokens come in, the others are one token further
        {"name": "fork_batch_48", "kind": "fork", "form": "batch", "groups": 48, "beams": 1, "kv": 4096, "page": 24, "Hkv": 2, "hd": 128,
         "grow": 777, "lens": 5},
        # 64 prompts with 8 beams, one token further, in pages of 256 KB
        {"name": "fork_beams_512", "kind": "fork", "form": "beams", "groups": 64, "beams": 8, "kv": 1024, "page": 64, "Hkv": 8, "hd": 128,
         "grow": 1, "lens": 3},
        # a small cache of which half is free
        {"name": "compact_1000", "kind": "compact", "pages": 1000, "page": 16, "Hkv": 2, "hd": 128, "batch": 8, "live": 0.5, "lens": 2},
        # 8192 pages of 64 KB, half of them free
        {"name": "compact_8192", "kind": "compact", "pages": 8192, "page": 16, "Hkv": 8, "hd": 128, "batch": 64, "live": 0.5, "lens": 4},
    ]


# ---- drawn cases -------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["matmul", "matmul", "layer", "layer", "select", "select", "fork", "fork", "compact"])
    if kind == "matmul":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        K = int(_log(rng, 16, 11009))
        K = max(8, K // 8 * 8) if dtype == "bf16" else K
        N = int(_log(rng, 8, 50258))
        return _no_more({"kind": kind, "M": max(1, int(_log(rng, 1, 16385))), "K": K, "N": N, "dtype": dtype}, "M")
    if kind == "layer":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        wide = lambda: 8 * rng.randint(8, 64) if rng.random() < 0.4 else 64 * rng.randint(8, 64)
        d_in, d_out = wide(), wide()
        r = max(16, 8 * (min(d_in, d_out) // rng.choice([2, 4, 4, 8]) // 8))
        return _no_more({"kind": kind, "T": max(1, int(_log(rng, 1, 16385))), "d_in": d_in, "r": min(r, 1024), "d_out": d_out, "dtype": dtype,
                         "silu": rng.random() < 0.7}, "T")
    if kind == "select":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        V = int(_log(rng, 100, 131073))
        beams = rng.choice([1, 2, 3, 4, 5, 8, 16])
        return _no_more({"kind": kind, "batch": max(1, int(_log(rng, 1, 129))), "beams": beams, "V": V, "n": rng.choice([beams, beams, 2 * beams]),
                         "dtype": dtype, "done": rng.choice([0.0, 0.0, 0.3]), "first": rng.random() < 0.2}, "batch")
    page, hd, Hkv = rng.choice([8, 16, 16, 24, 32, 64]), rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8])
    size = 2 * 2 * page * Hkv * hd
    if kind == "fork":
        beams = rng.choice([1, 2, 4, 5, 8])
        form = "batch" if beams == 1 else "beams"
        groups = max(1, int(_log(rng, 1, 512 // beams + 1)))
        kv = max(page, int(_log(rng, 16, 8193)))
        kv = max(page, min(kv, (1 << 28) // size * page // (groups * beams)))
        grow = rng.choice([1, 1, 4]) if form == "beams" else max(1, int(_log(rng, 1, 778)))
        return _no_more({"kind": kind, "form": form, "groups": groups, "beams": beams, "kv": kv, "page": page, "Hkv": Hkv, "hd": hd, "grow": grow,
                         "lens": rng.randint(1, 1 << 20)}, "groups")
    pages = max(4, min(int(_log(rng, 8, 8193)), (1 << 29) // size))
    return _no_more({"kind": kind, "pages": pages, "page": page, "Hkv": Hkv, "hd": hd, "batch": rng.randint(1, min(64, pages)),
                     "live": rng.choice([0.1, 0.5, 0.5, 0.9]), "lens": rng.randint(1, 1 << 20)}, "pages")


def _no_more(case, size):
    """The case with a size that costs no more than the largest listed one of its kind."""
    largest = [work(c) for c in listed() if c["kind"] == case["kind"]]
    while case[size] > 1 and any(work(case)[k] > max(w[k] for w in largest) for k in ("bytes", "flops")):
        case[size] = max(1, case[size] * 7 // 8)
        if "pages" in case:
            case["batch"] = min(case["batch"], case["pages"])
    return case


# ---- inputs ------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _acts(g, T, n, dtype):
    """Activations of which some channels are larger than the others."""
    x = torch.randn((T, n), generator=g, device=DEV)
    return (x * (1 + 7 * (torch.rand((n,), generator=g, device=DEV) < 0.01).float())).to(dtype)


def _weight(g, n, k):
    """A weight as a program that serves keeps it: integers in rows that start on 16 bytes, one scale for each row."""
    w = torch.randn((n, k), generator=g, device=DEV) / math.sqrt(k)
    s = w.abs().amax(1) / 127
    q = torch.zeros((n, -(-k // 16) * 16), dtype=torch.int8, device=DEV)[:, :k]
    q.copy_(torch.round(w / s[:, None]).clamp(-127, 127).to(torch.int8))
    return q, s


def _pool(case):
    """What the lists of a fork say, without the numbers of the pages: (lengths, pages that a sequence has in common with the first of its
    group, parent, grow), by the case alone."""
    rng = random.Random(case["lens"])
    G, W, page = case["groups"], case["beams"], case["page"]
    lens, common = [], []
    for _ in range(G):
        n = rng.randint(max(1, case["kv"] // 4), case["kv"])
        lens += [n] * W
        common += [0] + [rng.randint(0, n // page) for _ in range(W - 1)]
    if case["form"] == "beams":
        parent = [g * W + rng.randrange(W) for g in range(G) for _ in range(W)]
        grow = [case["grow"]] * (G * W)
    else:
        gone = set(rng.sample(range(G), G // 8))
        parent = [i for i in range(G) if i not in gone] + [-1] * len(gone)
        grow = [1] * (G - len(gone)) + [rng.randint(max(1, case["grow"] // 8), case["grow"]) for _ in gone]
    return lens, common, parent, grow


def _cols(case):
    lens, _, parent, grow = _pool(case)
    return max(-(-(grow[i] + (lens[p] if p >= 0 else 0)) // case["page"]) for i, p in enumerate(parent)) + 2


def _fresh(case):
    """Pages that the new sequences take, and the rows of half filled pages that are copied."""
    lens, _, parent, grow = _pool(case)
    page, seen, pages, rows = case["page"], set(), 0, 0
    for p, g in zip(parent, grow):
        n = lens[p] if p >= 0 else 0
        pages += -(-(n + g) // page) - n // page
        if p >= 0 and n % page:
            if p in seen:
                rows += n % page
            else:
                pages -= 1
        seen.add(p)
    return pages, rows


def _table(rows, cols):
    t = np.full((len(rows), cols), -1, dtype=np.int32)
    for b, row in enumerate(rows):
        t[b, :len(row)] = row
    return t


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] == "matmul":
        b, sb = _weight(g, case["N"], case["K"])
        return {"case": case, "x": _acts(g, case["M"], case["K"], _type(case)), "b": b, "sb": sb}
    if case["kind"] == "layer":
        down, s_down = _weight(g, case["r"], case["d_in"])
        up, s_up = _weight(g, case["d_out"], case["r"])
        return {"case": case, "x": _acts(g, case["T"], case["d_in"], _type(case)), "down": down, "s_down": s_down, "up": up, "s_up": s_up}
    if case["kind"] == "select":
        B, W, V = case["batch"], case["beams"], case["V"]
        ld = -(-V // 8) * 8                              # rows as a product leaves them
        score = -20 * torch.rand((B, W), generator=g, device=DEV)
        if case["first"]:
            score[:, 1:] = -math.inf                     # the first step: all beams are alike, one counts
        st = {"case": case, "logits": _randn(g, (B * W, ld), _type(case), 2.5)[:, :V], "score": score, "done": None}
        if case["done"]:
            st["done"] = (torch.rand((B, W), generator=g, device=DEV) < case["done"]).to(torch.int32)
        return st
    rng = np.random.default_rng(seed)
    page, Hkv, hd = case["page"], case["Hkv"], case["hd"]
    if case["kind"] == "fork":
        lens, common, parent, grow = _pool(case)
        need = [-(-n // page) - c for n, c in zip(lens, common)]
        n_pages = (sum(need) + _fresh(case)[0]) * 9 // 8 + 4
        order = rng.permutation(n_pages)
        rows, at = [], 0
        for i, (n, c) in enumerate(zip(need, common)):
            rows.append((list(rows[i - i % case["beams"]][:c]) if c else []) + list(order[at:at + n]))
            at += n
        refs = np.zeros(n_pages, dtype=np.int32)
        for row in rows:
            refs[row] += 1
        st = {"case": case, "refs": _dev(refs), "table": _dev(_table(rows, _cols(case))), "len": _dev(lens), "parent": _dev(parent), "grow": _dev(grow)}
    else:
        n_pages = case["pages"]
        lens = random.Random(case["lens"])
        live = rng.permutation(n_pages)[:max(1, int(case["live"] * n_pages))]
        cuts = sorted(lens.randint(0, len(live)) for _ in range(case["batch"] - 1))
        rows = [list(live[a:b]) for a, b in zip([0] + cuts, cuts + [len(live)])]
        refs = np.zeros(n_pages, dtype=np.int32)
        refs[live] = 1
        for row in rows[1:]:                             # the first pages of a prompt that several sequences share
            row[:0] = rows[0][:3]
            refs[rows[0][:3]] += 1
        st = {"case": case, "refs": _dev(refs), "table": _dev(_table(rows, max(len(r) for r in rows) + 1))}
    st |= {n: _randn(g, (n_pages, page, Hkv, hd), torch.bfloat16) for n in ("k_cache", "v_cache")}
    return st


# ---- one pass ----------------------------------------------------------------------------------------------
def run(st):
    return {"matmul": _run_matmul, "layer": _run_layer, "select": _run_select, "fork": _run_fork, "compact": _run_compact}[st["case"]["kind"]](st)


def _quantised(x):
    """Integers (in 32 bits) and scale of each row; the quotients in 64 bits, where a tie is one."""
    amax = x.abs().amax(1, keepdim=True)
    scale = (amax.float() / 127).clamp(min=2.0 ** -126)
    q = torch.where(amax.double() / 127 < 2.0 ** -126, x.double() * 2.0 ** 126, x.double() * 127 / amax.double())
    return torch.round(q).float(), scale


def _product(q, s, b, sb):
    return torch.matmul(q, b.float().t()) * s * sb[None, :]


def _run_matmul(st):
    if own:
        from paper_2512_12131_amd import binding as B
        q, s = B.lr_quant_rows(st["x"])
        return B.lr_matmul_q8(q, s, st["b"], st["sb"], dtype=st["x"].dtype)
    return _product(*_quantised(st["x"]), st["b"], st["sb"]).to(st["x"].dtype)


def _run_layer(st):
    c = st["case"]
    if own:
        from paper_2512_12131_amd import binding as B
        return B.lr_linear_q8_fwd(st["x"], st["down"], st["s_down"], st["up"], st["s_up"], act=B.LR_ACT_SILU if c["silu"] else B.LR_ACT_IDENTITY)
    z = _product(*_quantised(st["x"]), st["down"], st["s_down"])
    if c["silu"]:
        z = z / (1 + torch.exp(-z))
    return _product(*_quantised(z), st["up"], st["s_up"]).to(st["x"].dtype)


END = 2                                                  # the token that an ended beam goes on with


def _run_select(st):
    c = st["case"]
    B_, W, V, n = c["batch"], c["beams"], c["V"], c["n"]
    if own:
        from paper_2512_12131_amd import binding as B
        return B.lr_beam_select(st["logits"], st["score"], n, done=st["done"], done_token=END)
    x = st["logits"].double()
    m = x.amax(1, keepdim=True)
    lse = m + torch.log(torch.exp(x - m).sum(1, keepdim=True))
    score = st["score"].double().view(-1, 1)
    cand = score + (x - lse)
    if st["done"] is not None:
        at_end = torch.where(torch.arange(V, device=DEV)[None, :] == END, score, -math.inf)
        cand = torch.where(st["done"].view(-1, 1) != 0, at_end, cand)
    cand = cand.view(B_, W * V)
    where = torch.arange(W * V, device=DEV)[None, :]
    first = torch.arange(B_, device=DEV)[:, None] * W
    parent, token, best = [], [], []
    for _ in range(n):                                   # the largest, the first of equal ones; then without it
        top = cand.amax(1, keepdim=True)
        at = torch.where(cand == top, where, W * V).amin(1, keepdim=True)
        some = top > -math.inf
        parent.append(torch.where(some, first + at // V, -1))
        token.append(torch.where(some, at % V, -1))
        best.append(top)
        cand = torch.where(where == at, -math.inf, cand)
    return torch.cat(parent, 1).to(torch.int32), torch.cat(token, 1).to(torch.int32), torch.cat(best, 1).float()


def _copied(st, src, dst, rows):
    """The first `rows` tokens of page src onto page dst, pair by pair; pairs of -1 are passed over."""
    for name in ("k_cache", "v_cache"):
        cache = st[name]
        take = cache[src.long().clamp(min=0)]
        keep = cache[dst.long().clamp(min=0)]
        inside = torch.arange(cache.shape[1], device=DEV)[None, :, None, None] < rows[:, None, None, None]
        # pairs without pages write the last pair's page once more, or page 0 where there is no pair: what that holds anyway
        some = (dst >= 0)[:, None, None, None]
        last = torch.where(dst >= 0, torch.arange(dst.shape[0], device=DEV), -1).amax().clamp(min=0)
        new = torch.where(inside, take, keep)
        new = torch.where(some, new, torch.where(dst[last] >= 0, new[last], cache[0])[None])
        cache[torch.where(dst >= 0, dst, dst[last].clamp(min=0)).long()] = new


def _run_fork(st):
    c = st["case"]
    if own:
        from paper_2512_12131_amd import binding as B
        refs, table, length, (src, dst, rows), missing = B.lr_kv_fork(st["refs"], c["page"], st["table"], st["len"], st["parent"], st["grow"])
        B.lr_kv_copy(st["k_cache"], st["v_cache"], src, dst, rows)
        return refs, table, length, src, dst, rows, missing, st["k_cache"], st["v_cache"]
    refs, table, page = st["refs"], st["table"], c["page"]
    n_pages, cols, parent = refs.shape[0], table.shape[1], st["parent"].long()
    n_in, n_out = table.shape[0], parent.shape[0]
    has = parent >= 0
    par = parent.clamp(min=0)
    old = torch.where(has, st["len"].long()[par], 0)
    new = old + st["grow"].long()
    i = torch.arange(n_out, device=DEV)
    heir_of = torch.full((n_in,), n_out, device=DEV).scatter_reduce_(0, par, torch.where(has, i, n_out), "amin")
    heir = has & (heir_of[par] == i)
    col = torch.arange(cols, device=DEV)[None, :]
    mine = torch.where(has[:, None], table.long()[par], -1)
    full, part = (old // page)[:, None], (old % page)[:, None]
    half = (col == full) & (part > 0) & (mine >= 0)
    alone = refs[mine.clamp(min=0)] == 1
    keep = (col < full) | (heir[:, None] & (mine >= 0) & (~half | alone))
    needed = (col >= full) & (col * page < new[:, None])
    take = needed & ~keep
    free = refs == 0
    slots = torch.full((n_pages + 1,), -1, dtype=torch.int64, device=DEV)
    slots.scatter_(0, torch.where(free, torch.cumsum(free, 0) - 1, n_pages), torch.where(free, torch.arange(n_pages, device=DEV), -1))
    slots[n_pages] = -1
    nth = (torch.cumsum(take.flatten(), 0) - 1).view(n_out, cols)
    given = torch.where(take, slots[nth.clamp(min=0, max=n_pages)], -1)
    out = torch.where(keep, mine, given)
    fallen = ((new[:, None] + page - 1) // page - cols).clamp(min=0).sum()
    missing = ((take & (given < 0)).sum() + fallen).to(torch.int32).view(1)
    # every entry of the old tables lets go of its page, every one of the new tables holds one
    held = torch.zeros((n_pages + 1,), dtype=torch.int32, device=DEV)
    for entries, sign in ((table.long(), -1), (out, 1)):
        at = torch.where(entries >= 0, entries, n_pages).flatten()
        held.scatter_add_(0, at, torch.full_like(at, sign, dtype=torch.int32))
    moved = half & take & (given >= 0)
    src = torch.where(moved, mine, -1).amax(1)
    dst = torch.where(moved, given, -1).amax(1)
    rows = torch.where(src >= 0, part[:, 0], 0)
    _copied(st, src, dst, rows)
    i32 = torch.int32
    return refs + held[:-1], out.to(i32), new.to(i32), src.to(i32), dst.to(i32), rows.to(i32), missing, st["k_cache"], st["v_cache"]


def _run_compact(st):
    if own:
        from paper_2512_12131_amd import binding as B
        refs, table, (src, dst), where, live = B.lr_kv_compact(st["refs"], st["table"])
        B.lr_kv_copy(st["k_cache"], st["v_cache"], src, dst)
        return refs, table, src, dst, where, live, st["k_cache"], st["v_cache"]
    refs, table = st["refs"], st["table"]
    n = refs.shape[0]
    page = torch.arange(n, device=DEV)
    held = refs > 0
    live = held.sum()
    mover, hole = held & (page >= live), ~held & (page < live)
    lists = []
    for which in (mover, hole):
        full = torch.full((n + 1,), -1, dtype=torch.int64, device=DEV)
        full.scatter_(0, torch.where(which, torch.cumsum(which, 0) - 1, n), torch.where(which, page, -1))
        lists.append(full[:n // 2])
    src, dst = lists
    where = torch.where(held & ~mover, page, -1)
    to = torch.cat((dst, torch.full((1,), -1, dtype=torch.int64, device=DEV)))
    where = torch.where(mover, to[(torch.cumsum(mover, 0) - 1).clamp(min=0, max=to.shape[0] - 1)], where)
    new = torch.zeros((n + 1,), dtype=torch.int32, device=DEV)
    new.scatter_(0, torch.where(held, where, n), torch.where(held, refs, 0))
    out = torch.where((table >= 0) & (table < n), where[table.long().clamp(min=0, max=n - 1)], -1)
    if src.shape[0]:
        _copied(st, src, dst, torch.full_like(src, st["k_cache"].shape[1]))
    i32 = torch.int32
    return new[:n], out.to(i32), src.to(i32), dst.to(i32), where.to(i32), live.to(i32).view(1), st["k_cache"], st["v_cache"]


# ---- the work that no form can do without ------------------------------------------------------------------
def work(case):
    e = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if case["kind"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K * e + N * K + 4 * N + M * N * e, "flops": 2 * M * N * K}
    if case["kind"] == "layer":
        T, d, r, n = case["T"], case["d_in"], case["r"], case["d_out"]
        return {"bytes": T * (d + n) * e + r * (d + n) + 4 * (r + n), "flops": 2 * T * r * (d + n)}
    if case["kind"] == "select":
        R = case["batch"] * case["beams"]
        return {"bytes": R * case["V"] * e + R * 4 + case["batch"] * case["n"] * 12, "flops": 3 * R * case["V"]}
    size = 2 * 2 * case["Hkv"] * case["hd"]              # bytes of a token, keys and values
    if case["kind"] == "fork":
        lens, common, parent, _ = _pool(case)
        cols, (fresh, rows) = _cols(case), _fresh(case)
        held = sum(-(-n // case["page"]) - c for n, c in zip(lens, common))
        pages = (held + fresh) * 9 // 8 + 4
        return {"bytes": 4 * (len(lens) * (cols + 1) + len(parent) * (cols + 6) + 2 * pages) + 2 * rows * size,
                "flops": len(parent) * cols + pages}
    n = case["pages"]
    live = max(1, int(case["live"] * n))
    moves = live * (n - live) // n                       # on average over the inputs
    return {"bytes": 4 * (4 * n + 2 * (live + 4 * case["batch"])) + 2 * moves * case["page"] * size, "flops": 2 * n}


# ---- 64 bits and plain loops, from the definitions ---------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return {"matmul": _exact_matmul, "layer": _exact_layer, "select": _exact_select, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](st)


def _nearest(x):
    """The multiples of a 127th of the row's largest magnitude that are nearest to its values."""
    most = x.abs().amax(1, keepdim=True)
    most = torch.where(most > 0, most, 1.0)
    return torch.round(127 * x / most) * (most / 127)


def _exact_matmul(st):
    return _nearest(st["x"].double()) @ (st["b"].double() * st["sb"].double()[:, None]).t().contiguous()


def _exact_layer(st):
    z = _nearest(st["x"].double()) @ (st["down"].double() * st["s_down"].double()[:, None]).t().contiguous()
    a = z * torch.sigmoid(z) if st["case"]["silu"] else z
    return _nearest(a) @ (st["up"].double() * st["s_up"].double()[:, None]).t().contiguous()


def _exact_select(st):
    c = st["case"]
    W, V, n = c["beams"], c["V"], c["n"]
    parent = torch.full((c["batch"], n), -1, dtype=torch.int32)
    token, best = parent.clone(), torch.full((c["batch"], n), -math.inf, dtype=torch.float64)
    for b in range(c["batch"]):
        rows = []
        for w in range(W):
            row = torch.log_softmax(st["logits"][b * W + w].double(), 0) + st["score"][b, w].double()
            if st["done"] is not None and int(st["done"][b, w]):
                row = torch.full_like(row, -math.inf)
                row[END] = st["score"][b, w].double()
            rows.append(row)
        value, at = torch.sort(torch.cat(rows), descending=True, stable=True)
        value, at = value[:n].cpu(), at[:n].cpu()
        for i in range(min(n, value.shape[0])):
            if value[i] > -math.inf:
                parent[b, i], token[b, i], best[b, i] = b * W + int(at[i]) // V, int(at[i]) % V, value[i]
    return parent.to(DEV), token.to(DEV), best.to(DEV)


def _moved(st, pairs):
    out = []
    for name in ("k_cache", "v_cache"):
        cache = st[name].clone()
        for s, d, n in pairs:
            cache[d, :n] = st[name][s, :n]
        out.append(cache.double())
    return out


def _exact_fork(st):
    page = st["case"]["page"]
    refs, table, lens, parent, grow = (st[n].cpu().numpy() for n in ("refs", "table", "len", "parent", "grow"))
    cols, n_out = table.shape[1], len(parent)
    free, at, missing = [p for p in range(len(refs)) if refs[p] == 0], 0, 0
    new_refs, out, seen = refs.astype(np.int64), np.full((n_out, cols), -1, dtype=np.int32), set()
    length = np.zeros(n_out, dtype=np.int32)
    src, dst, rows = np.full(n_out, -1, dtype=np.int32), np.full(n_out, -1, dtype=np.int32), np.zeros(n_out, dtype=np.int32)
    for i, p in enumerate(parent):
        old = table[p] if p >= 0 else np.full(cols, -1, dtype=np.int32)
        n = int(lens[p]) if p >= 0 else 0
        heir = p >= 0 and p not in seen
        seen.add(p)
        length[i] = n + grow[i]
        for col in range(cols):
            half = col == n // page and n % page > 0 and old[col] >= 0
            if col < n // page or (heir and old[col] >= 0 and (not half or refs[old[col]] == 1)):
                out[i, col] = old[col]
            elif col * page < length[i]:
                if at == len(free):
                    missing += 1
                    continue
                out[i, col] = free[at]
                at += 1
                if half:
                    src[i], dst[i], rows[i] = old[col], out[i, col], n % page
        missing += max(0, -(-int(length[i]) // page) - cols)
    np.subtract.at(new_refs, table[table >= 0], 1)
    np.add.at(new_refs, out[out >= 0], 1)
    k, v = _moved(st, [(int(s), int(d), int(r)) for s, d, r in zip(src, dst, rows) if s >= 0])
    return (*(_dev(a) for a in (new_refs, out, length, src, dst, rows, [missing])), k, v)


def _exact_compact(st):
    refs, table = st["refs"].cpu().numpy(), st["table"].cpu().numpy()
    n = len(refs)
    live = int((refs > 0).sum())
    movers, holes = [p for p in range(live, n) if refs[p] > 0], [p for p in range(live) if refs[p] <= 0]
    src, dst, where, new = (np.full(m, -1, dtype=np.int32) for m in (n // 2, n // 2, n, n))
    src[:len(movers)], dst[:len(holes)] = movers, holes
    new[:] = 0
    for p in range(n):
        if refs[p] > 0 and p < live:
            where[p] = p
    for s, d in zip(movers, holes):
        where[s] = d
    for p in range(n):
        if where[p] >= 0:
            new[where[p]] = refs[p]
    out = np.where(table >= 0, where[np.maximum(table, 0)], -1)
    k, v = _moved(st, [(s, d, st["k_cache"].shape[1]) for s, d in zip(movers, holes)])
    return (*(_dev(a) for a in (new, out, src, dst, where, [live])), k, v)
