"""The paged cache at the edges of its lists: calls of fewer tokens than the lists count, batches of no or of very many sequences, values
that are no numbers in single columns, long runs of pages.  Bounds as in test_gpu_attention_paged.py."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2512_12131_amd import binding as B
from test_gpu_attention_paged import HD, _dense, call, compare
from test_gpu_kv_append import BF, DEV, lists, make, np64

pytestmark = pytest.mark.gpu


def against_64_bits(q, o, lse, c, seqs, H):
    """Every element of o and lse against 64 bits on the GPU, all heads of a sequence at once."""
    Hkv = c["k_cache"].shape[2]
    t0, grp = int(c["cu_q"][0]), H // Hkv
    for b, (n, kv) in enumerate(seqs):
        k, v = (x.double().view(kv, Hkv, HD).permute(1, 2, 0).contiguous() for x in _dense(c, b, kv))      # [Hkv, hd, keys]
        qq = q[t0:t0 + n, :H * HD].double().view(n, Hkv, grp, HD).permute(1, 0, 2, 3).reshape(Hkv, n * grp, HD)
        hidden = (torch.arange(kv, device=DEV)[None] > torch.arange(kv - n, kv, device=DEV)[:, None]).repeat_interleave(grp, 0)[None]
        s = torch.bmm(qq, k) * HD ** -0.5
        d = 128 * 2.0 ** -24 * (torch.bmm(qq.abs(), k.abs()) * HD ** -0.5).masked_fill(hidden, 0).amax(-1)
        s = s.masked_fill(hidden, float("-inf"))
        l = torch.logsumexp(s, -1)
        w, v = torch.exp(s - l[..., None]), v.transpose(1, 2).contiguous()
        rows = lambda x: x.view(Hkv, n, grp, -1).permute(1, 0, 2, 3).reshape(n, H, -1)
        ref, mag, d, l = rows(torch.bmm(w, v)), rows(torch.bmm(w, v.abs())), rows(d)[..., 0], rows(l)[..., 0]
        err = (o[t0:t0 + n, :H * HD].double().view(n, H, HD) - ref).abs()
        assert bool((err <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * d + 2.0 ** -18)[..., None] * mag).all()), b
        lerr = (lse[t0:t0 + n].double() - l).abs()
        assert bool((lerr <= d + 2.0 ** -20 * (1 + l.abs()) + kv * 2.0 ** -24).all()), (b, float(lerr.max()))
        t0 += n


# ---- lists that count more tokens than the call has ----------------------------------------------------------
@pytest.mark.parametrize("seqs,H,Hkv,T", [([(5, 30)], 1, 1, 3), ([(4, 4)], 8, 2, 1), ([(1, 40), (60, 200)], 4, 2, 45), ([(1, 300), (8, 900)], 8, 1, 4),
                                          ([(200, 1200), (1, 9)], 4, 2, 130), ([(150, 150), (3, 50)], 2, 2, 150)])
def test_attention_of_the_first_tokens_of_a_batch(seqs, H, Hkv, T):
    """A token's position is counted from its sequence's last one, whether or not the call has that."""
    print(f"first {T} tokens of {seqs}", flush=True)
    c, every = make(seqs, Hkv, HD, 16, seed=20)
    _, _, table = lists(c)
    cu = np.cumsum([0] + [n for n, _ in seqs])
    for b, (n, kv) in enumerate(seqs):                # what the tokens that are not there would have been the first to see
        for j in range(kv - min(n, max(0, int(cu[b + 1]) - T)), kv):
            c["k_cache"][table[b, j // 16], j % 16], c["v_cache"][table[b, j // 16], j % 16] = float("nan"), float("inf")
    q, o, lse = call(c, every, H)
    short, short_lse = torch.full_like(o[:T], 7.0), torch.full_like(lse[:T], 7.0)
    B.lr_attention_paged_fwd(q[:T], H=H, o=short, lse=short_lse, **c)
    torch.cuda.synchronize()
    assert bool(short.isfinite().all()) and bool(short_lse.isfinite().all())
    # the rows that the call has not are what the oracle computes, which knows of no call
    ref, lse_ref, *_ = po.attention_paged(np64(q).reshape(every, H, HD), *(np.nan_to_num(np64(c[n]), nan=0, posinf=0) for n in ("k_cache", "v_cache")),
                                          table, cu, [kv for _, kv in seqs], H, HD ** -0.5)
    rest, rest_lse = torch.from_numpy(ref[T:]).to(DEV, BF).view(every - T, -1), torch.from_numpy(lse_ref[T:]).to(DEV, torch.float32)
    compare(torch.cat([short, rest]), torch.cat([short_lse, rest_lse]), q, c, H)


def test_a_batch_of_no_sequences():
    """Every token belongs to nobody: nothing is written."""
    cache = torch.randn((4, 16, 2, HD), device=DEV).to(BF)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    none = {"k_cache": cache.clone(), "v_cache": cache.clone(), "page_table": i32(0, 4), "cu_q": i32(1), "kv_len": i32(0)}
    x = torch.randn((3, 4 * HD), device=DEV).to(BF)
    out = torch.full_like(x, 7.0)
    B.lr_kv_append(x, x, q=x, H=4, q_out=out, **none)
    q, o, lse = call(none, 3, 4)
    assert bool((out == 7).all()) and bool((o == 7).all()) and bool((lse == 7).all())
    assert torch.equal(none["k_cache"], cache) and torch.equal(none["v_cache"], cache)


# ---- large logits ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("seqs", [[(1, 777), (5, 70)], [(200, 700)], [(300, 3000)]])
def test_logits_up_to_the_stated_size(seqs):
    """Keys score 0, 1, .. 6 times 2^22, over and over (at most 2^24.6): a row is the mean of the values of its
    largest.  Probabilities of that mean are alike, so o is off by its own rounding and that of 32-bit sums; lse by half a step of the
    exponent's 32 bits (2^-24 of 2^25.2)."""
    H, Hkv, page = 4, 2, 16
    c, T = make(seqs, Hkv, HD, page, seed=26)
    _, _, table = lists(c)
    c["k_cache"].zero_()
    for b, (_, kv) in enumerate(seqs):
        for j in range(kv):
            c["k_cache"][table[b, j // page], j % page, :, 0] = j % 7
    q = torch.zeros((T, H, HD), dtype=BF, device=DEV)
    q[..., 0] = 1.0
    o, lse = B.lr_attention_paged_fwd(q.view(T, -1), H=H, scale=2.0 ** 22, **c)
    torch.cuda.synchronize()
    t0 = 0
    for b, (n, kv) in enumerate(seqs):
        v = _dense(c, b, kv)[1].double().view(kv, Hkv, HD)
        score = torch.arange(kv, device=DEV) % 7
        seen = torch.arange(kv, device=DEV)[None] <= torch.arange(kv - n, kv, device=DEV)[:, None]
        best = torch.where(seen, score, -1).amax(1)
        w = (seen & (score[None] == best[:, None])).double()
        for h in range(H):
            ref = w @ v[:, h // 2].contiguous() / w.sum(1, keepdim=True)
            mag = w @ v[:, h // 2].abs().contiguous() / w.sum(1, keepdim=True)
            err = (o[t0:t0 + n, h * HD:(h + 1) * HD].double() - ref).abs()
            assert bool((err <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -18) * mag).all()), (b, h)
            l = best.double() * 2.0 ** 22 + torch.log(w.sum(1))
            assert bool(((lse[t0:t0 + n, h].double() - l).abs() <= 2.0 ** -22 * (1 + l.abs())).all()), (b, h)
        t0 += n


# ---- values that are no numbers --------------------------------------------------------------------------------
# (new tokens, keys), H, Hkv, the key whose value it is: one item of few rows, few tiles, many tiles, keys in several splits, both joined
VALUES = [([(5, 41)], 4, 1, 39), ([(8, 700), (1, 90)], 4, 1, 696), ([(150, 150)], 4, 2, 70), ([(150, 470)], 1, 1, 400), ([(200, 1100)], 1, 1, 1003),
          ([(40, 360), (1, 200)], 2, 2, 330), ([(64, 3900), (1, 400)], 16, 8, 3871), ([(300, 3000)], 4, 1, 2800)]


@pytest.mark.parametrize("seqs,H,Hkv,at", VALUES)
def test_values_that_are_no_numbers_reach_their_columns(seqs, H, Hkv, at):
    """Finite keys: a row that sees the key has the infinity or NaN in exactly the columns of its value, the rows before, and all other
    columns, what they have without it."""
    print(f"values that are no numbers {seqs} H={H} Hkv={Hkv} at {at}", flush=True)
    n, kv = seqs[0]
    before = at - (kv - n)                            # tokens of the first sequence that don't see it
    assert 0 < before < n
    c, T = make(seqs, Hkv, HD, 16, seed=22)
    _, _, table = lists(c)
    clean = {**c, "v_cache": c["v_cache"].clone()}
    columns = {3: float("inf"), 64: float("-inf"), 77: float("nan"), 127: float("inf")}
    for col, x in columns.items():
        c["v_cache"][table[0, at // 16], at % 16, :, col] = x
        clean["v_cache"][table[0, at // 16], at % 16, :, col] = 0
    q, o, lse = call(c, T, H)
    _, o0, lse0 = call(clean, T, H)
    against_64_bits(q, o0, lse0, clean, seqs, H)
    assert torch.equal(lse, lse0)
    seen, got = o[before:n].float().view(-1, HD), o.clone()
    for col, x in columns.items():
        assert bool((seen[:, col] == x).all() if x == x else seen[:, col].isnan().all()), col
        got[before:n].view(-1, H, HD)[..., col] = o0[before:n].view(-1, H, HD)[..., col]
    assert torch.equal(got, o0)


# ---- long runs of pages, many sequences ------------------------------------------------------------------------
def _tiles(kv):
    return max(1, -(-kv // 64))


def _narrow_blocks(seqs, Hkv):
    """32-key blocks of the longest run that one wavefront takes, of a batch of single tokens: the kernel's rule for splits."""
    w = Hkv * sum(_tiles(kv) for _, kv in seqs)
    assert w > 4 * 512
    length = max(-(-w // 2048), int((w / 64) ** 0.5) + 1, 2)
    longest = 0
    for _, kv in seqs:
        splits = max(1, (_tiles(kv) + length // 2) // length)
        longest = max(longest, -(-(-(-_tiles(kv) // splits) * 2) // 4))
    return longest


@pytest.mark.parametrize("page", [8, 16, 48])
def test_single_tokens_over_long_runs_of_pages(page):
    """A wavefront's keys pass more than one window of 512, whose page numbers are on their way while others are worked on."""
    seqs = [(1, 8192 - 97 * b) for b in range(64)]
    assert _narrow_blocks(seqs, 8) >= 16           # (half a window and the two blocks around it are 10)
    c, T = make(seqs, 8, HD, page, seed=23)
    q, o, lse = call(c, T, 32)
    against_64_bits(q, o, lse, c, seqs, 32)
    again = call(c, T, 32)
    assert torch.equal(o, again[1]) and torch.equal(lse, again[2])


@pytest.mark.parametrize("seqs,H,Hkv,page", [
    # more sequences than lanes, long ones of many rows among the first 64, the next and the last
    ([(1, 300)] * 30 + [(70, 2000)] + [(1, 500)] * 60 + [(100, 2500), (2, 900)] + [(1, 200)] * 40 + [(300, 300), (1, 3000)], 8, 2, 16),
    ([(1, 2000)] * 100 + [(256, 4096)] + [(1, 2000)] * 19, 8, 2, 64),
    # very many
    ([(1, 1 + 7 * b % 301) for b in range(1500)], 4, 1, 8), ([(1 + b % 3, 3 + b % 40) for b in range(4200)], 2, 1, 8)])
def test_more_sequences_than_lanes(seqs, H, Hkv, page):
    print(f"{len(seqs)} sequences H={H} Hkv={Hkv} page={page}", flush=True)
    c, T = make(seqs, Hkv, HD, page, seed=24)
    q, o, lse = call(c, T, H)
    against_64_bits(q, o, lse, c, seqs, H)


# ---- what a row's rounding may cost ------------------------------------------------------------------------------
@pytest.mark.parametrize("n,kv", [(150, 700), (50, 100), (40, 640), (3, 640), (600, 8000)])
def test_a_row_that_one_key_takes(n, kv):
    """The largest probability of a row counts in full: where one key has nearly all of the weight, o is its value, rounded once.  The first
    key scores 0, key 70 5 a (a the query's, 0.8 .. 1.05), all others -30 a.  With w0 = exp(-5 a) <= 0.02 the first key's weight
    relative to the largest, rounded to bf16 (2^-8), and the others' at most kv exp(-28) < 2^-25:
    |o - ref| <= 2^-8 |ref| + (2^-8 w0 + 2^-18) 2 max|v|."""
    H, Hkv, page = 4, 2, 16
    c, T = make([(n, kv)], Hkv, HD, page, seed=25)
    _, _, table = lists(c)
    c["k_cache"].zero_()
    c["k_cache"][..., 0] = -30.0
    for j, x in ((0, 0.0), (70, 5.0)):
        c["k_cache"][table[0, j // page], j % page, :, 0] = x
    q = torch.zeros((T, H, HD), dtype=BF, device=DEV)
    q[..., 0] = torch.linspace(0.8, 1.05, T * H, device=DEV).view(T, H).to(BF)
    o, _ = B.lr_attention_paged_fwd(q.view(T, -1), H=H, scale=1.0, **c)
    torch.cuda.synchronize()
    k, v = (x.double().view(kv, Hkv, HD) for x in _dense(c, 0, kv))
    limit = torch.arange(kv - n, kv, device=DEV)
    rows = limit >= 70                               # tokens that see the key
    for h in range(H):
        s = q[:, h, 0].double()[:, None] * k[None, :, h // 2, 0]
        w = torch.softmax(s.masked_fill(torch.arange(kv, device=DEV)[None] > limit[:, None], float("-inf")), 1)
        ref, a = w @ v[:, h // 2].contiguous(), q[:, h, 0].double()[:, None]
        err = (o[:, h * HD:(h + 1) * HD].double() - ref).abs()
        bound = 2.0 ** -8 * ref.abs() + (2.0 ** -8 * torch.exp(-5 * a) + 2.0 ** -18) * 2 * v.abs().max()
        assert bool((err <= bound)[rows].all()), (h, float((err / bound)[rows].max()))


# ---- dimensions of one ------------------------------------------------------------------------------------------
def _one_row(t, pad=0):
    """The values of t [1, n] in a tensor whose row stride is 1, as a turned column has it."""
    out = torch.zeros((t.shape[1] + pad, 1), dtype=t.dtype, device=t.device).t()
    out[:, :t.shape[1]] = t
    assert out.stride() == (1, 1)
    return out


def test_one_token_with_any_row_stride():
    H, Hkv = 4, 2
    g = torch.Generator(device=DEV).manual_seed(27)
    q, k, v = (torch.randn((1, w * HD), generator=g, device=DEV).to(BF) for w in (H, Hkv, Hkv))
    rope = B.lr_rope_table(64, HD, device=DEV)
    got = []
    for row in (lambda t: t, _one_row, lambda t: _one_row(t, 3)):
        c, _ = make([(1, 40)], Hkv, HD, 16, seed=27)
        out = row(torch.zeros_like(q))
        qr = B.lr_kv_append(row(k), row(v), rope=rope, q=row(q), H=H, q_out=out, **c)
        turned = B.lr_rope_at(row(q), *rope, H, HD, pos=torch.full((1,), 39, dtype=torch.int32, device=DEV), out=row(torch.zeros_like(q)))
        place = row(q.clone())
        B.lr_rope_at(place, *rope, H, HD, pos=torch.full((1,), 39, dtype=torch.int32, device=DEV), out=place)
        o, lse = B.lr_attention_paged_fwd(qr, H=H, o=row(torch.zeros_like(q)), **c)
        torch.cuda.synchronize()
        assert qr.data_ptr() == out.data_ptr()
        got.append([c["k_cache"], c["v_cache"], qr[:, :H * HD], turned[:, :H * HD], place[:, :H * HD], o[:, :H * HD], lse])
    assert torch.equal(got[0][3], got[0][2])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_one_page_and_one_head_with_any_stride():
    """Turned dimensions of one: the bits of the plain cache."""
    g = torch.Generator(device=DEV).manual_seed(28)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    for pages, heads in ((1, 2), (4, 1)):
        plain = [torch.randn((pages, 48, heads, HD), generator=g, device=DEV).to(BF) for _ in range(2)]
        lens = {"page_table": i32([list(range(pages))[::-1]]), "cu_q": i32([0, 3]), "kv_len": i32([48 * pages - 5])}
        k, v, q = (torch.randn((3, w * HD), generator=g, device=DEV).to(BF) for w in (heads, heads, 4))
        dim, got = (0 if pages == 1 else 2), []
        for turn in (False, True):
            caches = [x.clone() for x in plain]
            if turn:
                caches = [torch.stack([x.select(dim, 0)], -1).movedim(-1, dim) for x in caches]
                assert caches[0].stride(dim) == 1
                caches[1] = plain[1].clone()                       # strides of its own
            c = {"k_cache": caches[0], "v_cache": caches[1], **lens}
            B.lr_kv_append(k, v, **c)
            o, lse = B.lr_attention_paged_fwd(q, H=4, **c)
            torch.cuda.synchronize()
            got.append([o, lse, *caches])
        assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("seqs", [[(1, 300), (3, 70)], [(150, 150)], [(200, 1500)]])
def test_rows_whose_logits_are_all_minus_infinity(seqs):
    """They are as rows without keys; beside them, rows that see one finite key are its value."""
    H, Hkv, page = 4, 2, 16
    c, T = make(seqs, Hkv, HD, page, seed=29)
    _, _, table = lists(c)
    n, kv = seqs[0]
    last = tuple(torch.tensor(x, device=DEV) for x in (table[0, (kv - 1) // page], (kv - 1) % page))
    c["k_cache"].zero_()
    c["k_cache"][..., 0] = float("-inf")
    c["k_cache"][last[0], last[1], :, 0] = 2.0          # the last key of the first sequence
    q = torch.zeros((T, H, HD), dtype=BF, device=DEV)
    q[..., 0] = 1.0
    o, lse = B.lr_attention_paged_fwd(q.view(T, -1), H=H, **c)
    torch.cuda.synchronize()
    v = c["v_cache"][last].repeat_interleave(H // Hkv, 0)
    seen = torch.arange(T, device=DEV) == n - 1
    assert torch.equal(o[seen].view(H, HD), v) and bool((lse[seen] - 2 * HD ** -0.5).abs().max() < 2.0 ** -20)
    assert bool((o[~seen] == 0).all()) and bool(lse[~seen].isneginf().all())
