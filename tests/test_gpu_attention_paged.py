"""Attention over the pages of a cache against the fp64 oracle, element by element.

Bounds, for an output o = sum_j w_j v_j with softmax weights w: a score is a sum of 128 products in 32 bits, off by at most
d = 128 * 2^-24 of its products' magnitudes, and its exponential by some steps more; a weight may be rounded to bf16 before the
product with v (half a step, 2^-8); o is rounded once when it is stored.  So |got - o| <= 2^-8 |o| + (2^-8 + 2 d + 2^-18) sum_j w_j |v_j|,
and lse is off by at most d plus some steps of 32 bits of its size and one for each key that is summed up."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2512_12131_amd import binding as B
from test_gpu_kv_append import BF, DEV, lists, make, np64

pytestmark = pytest.mark.gpu
HD = 128


def compare(o, lse, q, c, H, scale=HD ** -0.5, o0=7.0):
    T = q.shape[0]
    cu, kv_len, table = lists(c)
    clean = lambda t: np.nan_to_num(np64(t), nan=0.0, posinf=0.0, neginf=0.0)      # (where a test put something else, no token may see it)
    ref, lse_ref, mag, dots = po.attention_paged(np64(q[:, :H * HD]).reshape(T, H, HD), clean(c["k_cache"]), clean(c["v_cache"]), table, cu, kv_len, H,
                                                 scale)
    got, got_lse = np64(o[:, :H * HD]).reshape(T, H, HD), np64(lse)
    nobody = np.isnan(lse_ref)
    assert (got[nobody] == o0).all() and (got_lse[nobody] == o0).all()
    none = np.isneginf(lse_ref)
    assert (got[none] == 0).all() and np.isneginf(got_lse[none]).all()
    m = ~nobody & ~none
    if not m.any():
        return
    d = 128 * 2.0 ** -24 * dots[m]
    err = np.abs(got[m] - ref[m])
    bound = 2.0 ** -8 * np.abs(ref[m]) + (2.0 ** -8 + 2 * d + 2.0 ** -18)[:, None] * mag[m]
    assert (err <= bound).all(), f"o: {float((err / bound).max()):.2f} of its bound"
    keys = c["page_table"].shape[1] * c["k_cache"].shape[1]
    lerr = np.abs(got_lse[m] - lse_ref[m])
    assert (lerr <= d + 2.0 ** -20 * (1 + np.abs(lse_ref[m])) + keys * 2.0 ** -24).all(), float(lerr.max())


def call(c, T, H, pad=0, scale=None, seed=5, std=2.0, **kw):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (torch.randn((T, H * HD + pad), generator=g, device=DEV) * std).to(BF)
    o = torch.full((T, H * HD + 2 * pad), 7.0, dtype=BF, device=DEV)
    lse = torch.full((T, H), 7.0, device=DEV)
    B.lr_attention_paged_fwd(q, H=H, scale=scale, o=o, lse=lse, **c, **kw)
    torch.cuda.synchronize()
    return q, o, lse


CASES = [
    # (new tokens, keys) of the sequences, H, Hkv, page, layout, tokens of nobody in front and behind
    ([(1, 1)], 1, 1, 16, "token", 0, 0),
    ([(1, n) for n in (2, 7, 8, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257)], 4, 2, 16, "token", 0, 3),
    ([(1, 777)], 32, 8, 16, "token", 0, 0),
    ([(1, 3001), (1, 12), (0, 40), (1, 1999), (0, 0)], 8, 1, 48, "head", 1, 2),
    ([(2, 500), (4, 77), (3, 3), (1, 1300)], 6, 2, 24, "wide", 0, 0),             # a few tokens each, groups of 3
    ([(8, 200), (9, 300), (7, 7)], 16, 4, 8, "token", 0, 0),                      # rows around a tile of 32
    ([(1, 90)] * 130, 2, 2, 32, "token", 2, 0),                                   # more sequences than lanes
    ([(40, 40), (33, 100), (64, 64)], 4, 4, 16, "token", 0, 5),                   # prompts, every head its own keys
    ([(131, 131), (1, 260), (63, 700)], 8, 2, 64, "head", 3, 1),                  # mixed
    ([(257, 300)], 5, 1, 40, "token", 0, 0),                                      # groups of 5: tokens that straddle tiles
    ([(96, 611)], 7, 1, 128, "wide", 0, 0),
    ([(130, 1500)], 16, 16, 24, "token", 0, 0),
    ([(200, 5)], 4, 2, 16, "token", 0, 0), ([(3, 1), (2, 0), (5, -4)], 4, 1, 16, "token", 0, 0),    # rows that see nothing
    ([(2, 70)], 40, 1, 16, "token", 0, 0), ([(1, 70)], 64, 1, 16, "token", 0, 0),                   # more heads in a group than a tile has rows
    ([(1, 400), (2, 517), (1, 64)] * 24, 2, 2, 16, "head", 0, 1),                 # split, and more sequences than lanes
    ([(60, 1200), (1, 900), (40, 70)], 3, 1, 32, "token", 1, 0),                  # split, an odd number of heads
    ([(140, 260), (30, 1100)], 4, 2, 8, "wide", 0, 2),                            # splits behind all keys of the first blocks
]


@pytest.mark.parametrize("seqs,H,Hkv,page,layout,lead,tail", CASES)
def test_against_the_oracle(seqs, H, Hkv, page, layout, lead, tail):
    print(f"paged attention {seqs[:6]}.. H={H} Hkv={Hkv} page={page} {layout}", flush=True)
    c, T = make(seqs, Hkv, HD, page, layout, lead, tail, seed=H)
    q, o, lse = call(c, T, H, pad=8 * (H % 3))
    compare(o, lse, q, c, H)
    assert bool((o[:, H * HD:] == 7).all())
    again = call(c, T, H, pad=8 * (H % 3))                        # no order of arrival in any sum
    assert torch.equal(o, again[1]) and torch.equal(lse, again[2])


@pytest.mark.parametrize("scale,std", [(1.0, 1.0), (0.01, 2.0), (3.0, 2.0), (1e-30, 1.0)])
def test_scales(scale, std):
    """Logits up to some hundreds: one key takes it all; and all alike."""
    c, T = make([(1, 300), (20, 150)], 2, HD, 16, seed=2)
    q, o, lse = call(c, T, 4, scale=scale, std=std)
    compare(o, lse, q, c, 4, scale)


def test_one_row_of_large_logits_beside_small_ones():
    """The running maximum climbs from tile to tile, or the first key keeps it."""
    for order in (1.0, -1.0):
        c, T = make([(1, 640), (40, 640)], 1, HD, 32, seed=3)
        ramp = torch.linspace(-1, 1, 640, device=DEV) * order
        cu, kv, table = lists(c)
        for b in range(2):
            for j in range(640):
                c["k_cache"][table[b, j // 32], j % 32] = (ramp[j] * 3).to(BF)
        q, o, lse = call(c, T, 2, std=1.0)
        compare(o, lse, q, c, 2)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_lies_behind_the_keys_is_not_seen(bad):
    """Rows of the last page behind kv_len and pages of nobody hold anything."""
    for seqs, H, Hkv in (([(1, 37), (1, 64), (1, 130)], 4, 1), ([(3, 37), (20, 70), (70, 165)], 4, 2)):
        c, T = make(seqs, Hkv, HD, 32, seed=4)
        cu, kv, table = lists(c)
        keep = torch.zeros(c["k_cache"].shape[:2], dtype=torch.bool, device=DEV)
        for b, (_, n) in enumerate(seqs):
            for j in range(n):
                keep[table[b, j // 32], j % 32] = True
        c["k_cache"][~keep], c["v_cache"][~keep] = bad, bad
        q, o, lse = call(c, T, H)
        compare(o, lse, q, c, H)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_tokens_do_not_see_later_ones(bad):
    """A key and a value that are no numbers reach the tokens from their own on, not the ones before in the same chunk."""
    for seqs, H, Hkv, at in (([(5, 41)], 4, 1, 39), ([(150, 150)], 4, 2, 70), ([(150, 470)], 1, 1, 400), ([(40, 360), (1, 200)], 2, 2, 330)):
        c, T = make(seqs, Hkv, HD, 32, seed=4)
        cu, kv, table = lists(c)
        c["k_cache"][table[0, at // 32], at % 32] = bad
        c["v_cache"][table[0, at // 32], at % 32, :, ::3] = bad
        q, o, lse = call(c, T, H)
        before = at - (seqs[0][1] - seqs[0][0])           # tokens of the first sequence that don't see it
        assert 0 < before < seqs[0][0]
        short = {**c, "cu_q": torch.tensor([0, before], dtype=torch.int32, device=DEV), "kv_len": torch.tensor([at], dtype=torch.int32, device=DEV),
                 "page_table": c["page_table"][:1]}
        compare(o[:before], lse[:before], q[:before], short, H)
        seen = o[before:seqs[0][0]].float()
        assert bad == bad and bad < 0 or bool(seen.isnan().any(-1).all() | (seen.isinf().any(-1).all()))
        if len(seqs) > 1:
            assert bool(o[seqs[0][0]:].isfinite().all())


def test_pages_that_are_none_hold_zeros():
    c, T = make([(1, 100), (40, 100), (2, 64)], 2, HD, 16, seed=6)
    table = c["page_table"]
    table[0, 1], table[1, 0], table[2, 3], table[2, 2] = -1, 10 ** 9, -(1 << 31), c["k_cache"].shape[0]
    q, o, lse = call(c, T, 4)
    compare(o, lse, q, c, 4)


def test_lists_that_lead_nowhere():
    """Keys past the table's columns do not exist; bounds of sequences outside the tokens cover what tokens there are."""
    c, T = make([(1, 100), (40, 100)], 2, HD, 16, seed=7, extra_cols=0)
    c["kv_len"][0] = (1 << 31) - 1
    q, o, lse = call(c, T, 4)
    compare(o, lse, q, c, 4)
    c, T = make([(1, 100), (40, 100)], 2, HD, 16, seed=7)
    c["cu_q"][2] = 10 ** 9                     # not the lists of any batch: only that nothing faults
    call(c, T, 4)
    c["cu_q"][:] = torch.tensor([30, -5, 1 << 30], dtype=torch.int32)
    call(c, T, 4)
    c["kv_len"][:] = -(1 << 31)
    call(c, T, 4)


def test_far_pages():
    """Offsets past 2^32 bytes and 2^31 elements."""
    page, Hkv, n_pages = 256, 8, 10400
    g = torch.Generator(device=DEV).manual_seed(1)
    cache = torch.zeros((n_pages, page, Hkv, HD), dtype=BF, device=DEV)
    assert cache.numel() > 1 << 31
    used = [n_pages - 1, 3, 8200, n_pages - 2, 9000]
    cache[used] = torch.randn((len(used), page, Hkv, HD), generator=g, device=DEV).to(BF)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    far = {"k_cache": cache, "v_cache": cache, "page_table": i32([[n_pages - 1, 3, 8200], [n_pages - 2, 9000, 0]]), "cu_q": i32([0, 1, 41]),
           "kv_len": i32([700, 300])}
    near = {**far, "k_cache": cache[used].contiguous(), "page_table": i32([[0, 1, 2], [3, 4, 5]])}
    near["v_cache"] = near["k_cache"]
    a, b = call(far, 41, 16), call(near, 41, 16)
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    compare(b[1], b[2], b[0], {**near, "page_table": i32([[0, 1, 2], [3, 4, 0]])}, 16)


def _dense(c, b, n):
    _, _, table = lists(c)
    page = c["k_cache"].shape[1]
    rows = [(table[b, j // page], j % page) for j in range(n)]
    at = tuple(torch.tensor(x, device=DEV) for x in zip(*rows))
    return c["k_cache"][at].flatten(1).contiguous(), c["v_cache"][at].flatten(1).contiguous()


@pytest.mark.parametrize("H,Hkv", [(32, 8), (16, 16)])
def test_a_whole_prompt_is_the_dense_attention(H, Hkv):
    """lr_attention_gqa_fwd on the same keys and values, both within a bf16 step of the other's bound."""
    S = 1031
    c, T = make([(S, S)], Hkv, HD, 64, seed=8)
    q, o, lse = call(c, T, H)
    k, v = _dense(c, 0, S)
    o_ref, lse_ref = B.lr_attention_gqa_fwd(q[:, :H * HD].contiguous(), k, v, 1, S, H, Hkv, HD)
    torch.cuda.synchronize()
    assert float((lse - lse_ref[0].t()).abs().max()) < 1e-4
    rms = float(o_ref.float().square().mean().sqrt())
    assert float((o[:, :H * HD].float() - o_ref.float()).norm() / o_ref.float().norm()) < 2.0 ** -8
    assert float((o[:, :H * HD].float() - o_ref.float()).abs().max()) < 8 * rms * 2.0 ** -6


@pytest.mark.parametrize("interleaved", [False, True])
def test_prompt_in_chunks_then_tokens(interleaved):
    """Tables, append and attention as a server runs them: a prompt in chunks, then single tokens, two sequences side by side; every
    step's output against one causal attention over everything, with the rotation done by lr_rope_at."""
    H, Hkv, page, total = 8, 2, 16, (210, 135)
    g = torch.Generator(device=DEV).manual_seed(3)
    cos, sin = B.lr_rope_table(256, HD, factor=4.0, ramp=(64.0, 1.0, 8.0), device=DEV)
    qs, ks, vs = ([torch.randn((n, w * HD), generator=g, device=DEV).to(BF) for n in total] for w in (H, Hkv, Hkv))
    want = []
    for q, k, v, n in zip(qs, ks, vs, total):
        turned = [B.lr_rope_at(t, cos, sin, w, HD, interleaved=interleaved) for t, w in ((q, H), (k, Hkv))]
        want.append(B.lr_attention_gqa_fwd(turned[0], turned[1], v, 1, n, H, Hkv, HD)[0])
    cache = {"k_cache": torch.full((40, page, Hkv, HD), float("nan"), dtype=BF, device=DEV)}
    cache["v_cache"] = cache["k_cache"].clone()
    cache["page_table"] = torch.randperm(40, generator=g, device=DEV)[:28].to(torch.int32).view(2, 14).contiguous()
    at = [0, 0]
    for steps in ((100, 1), (37, 64), (70, 69), (1, 1), (1, 0), (1, 0)):
        cu = torch.tensor([0, steps[0], sum(steps)], dtype=torch.int32, device=DEV)
        new = [slice(a, a + n) for a, n in zip(at, steps)]
        at = [a + n for a, n in zip(at, steps)]
        lens = torch.tensor(at, dtype=torch.int32, device=DEV)
        q, k, v = (torch.cat([x[s] for x, s in zip(xs, new)]) for xs in (qs, ks, vs))
        qr = B.lr_kv_append(k, v, cu_q=cu, kv_len=lens, rope=(cos, sin), interleaved=interleaved, q=q, H=H, **cache)
        o, _ = B.lr_attention_paged_fwd(qr, cu_q=cu, kv_len=lens, H=H, **cache)
        torch.cuda.synchronize()
        ref = torch.cat([w[s] for w, s in zip(want, new)]).float()
        assert float((o.float() - ref).norm() / ref.norm()) < 2.0 ** -8, steps
    assert at == list(total)


def test_replayed_from_a_graph_with_other_lists():
    """Append and attention captured once for a padded batch of 4 sequences and 6 tokens, replayed for batches of other lengths; eager work
    between the replays."""
    H, Hkv, page, T = 8, 2, 16, 6
    g = torch.Generator(device=DEV).manual_seed(3)
    cos, sin = B.lr_rope_table(512, HD, device=DEV)
    c = {"k_cache": torch.randn((64, page, Hkv, HD), generator=g, device=DEV).to(BF), "v_cache": torch.randn((64, page, Hkv, HD), generator=g, device=DEV).to(BF),
         "page_table": torch.randperm(64, generator=g, device=DEV).to(torch.int32).view(4, 16).contiguous(),
         "cu_q": torch.zeros(5, dtype=torch.int32, device=DEV), "kv_len": torch.zeros(4, dtype=torch.int32, device=DEV)}
    x = torch.empty((T, (H + 2 * Hkv) * HD), dtype=BF, device=DEV)
    q, k, v = x[:, :H * HD], x[:, H * HD:(H + Hkv) * HD], x[:, (H + Hkv) * HD:]
    qo, o = (torch.empty((T, H * HD), dtype=BF, device=DEV) for _ in range(2))
    lse = torch.empty((T, H), device=DEV)
    ws = torch.empty(max(256, B.lr_attention_paged_workspace_bytes(c["k_cache"], c["page_table"], T, H)), dtype=torch.uint8, device=DEV)

    def step(cache):
        B.lr_kv_append(k, v, rope=(cos, sin), q=q, H=H, q_out=qo, **cache)
        B.lr_attention_paged_fwd(qo, H=H, o=o, lse=lse, ws=ws, **cache)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c)
    torch.cuda.synchronize()
    for cu, kv in (([0, 1, 2, 3, 4], [200, 1, 77, 16]), ([0, 3, 3, 6, 6], [3, 0, 250, 9]), ([0, 1, 1, 1, 1], [100, 0, 0, 0]), ([0, 1, 2, 3, 4], [201, 2, 78, 17])):
        c["cu_q"].copy_(torch.tensor(cu, dtype=torch.int32)), c["kv_len"].copy_(torch.tensor(kv, dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=g, device=DEV).to(BF))
        got = []
        for run in (graph.replay, lambda: step(c)):
            cache0 = c["k_cache"].clone(), c["v_cache"].clone()
            for t in (qo, o, lse):
                t.fill_(7)
            ws.fill_(0xFF)                      # nothing that another call left there is read
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            got.append([t.clone() for t in (c["k_cache"], c["v_cache"], qo, o, lse)])
            if run is graph.replay:
                c["k_cache"].copy_(cache0[0]), c["v_cache"].copy_(cache0[1])
        assert all(torch.equal(a, b) for a, b in zip(*got)), (cu, kv)
        compare(o, lse, qo, c, H)


def test_on_a_stream_of_its_own():
    c, T = make([(1, 900), (30, 300)], 2, HD, 16, seed=9)
    q, o, lse = call(c, T, 8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o2, lse2 = B.lr_attention_paged_fwd(q, H=8, **c)
    s.synchronize()
    assert torch.equal(o[:, :8 * HD], o2) and torch.equal(lse, lse2)


# Real sizes, in the long form of an item and with keys in many splits: (new tokens, keys) of the sequences, H, Hkv, page
@pytest.mark.parametrize("seqs,H,Hkv,page", [([(512, 8192)], 32, 8, 16), ([(1, 16384), (1, 300)], 32, 8, 48), ([(2047, 2047), (130, 900)], 8, 8, 64),
                                             ([(1, 4096)] * 6 + [(200, 4096), (77, 3000)], 32, 8, 16), ([(600, 5000)], 6, 1, 24),
                                             ([(1, 2500)] * 20 + [(300, 4096)] + [(1, 2500)] * 20, 8, 8, 16), ([(64, 3900), (1, 4000)] * 16, 16, 8, 32)])
def test_real_sizes(seqs, H, Hkv, page):
    """Against 64 bits on the GPU, every element; bounds as above."""
    print(f"paged attention {seqs} H={H} Hkv={Hkv} page={page}", flush=True)
    c, T = make(seqs, Hkv, HD, page, seed=11)
    q, o, lse = call(c, T, H)
    t0, grp = 0, H // Hkv
    for b, (n, kv) in enumerate(seqs):
        k, v = (x.double().view(kv, Hkv, HD) for x in _dense(c, b, kv))
        hidden = torch.arange(kv, device=DEV)[None] > torch.arange(kv - n, kv, device=DEV)[:, None]
        for h in range(H):
            qq, kk, vv = q[t0:t0 + n, h * HD:(h + 1) * HD].double(), k[:, h // grp].contiguous(), v[:, h // grp].contiguous()
            s = (qq @ kk.t().contiguous()) * HD ** -0.5
            d = 128 * 2.0 ** -24 * (qq.abs() @ kk.abs().t().contiguous() * HD ** -0.5).masked_fill(hidden, 0).amax(1)
            s = s.masked_fill(hidden, float("-inf"))
            l = torch.logsumexp(s, 1)
            w = torch.exp(s - l[:, None])
            ref, mag = w @ vv, w @ vv.abs()
            err = (o[t0:t0 + n, h * HD:(h + 1) * HD].double() - ref).abs()
            assert bool((err <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * d + 2.0 ** -18)[:, None] * mag).all()), (b, h)
            lerr = (lse[t0:t0 + n, h].double() - l).abs()
            assert bool((lerr <= d + 2.0 ** -20 * (1 + l.abs()) + kv * 2.0 ** -24).all()), (b, h, float(lerr.max()))
        t0 += n
    again = call(c, T, H)
    assert torch.equal(o, again[1]) and torch.equal(lse, again[2])


def test_sequences_that_share_pages():
    """A common beginning in the same pages, and a page twice in one row: as with copies of them."""
    H, Hkv, page = 8, 2, 16
    c, T = make([(1, 100), (40, 130), (3, 64)], Hkv, HD, page, seed=12, extra_pages=30)
    table = c["page_table"].clone()
    table[1, :4], table[2, :4], table[1, 6] = table[0, :4], table[0, :4], table[1, 5]
    q, o, lse = call({**c, "page_table": table}, T, H)
    compare(o, lse, q, {**c, "page_table": table}, H)
    copies, free = table.clone(), [i for i in range(c["k_cache"].shape[0]) if i not in table.flatten().tolist()]
    for at in [(1, j) for j in range(4)] + [(2, j) for j in range(4)] + [(1, 6)]:
        to = free.pop()
        for x in (c["k_cache"], c["v_cache"]):
            x[to] = x[int(table[at])]
        copies[at] = to
    _, o2, lse2 = call({**c, "page_table": copies}, T, H)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_two_graphs_on_one_workspace():
    """Replayed in turn: what the other left in the workspace is not read."""
    H, Hkv = 8, 2
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    runs = []
    for seqs, seed in (([(1, 3000), (1, 500)], 13), ([(70, 1500), (2, 900)], 14)):
        c, T = make(seqs, Hkv, HD, 16, seed=seed)
        q, o, lse = call(c, T, H)
        out, out_lse = torch.zeros_like(o), torch.zeros_like(lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.lr_attention_paged_fwd(q, H=H, o=out, lse=out_lse, ws=ws, **c)
        runs.append((graph, out, out_lse, o, lse, c, q))
    for k in (0, 1, 0, 0, 1, 1, 0):
        graph, out, out_lse, o, lse, _, _ = runs[k]
        out.zero_(), out_lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(out_lse, lse), k


def test_a_workspace_of_the_size_asked_for_is_enough():
    for seqs, H, Hkv in (([(1, 3000)], 8, 2), ([(40, 2000), (1, 10)], 8, 8), ([(1, 500)] * 3, 4, 4)):
        c, T = make(seqs, Hkv, HD, 16, seed=10)
        size = B.lr_attention_paged_workspace_bytes(c["k_cache"], c["page_table"], T, H)
        buf = torch.full((size + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
        q, o, lse = call(c, T, H, ws=buf[:size])
        assert bool((buf[size:] == 0x5A).all())
        compare(o, lse, q, c, H)
        if size:
            with pytest.raises(B.LrError, match="LR_EWORKSPACE"):
                B.lr_attention_paged_fwd(q, H=H, ws=buf[:size - 256], **c)
