"""Steps of a beam search as a server runs them: the last hidden rows as 8-bit integers, their product with the vocabulary, the choice over beams
and vocabulary, the page tables of the beams that go on, copies of half filled pages, the new tokens' keys and values, attention and a bottleneck
layer of 8-bit integers.

Keys, values and queries are functions of token and position alone, so a beam's whole cache can be laid out again from its tokens: attention over
the forked pages has to give the same bits as over a cache that never shared a page, and so has everything behind it."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
H, HKV, HD, PAGE, COLS, V, MOST = 4, 2, 128, 16, 9, 1003, 128


def i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32, device=DEV)


class Model:
    def __init__(self, seed, rank=72):
        g = torch.Generator(device=DEV).manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device=DEV)
        self.token = {n: randn(V, h * HD) for n, h in (("q", H), ("k", HKV), ("v", HKV))}
        self.place = {n: randn(MOST, h * HD) for n, h in (("q", H), ("k", HKV), ("v", HKV))}
        d = H * HD
        self.layer = (*B.lr_quant_rows(randn(rank, d)), *B.lr_quant_rows(randn(d, rank) / 8))
        self.words = B.lr_quant_rows(randn(V, d) / 16)

    def rows(self, name, token, place):
        return (self.token[name][token.long()] + self.place[name][place.long()]).to(BF)

    def logits(self, o):
        hidden = o + B.lr_linear_q8_fwd(o, *self.layer)
        return B.lr_matmul_q8(*B.lr_quant_rows(hidden), *self.words, dtype=torch.float32)


def afresh(m, history, pages_of):
    """Attention of every beam's last token over a cache of its own."""
    n = [len(h) for h in history]
    cu, cols = np.concatenate([[0], np.cumsum(n)]), -(-max(n) // PAGE)
    table = i32(pages_of[:len(n) * cols].reshape(len(n), cols))
    k, v = (torch.zeros((len(pages_of), PAGE, HKV, HD), dtype=BF, device=DEV) for _ in range(2))
    token, place = i32(np.concatenate(history)), i32(np.concatenate([np.arange(i) for i in n]))
    B.lr_kv_append(m.rows("k", token, place), m.rows("v", token, place), k, v, table, i32(cu), i32(n))
    last = i32([h[-1] for h in history])
    one = i32(np.arange(len(n) + 1))
    return B.lr_attention_paged_fwd(m.rows("q", last, i32(n) - 1), k, v, table, one, i32(n), H)[0]


@pytest.mark.parametrize("prompts,beams,steps", [([5, 37, 16], 4, 24), ([1], 1, 18), ([31, 2], 3, 40)])
def test_beam_search_over_forked_pages(prompts, beams, steps):
    rng = np.random.default_rng(sum(prompts))
    m, G, pages = Model(sum(prompts)), len(prompts), 400
    n = G * beams
    k, v = (torch.full((pages, PAGE, HKV, HD), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    refs, table, length = i32(np.zeros(pages)), i32(np.full((1, COLS), -1)), i32([0])
    history = [rng.integers(0, V, p) for p in prompts]
    # the prompts: one sequence each
    refs, table, length, copies, missing = B.lr_kv_fork(refs, PAGE, table, length, i32([-1] * G), i32(prompts))
    token, place = i32(np.concatenate(history)), i32(np.concatenate([np.arange(p) for p in prompts]))
    B.lr_kv_append(m.rows("k", token, place), m.rows("v", token, place), k, v, table, i32(np.concatenate([[0], np.cumsum(prompts)])), length)
    o = B.lr_attention_paged_fwd(m.rows("q", i32([h[-1] for h in history]), length - 1), k, v, table, i32(np.arange(G + 1)), length, H)[0]
    score = torch.zeros((G, 1), device=DEV)
    for step in range(steps):
        logits = m.logits(o)
        # (done: the first prompt's first beam has ended from the seventh step on and repeats its last token)
        done = torch.zeros(score.shape, dtype=torch.int32, device=DEV)
        done[0, 0] = int(step > 6)
        parent, token, best = B.lr_beam_select(logits, score, beams, done=done, done_token=3)
        want = so.beam_select(logits.double().cpu().numpy(), score.double().cpu().numpy(), beams, done.cpu().numpy(), 3)
        assert np.array_equal(parent.cpu().numpy(), want[0]) and np.array_equal(token.cpu().numpy(), want[1]), step
        score, parent, token = best, parent.view(-1), token.view(-1)
        history = [np.append(history[p], t) for p, t in zip(parent.tolist(), token.tolist())]
        refs, table, length, copies, missing = B.lr_kv_fork(refs, PAGE, table, length, parent, i32(np.ones(n)))
        assert int(missing) == 0 and length.tolist() == [len(h) for h in history]
        B.lr_kv_copy(k, v, *copies)
        B.lr_kv_append(m.rows("k", token, length - 1), m.rows("v", token, length - 1), k, v, table, i32(np.arange(n + 1)), length)
        o = B.lr_attention_paged_fwd(m.rows("q", token, length - 1), k, v, table, i32(np.arange(n + 1)), length, H)[0]
        if step % 8 == 5 or step == steps - 1:
            fresh = afresh(m, history, rng.permutation(pages))
            assert torch.equal(o, fresh) and torch.equal(m.logits(o), m.logits(fresh)), step
        if step % 8 == 3:                                       # the pages in use to the front
            refs, table, moves, _, live = B.lr_kv_compact(refs, table)
            B.lr_kv_copy(k, v, *moves)
            held = int(live)
            k[held:], v[held:] = float("nan"), float("nan")
            assert not refs[held:].any() and refs[:held].all()
            assert torch.equal(o, B.lr_attention_paged_fwd(m.rows("q", token, length - 1), k, v, table, i32(np.arange(n + 1)), length, H)[0]), step
    # all sequences end
    refs = B.lr_kv_fork(refs, PAGE, table, length, i32([]), i32([]))[0]
    assert not refs.any()


def test_captured_step_of_beams():
    """One captured step from hidden rows to attention, replayed 20 times with the new lists written back over the old ones, against eager steps."""
    G, beams, pages, n = 2, 3, 200, 6
    m = Model(7)
    rng = np.random.default_rng(7)
    refs, table, length, _, _ = B.lr_kv_fork(i32(np.zeros(pages)), PAGE, i32(np.full((1, COLS), -1)), i32([0]), i32([-1] * n), i32([9] * n))
    k, v = (torch.zeros((pages, PAGE, HKV, HD), dtype=BF, device=DEV) for _ in range(2))
    token, place = i32(rng.integers(0, V, 9 * n)), i32(np.tile(np.arange(9), n))
    B.lr_kv_append(m.rows("k", token, place), m.rows("v", token, place), k, v, table, i32(np.arange(n + 1) * 9), length)
    ones, cu = i32(np.ones(n)), i32(np.arange(n + 1))
    o = B.lr_attention_paged_fwd(m.rows("q", token[8::9], length - 1), k, v, table, cu, length, H)[0]
    score = torch.randn((G, beams), device=DEV)
    state = [refs, table, length, k, v, o, score]

    def step(refs, table, length, k, v, o, score):
        parent, token, best = B.lr_beam_select(m.logits(o), score)
        refs_, table_, length_, copies, _ = B.lr_kv_fork(refs, PAGE, table, length, parent.view(-1), ones)
        B.lr_kv_copy(k, v, *copies)
        token = token.view(-1)
        B.lr_kv_append(m.rows("k", token, length_ - 1), m.rows("v", token, length_ - 1), k, v, table_, cu, length_)
        o_ = B.lr_attention_paged_fwd(m.rows("q", token, length_ - 1), k, v, table_, cu, length_, H)[0]
        for t, new in ((refs, refs_), (table, table_), (length, length_), (o, o_), (score, best)):
            t.copy_(new)

    captured = [t.clone() for t in state]
    step(*[t.clone() for t in state])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    for turn in range(20):
        graph.replay()
        step(*state)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, state)), turn
