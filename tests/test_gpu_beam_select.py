"""Beam search's choice against the fp64 oracle: parents and tokens are equal, scores are rounded once."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")


def check(logits, score, n, done=None, done_token=0):
    got = B.lr_beam_select(logits, score, n, done=done, done_token=done_token)
    parent, token, best = so.beam_select(logits.double().cpu().numpy(), score.double().cpu().numpy(), n, None if done is None else done.cpu().numpy(), done_token)
    assert np.array_equal(got[0].cpu().numpy(), parent), (got[0].cpu().numpy(), parent)
    assert np.array_equal(got[1].cpu().numpy(), token)
    g = got[2].double().cpu().numpy()
    fin = np.isfinite(best)
    assert np.array_equal(fin, np.isfinite(g))
    # every exponential is within 6e-11 of it, of its size, and so is their sum; the logarithm of a sum of at least one is then off by at most 6e-11, and the
    # roundings of 64 bits add less than 1e-11 here; then one rounding to fp32
    assert np.all(np.abs(g[fin] - best[fin]) <= 2.0 ** -24 * np.abs(best[fin]) + 7e-11)


def make(batch, beams, V, dtype, seed, ld=None, scale=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    logits = (torch.randn((batch * beams, ld or V), generator=g, device=DEV) * scale).to(dtype)[:, :V]
    return logits, -20 * torch.rand((batch, beams), generator=g, device=DEV)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("batch,beams,V,n", [(1, 1, 1, 1), (1, 1, 5, 5), (2, 3, 7, 25), (1, 4, 32000, 4), (3, 5, 1000, 10), (2, 8, 50257, 16), (5, 2, 2047, 1), (4, 4, 2049, 8),
                                             (1, 64, 300, 64), (2, 16, 4096, 64), (1, 2, 1 << 20, 4), (300, 4, 777, 4), (700, 8, 4100, 8), (0, 4, 100, 4)])
def test_select(batch, beams, V, n, dtype):
    check(*make(batch, beams, V, dtype, seed=V + n), n)


@pytest.mark.parametrize("dtype,ld,first", [(BF, 1003, 0), (BF, 1003, 3), (F32, 1001, 1), (BF, 1008, 0), (F32, 2000, 5), (BF, 1009, 8)])
def test_rows_that_start_anywhere(dtype, ld, first):
    wide, score = make(3, 4, ld, dtype, seed=ld)
    check(wide[:, first:first + 995], score, 6)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_equal_candidates_go_by_beam_and_token(dtype):
    logits = torch.zeros((8, 3000), dtype=dtype, device=DEV)
    check(logits, torch.zeros((2, 4), device=DEV), 5)                          # everything is alike
    check(logits, torch.zeros((2, 4), device=DEV), 64)
    logits[:, 100::7] = 1                                                      # some hundred are
    logits[3, 2999] = -0.0
    check(logits, torch.zeros((2, 4), device=DEV), 20)
    row = make(1, 1, 5000, dtype, 3)[0]
    check(row.repeat(6, 1), torch.full((2, 3), -1.5, device=DEV), 9)           # beams alike: the first one's


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1, 7, 1003, 2051, 50257])
def test_beams_of_the_same_logits_stay_equal_at_any_alignment(dtype, V):
    """Every beam has the same logits and score, in rows that each start elsewhere against 16 bytes: sums are the same, so the order is by token and beam."""
    row = torch.randn(V, generator=torch.Generator(device=DEV).manual_seed(V), device=DEV) * 3
    row[V // 2:V // 2 + 2] = row.max()
    logits = row.to(dtype).repeat(6, 1)
    score = torch.full((2, 3), -1.5, device=DEV)
    check(logits, score, min(7, 3 * V))
    parent, token, best = (t.cpu().numpy() for t in B.lr_beam_select(logits, score, min(6, 3 * V)))
    for b in range(2):
        for value in set(best[b]):                                    # equal scores: the beams in order, each with its tokens in order
            at = [(parent[b, i], token[b, i]) for i in range(len(best[b])) if best[b, i] == value]
            assert at == sorted(at)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [4, 64])
def test_orders_that_are_worst(dtype, n):
    up = torch.arange(20000, device=DEV).float() / 500
    for row in (up, up.flip(0), up % 1, (up * 50).round()):
        check(row.to(dtype).repeat(4, 1), torch.tensor([[-1.0, -2.0, -3.0, -4.0]], device=DEV), n)


def test_masked_logits_and_beams():
    logits, score = make(4, 3, 6000, BF, 11)
    logits[0, 10:] = -INF                                                      # ten tokens allowed
    logits[1] = -INF                                                           # none
    logits[2, :5990] = torch.finfo(BF).min                                     # the lowest value is no mask
    score[1] = torch.tensor([0.0, -INF, -INF])                                 # a first step
    score[2, 0], score[2, 1] = float("nan"), INF
    logits[9, 77], logits[10, 4000] = float("nan"), INF
    for n in (3, 8, 64):
        check(logits, score, n)
    score[3] = -INF
    check(logits, score, 3)
    logits[:3] = -INF
    logits[0, 5999] = 0.0                                                      # one candidate for a prompt
    check(logits, score, 3)


def test_ended_beams():
    logits, score = make(3, 4, 5000, BF, 12)
    done = torch.tensor([[0, 1, 0, 0], [1, 1, 1, 1], [0, 0, 0, 2]], dtype=torch.int32, device=DEV)
    score[0, 1] = -0.5
    logits[1] = float("nan")                                                   # (an ended beam's logits are not looked at)
    score[1, 2] = -INF
    for token in (0, 2, 4999):
        check(logits, score, 6, done, token)
    check(logits, score, 4, torch.zeros_like(done))


def test_far_apart_logits():
    """Sums whose reference is left far behind, and logits that differ by more than an exponent holds."""
    logits, score = make(2, 2, 40000, F32, 13)
    logits[0, 30000], logits[0, 39999] = 5000.0, 5001.0
    logits[1] *= 1e30
    logits[2] = torch.arange(40000, device=DEV) * 0.5
    logits[3] = -1e38
    logits[3, 17] = -0.9e38
    check(logits, score, 4)


def test_shared_workspace_graphs_and_streams():
    """Two captured calls on one workspace, replayed in turn with other inputs and eager calls between; another stream."""
    a, b = make(2, 4, 9000, BF, 21), make(3, 2, 3000, F32, 22)
    nb = max(B.lr_beam_select_workspace_bytes(2, 4, 9000, 8), B.lr_beam_select_workspace_bytes(3, 2, 3000, 5))
    ws = torch.full((nb + 256,), 99, dtype=torch.uint8, device=DEV)
    outs, graphs = [], []
    for (x, s), n in ((a, 8), (b, 5)):
        outs.append(B.lr_beam_select(x, s, n, ws=ws[:nb]))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.lr_beam_select(x, s, n, out=outs[-1], ws=ws[:nb])
        graphs.append(graph)
    for turn in range(3):
        for (x, s), n, out, graph in zip((a, b), (8, 5), outs, graphs):
            x.copy_(torch.randn(x.shape, device=DEV))
            s.uniform_(-9, 0)
            graph.replay()
            want = B.lr_beam_select(x, s, n)
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(out, want)), turn
    assert bool((ws[nb:] == 99).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.lr_beam_select(a[0], a[1], 8)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, B.lr_beam_select(a[0], a[1], 8)))


def test_scores_are_written_over_the_old_ones():
    """score itself as the new scores, where each prompt has as many."""
    logits, score = make(40, 6, 3001, BF, 31)
    want = B.lr_beam_select(logits, score)
    out = (torch.empty_like(want[0]), torch.empty_like(want[1]), score)
    got = B.lr_beam_select(logits, score, out=out)
    assert got[2].data_ptr() == score.data_ptr() and all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(B.LrError):
        B.lr_beam_select(logits[:120], score[:20], out=tuple(t.view(40, 6)[10:30] for t in out))


def test_offsets_past_32_bits():
    """More than 2^31 logits: the last prompts' choices are those of the prompts alone."""
    batch, beams, V = 700, 4, 800000
    g = torch.Generator(device=DEV).manual_seed(41)
    logits = torch.randint(-20000, 20000, (batch * beams, V // 8), generator=g, device=DEV, dtype=torch.int16)
    logits = (logits.to(BF) / 4096).repeat(1, 8)
    logits[:, V // 2] = 9
    assert logits.numel() > 2 ** 31
    score = torch.randn((batch, beams), generator=g, device=DEV)
    got = B.lr_beam_select(logits, score)
    for p in (0, 350, batch - 1):
        alone = B.lr_beam_select(logits[p * beams:(p + 1) * beams].clone(), score[p:p + 1])
        assert torch.equal(got[0][p] - p * beams, alone[0][0]) and torch.equal(got[1][p], alone[1][0])
        assert float((got[2][p] - alone[2][0]).abs().max()) <= 2.0 ** -23 * 64      # (other runs, another order of the sum: neighbouring roundings)
