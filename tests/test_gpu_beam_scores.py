"""Scores and the order of beams in beam search's choice are those of 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def chosen(logits, score, n):
    return [t.cpu().numpy() for t in B.lr_beam_select(logits, score, n)]


def sharp(row):
    """log sum exp of fp64 logits, each step rounded by half a last place at most."""
    most = row.max()
    return most, math.log(math.fsum(np.exp(row - most)))


def slack(V, most):
    """How far a score may be from its definition.  An exponential: its exponent, of which most * log2(e) is rounded (2^-53 |most|), the polynomial and its
    steps (2^-51).  A sum: as many roundings as a lane adds numbers, V / 64 and a few.  The logarithm of at least one and three sums of numbers below 64:
    2^-53 of them each."""
    return 2.0 ** -53 * (abs(most) + V / 64 + 100 + 4 + 4 * 64)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,scale", [(3, 1.0), (500, 3.0), (4100, 2.5), (32000, 2.5), (131072, 1.0), (32000, 0.01)])
def test_scores_are_those_of_64_bits(V, scale, dtype):
    """Scores that are next to zero, where the rounding to fp32 hides nothing: the old one is log sum exp - largest, rounded."""
    g = torch.Generator(device=DEV).manual_seed(V)
    rows = 24
    logits = (torch.randn((rows, V), generator=g, device=DEV) * scale).to(dtype)
    x = logits.double().cpu().numpy()
    score = torch.tensor([[sharp(row)[1]] for row in x], dtype=F32)
    best = chosen(logits, score.to(DEV), 1)[2][:, 0].astype(np.float64)
    for b in range(rows):
        most, rest = sharp(x[b])
        want = float(score[b, 0]) - rest
        assert abs(best[b] - want) <= 2.0 ** -24 * abs(want) + slack(V, most), (b, best[b] - want)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_beams_closer_than_a_part_in_ten_thousand_millions(dtype):
    """64 beams whose best candidates differ by 1e-7 at most, neighbours by less than 1e-10 here and there: they come in the order of 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(3)
    V, prompts = 1000, 40
    logits = (torch.randn((prompts * 64, V), generator=g, device=DEV) * 2.5).to(dtype)
    top = logits.argmax(1, keepdim=True)
    logits.scatter_add_(1, top, torch.full_like(top, 0.125, dtype=dtype))      # (one best candidate of a beam)
    x = logits.double().cpu().numpy()
    rest = np.array([sharp(row) for row in x])
    score = torch.tensor(rest[:, 1], dtype=F32).view(prompts, 64)
    value = score.double().numpy() - rest[:, 1].reshape(prompts, 64)
    gap = np.diff(np.sort(value, axis=1), axis=1)
    limit = 2 * slack(V, np.abs(x).max())
    assert np.sum((gap < 1e-10) & (gap > limit)) > 10
    parent = chosen(logits, score.to(DEV), 64)[0]
    for b in range(prompts):
        order = value[b][parent[b] - 64 * b]
        assert sorted(parent[b] - 64 * b) == list(range(64)) and np.all(order[:-1] >= order[1:] - limit), b
