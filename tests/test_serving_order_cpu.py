"""Pins of the oracle's order of a choice."""
import numpy as np

from oracle import serving_oracle as so


def test_one_score_of_several_logits():
    """Logits whose difference the score can't hold come in their own order; equal ones by token; beams of one score one after the other."""
    logits = np.array([[0.0, 1e-20, -0.0, 1e-20], [5e-21, 0.0, 0.0, 2e-20]])
    for score in (0.0, -1e9, -1e20):
        for n in range(1, 9):
            parent, token, best = so.beam_select(logits, np.full((1, 2), score), n)
            assert parent[0].tolist() == [0, 0, 0, 0, 1, 1, 1, 1][:n] and token[0].tolist() == [1, 3, 0, 2, 3, 0, 1, 2][:n]
            assert np.all(best == score - np.log(4.0))
