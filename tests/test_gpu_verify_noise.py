"""grid_verify with random numbers outside their distributions: tokens stay in the vocabulary and among the allowed."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_verify import G, Case  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 400, 9000])
@pytest.mark.parametrize("noise", [math.inf, math.nan])
def test_noise_that_leaves_no_token(G, noise, V, dtype):
    """a refused draft is no answer unless it is allowed: ids outside the vocabulary, far and near, and masked ones"""
    c = Case(6, 1, V, dtype, seed=V, share=0.5, probs=False, ragged=False)
    c.bits[:, :, :2] = True
    c.bits[3:5, 0, V - 1] = False
    c.noise[:] = noise
    c.uniform[:] = 2.0  # no draft is accepted
    c.draft[:, 0] = [V, 1 << 30, -(1 << 31), V - 1, V - 1, 1]
    tokens, accepted, logprobs = c.run(G)
    assert accepted.tolist() == [0] * 6
    assert tokens.tolist() == [[-1, -1]] * 5 + [[1, -1]]
    assert (logprobs[:5] == 0).all() and np.isfinite(logprobs).all()


def test_a_refused_draft_that_was_all(G):
    """uniform numbers of 1 and more refuse even certain drafts; the only allowed token is the answer all the same"""
    c = Case(4, 2, 700, "f32", seed=3, share=0.5, probs=False, ragged=False)
    c.bits[:] = False
    c.bits[:, 0, 77], c.bits[:, 1, 78] = True, True
    c.bits[:, 2] = True
    c.draft[:] = [77, 78]
    c.uniform[:] = np.array([[1.0, 0.5], [0.5, 1.0], [0.5, 0.5], [7.0, 7.0]], np.float32)
    tokens, accepted, logprobs = c.run(G)
    assert accepted.tolist() == [0, 1, 2, 0]
    assert tokens[0].tolist() == tokens[3].tolist() == [77, -1, -1] and tokens[1].tolist() == [77, 78, -1]
    assert (np.abs(logprobs[[0, 1, 3], 0]) < 1e-6).all()
