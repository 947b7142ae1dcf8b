"""The example that decodes with trees (examples/tree_decode.py) on prompts that are longer than a tree: their tokens go through
the model in pieces, and the decode is still the model's (as test_gpu_tree_decode.py checks it, with its bound)."""

import copy

import pytest

torch = pytest.importorskip("torch")

import test_gpu_tree_decode  # noqa: E402
from test_gpu_tree_decode import example  # noqa: E402, F401
from workloads import make_workload  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes", [1, 7, 45, 46])
def test_prompts_in_pieces(example, monkeypatch, nodes):  # noqa: F811
    """prompts of 19 to 84 tokens: some end in an earlier piece than others, some with a piece"""
    monkeypatch.setattr(example, "NODES", nodes)
    test_gpu_tree_decode.test_greedy_decode_is_the_models(example, 3, 4)


def test_a_prompt_longer_than_a_tree(example, monkeypatch):  # noqa: F811
    wl = copy.copy(make_workload(2, rows=4))
    wl.prefixes = list(wl.prefixes)
    wl.prefixes[1] = b"SELECT " + b"86929 , " * 500 + wl.prefixes[1][7:]
    monkeypatch.setattr(test_gpu_tree_decode, "make_workload", lambda *a, **kw: wl)
    test_gpu_tree_decode.test_greedy_decode_is_the_models(example, 3, 4)
