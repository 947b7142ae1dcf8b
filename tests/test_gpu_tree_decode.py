"""The example that runs the calls of a step with trees together (examples/tree_decode.py), checked without them: the greedy
decode with trees and shared pages against the model evaluated whole, in 64 bits, with plain attention.  An emitted token has
to be allowed, and within 0.05 of the best allowed logit (the bound of test_gpu_draft_decode.py: the same model)."""

import importlib.util
import sys
from pathlib import Path

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_draft_decode import whole  # noqa: E402
from workloads import make_workload  # noqa: E402

pytestmark = pytest.mark.gpu

PATH = Path(__file__).resolve().parent.parent / "examples" / "tree_decode.py"


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("tree_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    sys.modules["tree_decode"] = m
    spec.loader.exec_module(m)
    return m


def allowed_after(G, grid, slot, wl, tokens, n):
    """the allowed tokens after each of the prefixes of n and more tokens"""
    texts = [b"".join(wl.vocab[t] for t in tokens[:i]) for i in range(n, len(tokens))]
    cfgs, pool = grid.configs(texts, [slot] * len(texts))  # every prefix is viable
    mask = grid.mask(*grid.configs_to_device(cfgs, pool), len(texts))[0].cpu().numpy().view(np.uint8)
    return np.unpackbits(mask, axis=1, bitorder="little")[:, :wl.V].astype(bool)


@pytest.mark.parametrize("branches,depth", [(0, 0), (1, 5), (3, 4)])
def test_greedy_decode_is_the_models(example, branches, depth):
    import paper_2607_11951_amd as G
    wl = make_workload(2, rows=4)
    model = example.TreeModel(wl.V, seed=1)
    got = example.decode(model, wl, rows=4, samples=2, new_tokens=40, branches=branches, depth=depth)
    grid, slots = G.from_workload(wl)
    grid.to_device("cuda")
    for b, (p, h) in enumerate(zip(got["prompts"], got["histories"])):
        assert h[:len(p)] == p and len(h) > len(p)
        allowed = allowed_after(G, grid, slots[wl.slots[b // 2]], wl, h, len(p))
        logits = whole(model, h).cpu().numpy()
        for i, t in enumerate(h[len(p):]):
            assert allowed[i, t], (b, i)
            best = np.where(allowed[i], logits[len(p) + i - 1], -np.inf)
            assert best.max() - best[t] <= 0.05, (b, i, best.max() - best[t])
    if branches:
        assert 0 < got["accepted"] <= got["drafted"]


def test_sampled_decode(example):
    """allowed tokens only; the same seed gives the same sequences, another one others; rows of one prompt differ"""
    import paper_2607_11951_amd as G
    wl = make_workload(2, rows=3)
    model = example.TreeModel(wl.V, seed=3)

    def decode(seed, **kw):
        return example.decode(model, wl, rows=3, samples=3, new_tokens=24, temperature=1.0, top_k=40, top_p=0.95, min_p=0.001,
                              seed=seed, **kw)

    first, again, other = decode(4), decode(4), decode(5)
    assert first["histories"] == again["histories"] and first["histories"] != other["histories"]
    assert any(first["histories"][0] != h for h in first["histories"][1:3])
    grid, slots = G.from_workload(wl)
    grid.to_device("cuda")
    for b, (p, h) in enumerate(zip(first["prompts"], first["histories"])):
        allowed = allowed_after(G, grid, slots[wl.slots[b // 3]], wl, h, len(p))
        assert all(allowed[i, t] for i, t in enumerate(h[len(p):]))
