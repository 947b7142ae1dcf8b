"""The example that runs the step's calls together (examples/draft_decode.py), checked without them: the greedy decode
with drafts and forced spans against the model evaluated whole, in 64 bits, with plain attention.

The model's activations are rounded to float16 at three places a layer (projections, rotated vectors, attention's
output; 2^-11 each) and its other products are in float32; its logits are of size 3 and its residual stream averages the
errors of 256 entries, so they are off by well under 3 * 2^-6 = 0.05 in 64-bit terms.  An emitted token has to be within
that of the best allowed logit."""

import importlib.util
import sys
from pathlib import Path

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from workloads import make_workload  # noqa: E402

pytestmark = pytest.mark.gpu

PATH = Path(__file__).resolve().parent.parent / "examples" / "draft_decode.py"


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("draft_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    sys.modules["draft_decode"] = m
    spec.loader.exec_module(m)
    return m


def whole(model, tokens):
    """The model's logits after every token, in 64 bits, over the whole sequence at once."""
    def normed(x):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)

    n, h, kh, D = len(tokens), model.heads, model.kv_heads, model.head_dim
    x = model.embed.double()[torch.tensor(tokens, device="cuda")]
    cos, sin = model.cos.double()[:n, None], model.sin.double()[:n, None]
    later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
    for w in model.layers:
        qkv = (normed(x) @ w["qkv"].double()).view(n, h + 2 * kh, D)
        turned = []
        for y in (qkv[:, :h], qkv[:, h:h + kh]):
            y = normed(y)
            a, c = y[..., :D // 2], y[..., D // 2:]
            turned.append(torch.cat([a * cos - c * sin, c * cos + a * sin], -1))
        q, k, v = turned[0], turned[1], qkv[:, h + kh:]
        out = []
        for i in range(h):
            g = i // (h // kh)
            s = (q[:, i] @ k[:, g].T.contiguous()) / D ** 0.5
            out.append(torch.softmax(s.masked_fill(later, -float("inf")), -1) @ v[:, g].contiguous())
        x = x + torch.cat(out, -1) @ w["out"].double()
        x = x + torch.relu(normed(x) @ w["up"].double()) @ w["down"].double()
    return normed(x) @ model.unembed.double()


@pytest.mark.parametrize("drafts", [0, 1, 4])
def test_greedy_decode_is_the_models(example, drafts):
    import paper_2607_11951_amd as G
    wl = make_workload(2, rows=6)
    model = example.Model(wl.V, seed=1)
    got = example.decode(model, wl, rows=6, new_tokens=40, drafts=drafts)
    grid, slots = G.from_workload(wl)
    grid.to_device("cuda")
    for b, (p, h) in enumerate(zip(got["prompts"], got["histories"])):
        assert h[:len(p)] == p and len(h) > len(p)
        logits = whole(model, h).cpu().numpy()
        slot = slots[wl.slots[b]]
        texts = [b"".join(wl.vocab[t] for t in h[:i]) for i in range(len(p), len(h))]
        cfgs, pool = grid.configs(texts, [slot] * len(texts))  # every prefix is viable
        c, s = grid.configs_to_device(cfgs, pool)
        mask = grid.mask(c, s, len(texts))[0].cpu().numpy().view(np.uint8)
        allowed = np.unpackbits(mask, axis=1, bitorder="little")[:, :wl.V].astype(bool)
        for i, t in enumerate(h[len(p):]):
            assert allowed[i, t], (b, i)
            best = np.where(allowed[i], logits[len(p) + i - 1], -np.inf)
            assert best.max() - best[t] <= 0.05, (b, i, best.max() - best[t])
    if drafts == 4:
        assert got["accepted"] > 0 and got["drafted"] >= got["accepted"]


def test_drafts_do_not_change_what_is_decoded(example):
    wl = make_workload(2, rows=4)
    model = example.Model(wl.V, seed=2)
    one = example.decode(model, wl, rows=4, new_tokens=32, drafts=0)
    more = example.decode(model, wl, rows=4, new_tokens=32, drafts=5)
    for a, b in zip(one["histories"], more["histories"]):
        n = min(len(a), len(b))  # a step may go past the asked number of tokens
        assert a[:n] == b[:n]
    assert more["steps"] <= one["steps"]


def test_sampled_decode(example):
    wl = make_workload(2, rows=5)
    model = example.Model(wl.V, seed=3)
    first = example.decode(model, wl, rows=5, new_tokens=24, drafts=3, temperature=1.0, seed=4)
    again = example.decode(model, wl, rows=5, new_tokens=24, drafts=3, temperature=1.0, seed=4)
    other = example.decode(model, wl, rows=5, new_tokens=24, drafts=3, temperature=1.0, seed=5)
    assert first["histories"] == again["histories"] and first["histories"] != other["histories"]
