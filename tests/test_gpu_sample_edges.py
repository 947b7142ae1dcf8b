"""grid_sample at its edges, against its definition in 64 bits (the reference of test_gpu_sample.py).

Tokens are equal where rounding does not decide.  Bounds of a log probability (l - m) / T - log z: 2^-22 (|l - m| / T + |log z| + 1)
for its own roundings, and the relative error of z.  A weight is off by less than 2^-21 (an exponential of one unit in the
last place and a rounded argument); sums that a thread and the joins of a row add up in 64 steps at most, by 64 * 2^-24 =
2^-18; listed weights are added as whole numbers of 2^-40 or less.  Where a nucleus ends among equals one of them more or less
changes z by 1 / (kept tokens).  Together below 2^-17 + 1 / kept.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_sample import DT, G, Rows  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def check(x, G, rows=None):  # noqa: F811
    tokens, logp, _, close, kept = x.reference()
    assert not close.any(), "inputs that rounding decides"
    got = [y.cpu().numpy() for y in x.run(G)]
    assert np.array_equal(got[0], tokens), (got[0], tokens)
    l = x.logits.double().numpy()
    for b in range(x.B):
        ids = np.arange(x.V) if x.bits is None else x.bits[b].nonzero()[0]
        T = 1.0 if x.temps is None else float(x.temps[b])
        d = (l[b, tokens[b]] - l[b, ids].max()) / T
        tol = 2.0 ** -22 * (2 * abs(d) + abs(logp[b]) + 1) + 2.0 ** -17 + 1 / len(kept[b]) * (len(kept[b]) > 1000)
        assert abs(got[1][b] - logp[b]) <= tol, (b, got[1][b], logp[b], tol)


@pytest.mark.parametrize("V,share,low,filters", [
    (1000000, 0.4, -1.0, {"p": [0.6]}),                     # a nucleus that ends among 400000 equals
    (1 << 20, 0.4, -30.0, {"p": [0.9]}),
    (1 << 20, 0.4, -1.0, {"k": [280000]}),                  # so many of them
    (1000000, 0.4, -1.0, {"k": [390000], "p": [0.8]}),
    (600011, 0.45, -1.0, {"p": [0.55], "q": [0.5]}),
    (3000001, 0.4, -1.0, {"p": [0.6]})])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_vocabularies_with_many_equals(G, V, share, low, filters, dtype):  # noqa: F811
    """more weights in one bin than 64 bits hold at 46 bits each, and not so many in a piece that one workgroup takes the row"""
    x = Rows(1, V, dtype, seed=V, **filters)
    r = np.random.default_rng(V)
    x.logits = torch.from_numpy(np.where(r.random((1, V)) < share, 0.0, low).astype(np.float32)).to(DT[dtype])
    check(x, G)


def test_large_vocabularies_under_a_mask(G):  # noqa: F811
    """flat logits, of which a mask leaves two fifths"""
    x = Rows(1, 1 << 20, "f32", seed=3, share=0.4, std=1e-3, p=[0.9])
    check(x, G)
    x = Rows(1, 1 << 20, "bf16", seed=4, share=0.4, std=0.0, p=[0.9])
    check(x, G)


@pytest.mark.parametrize("temp", [1e-8, 1e-10, 1e-20, 1e-30])
@pytest.mark.parametrize("shift", [0.0, 20.0, -300.0, 1e4])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_min_p_alone_at_low_temperatures(G, temp, shift, dtype):  # noqa: F811
    """scaled logits far outside of what a bin's number or a float's unit tells apart"""
    x = Rows(6, 9000, dtype, seed=21, temps=[temp], q=[0.05, 0.5, 0.9])
    x.logits = (x.logits.float() + shift).to(DT[dtype])
    check(x, G)


@pytest.mark.parametrize("filters", [{}, {"q": [1e-4]}, {"k": [30000]}])
def test_equals_in_different_pieces(G, filters):  # noqa: F811
    """equal logits with equal noise, below other largest logits all over the row: the lowest index"""
    B, V = 64, 45000
    x = Rows(B, V, "f32", seed=22, temps=[1.0, 0.7, 1.9], **filters)
    r = np.random.default_rng(5)
    x.logits = torch.full((B, V), -9.0)
    x.noise[:] = 1.0
    first = []
    for b in range(B):
        tops, equals = r.choice(V, 40, replace=False), np.sort(r.choice(V, 30, replace=False))
        x.logits[b, tops] = torch.from_numpy(r.uniform(0.1, 3.0, 40).astype(np.float32))
        x.noise[b, tops] = 1e6
        x.logits[b, equals] = float(r.uniform(-0.5, 0.0))
        x.noise[b, equals] = 1e-3
        first.append(int(equals[0]))
    assert x.run(G)[0].tolist() == first
