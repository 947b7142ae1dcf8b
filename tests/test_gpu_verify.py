"""grid_verify on the GPU against its definition in 64 bits.

Tokens are decisions: they are equal unless a uniform number or two racers come within rounding (a relative 1e-5 here,
for which the reference says whether it was that close; random inputs hardly ever are).  A log probability is
(l - m) / T - log z in 32 bits: off by at most 2^-22 (|l - m| / T + |log z| + 1) and a relative error of z, a sum of V
terms added in trees of at most 640 in a row and some twenty joins: below 700 * 2^-24 = 2^-14.6.
"""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def G():
    import paper_2607_11951_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    pkg.lib()
    return pkg


def pack(bits):
    """bool [..., V] -> int32 words"""
    V = bits.shape[-1]
    W = (V + 31) // 32
    full = np.zeros(bits.shape[:-1] + (W * 32,), bool)
    full[..., :V] = bits
    return np.packbits(full, axis=-1, bitorder="little").view("<i4")


class Case:
    def __init__(self, B, K, V, dtype="f32", seed=0, share=None, probs=True, temps=None, ragged=True, std=2.0):
        r = np.random.default_rng(seed)
        self.B, self.K, self.V = B, K, V
        self.logits = torch.from_numpy((std * r.standard_normal((B, K + 1, V))).astype(np.float32)).to(DT[dtype]).cuda()
        self.bits = None if share is None else r.random((B, K + 1, V)) < share
        self.len = r.integers(0, K + 1, B).astype(np.int32) if ragged else np.full(B, K, np.int32)
        near = self.logits.double().cpu().numpy()[:, :K] + 0.7 * r.standard_normal((B, K, V))
        if self.bits is not None:
            near = np.where(self.bits[:, :K], near, -np.inf)
        near = near - np.maximum(near.max(-1, keepdims=True, initial=-1e300), -1e300)
        q = np.exp(near)
        self.probs = (q / np.maximum(q.sum(-1, keepdims=True), 1e-300)).astype(np.float32)
        self.draft = (self.probs / r.exponential(size=(B, K, V))).argmax(-1).astype(np.int32) if K else np.zeros((B, 0), np.int32)
        self.probs = self.probs if probs else None
        self.uniform = r.random((B, K)).astype(np.float32)
        self.noise = np.maximum(r.exponential(size=(B, V)), 1e-20).astype(np.float32)
        self.temps = temps if temps is None else np.resize(np.array(temps, np.float32), B)

    def run(self, G, greedy=False, **kw):
        def dev(x):
            return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
        args = dict(draft_len=dev(self.len), mask=None if self.bits is None else dev(pack(self.bits)),
                    draft_probs=dev(self.probs), uniform=dev(self.uniform), noise=dev(self.noise),
                    temperature=dev(self.temps))
        if greedy:
            args.update(draft_probs=None, uniform=None, noise=None)
        args.update(kw)
        got = G.verify(self.logits, dev(self.draft), **args)
        return [x.cpu().numpy() for x in got]

    def reference(self, greedy=False):
        B, K, V = self.B, self.K, self.V
        l = self.logits.double().cpu().numpy()
        tokens, accepted = np.full((B, K + 1), -1, np.int64), np.zeros(B, np.int64)
        logp, tol = np.zeros((B, K + 1)), np.zeros((B, K + 1))
        close = np.zeros(B, bool)
        for b in range(B):
            T = 1.0 if self.temps is None else float(self.temps[b])
            cold = greedy or not T > 0
            T = 1.0 if cold else T
            n = min(max(int(self.len[b]), 0), K)
            for j in range(n + 1):
                allowed = np.ones(V, bool) if self.bits is None else self.bits[b, j]
                x = np.where(allowed, l[b, j], -np.inf)
                top = np.nan if np.isnan(x).any() else x.max(initial=-np.inf)
                alive = np.isfinite(top)
                if alive:
                    w = np.exp((x - top) / T)
                    z = w.sum()
                    p = w / z
                accepted[b] = j
                if j < n and alive:
                    d = int(self.draft[b, j])
                    pd = p[d] if 0 <= d < V else 0.0
                    if cold:
                        ok = d == int(x.argmax())
                    else:
                        qd = (float(self.probs[b, j, d]) if 0 <= d < V else 1.0) if self.probs is not None else 1.0
                        ok = float(self.uniform[b, j]) * qd < pd
                        close[b] |= abs(float(self.uniform[b, j]) * qd - pd) < 1e-5 * pd
                    if ok:
                        tokens[b, j] = d
                        self._logp(b, j, d, x, top, T, z, logp, tol)
                        continue
                if not alive:
                    break
                if cold:
                    t = int(x.argmax())
                else:
                    left = p
                    if j < n:
                        if self.probs is not None:
                            left = np.maximum(p - self.probs[b, j].astype(np.float64), 0)
                        else:
                            left = p.copy()
                            if 0 <= self.draft[b, j] < V:
                                left[self.draft[b, j]] = 0
                        if not (left > 0).any():
                            left = p
                    score = left / self.noise[b].astype(np.float64)
                    t = int(score.argmax())
                    # what is left of p after q is off by some 1e-6 p
                    off = 1e-5 * score + 2e-6 * p / self.noise[b].astype(np.float64)
                    rest = np.delete(score + off, t)
                    close[b] |= bool(len(rest)) and score[t] - off[t] <= rest.max()
                tokens[b, j] = t
                self._logp(b, j, t, x, top, T, z, logp, tol)
                break
        return tokens, accepted, logp, tol, close

    @staticmethod
    def _logp(b, j, t, x, top, T, z, logp, tol):
        logp[b, j] = (x[t] - top) / T - math.log(z)
        tol[b, j] = 2.0 ** -22 * ((top - x[t]) / T + abs(math.log(z)) + 1) + 2.0 ** -14.6

    def check(self, G, greedy=False, may_be_close=0, **kw):
        got = self.run(G, greedy, **kw)
        tokens, accepted, logp, tol, close = self.reference(greedy)
        assert close.sum() <= may_be_close, "inputs that rounding decides"
        far = ~close
        assert np.array_equal(got[0][far], tokens[far])
        assert np.array_equal(got[1][far], accepted[far])
        assert (np.abs(got[2] - logp)[far] <= tol[far]).all(), np.abs(got[2] - logp)[far].max()
        return got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 31, 33, 500, 2047, 4099, 20000])
def test_sizes(G, dtype, probs, V):
    Case(9, 4, V, dtype, seed=V, share=0.6 if V > 40 else None, probs=probs, temps=[1.0, 0.6, 0.0, 1.7]).check(G)


@pytest.mark.parametrize("K", [0, 1, 2, 7, 8, 63])
@pytest.mark.parametrize("B", [1, 5, 130])
def test_drafts_and_batches(G, K, B):
    Case(B, K, 97, "f32", seed=100 * K + B, share=0.5, std=1.0).check(G)


@pytest.mark.parametrize("V,dtype", [(151936, "bf16"), (128256, "f16"), (50257, "f32"), (50257, "bf16")])
@pytest.mark.parametrize("B,K", [(1, 4), (3, 2)])
def test_large_vocabularies(G, V, dtype, B, K):
    Case(B, K, V, dtype, seed=V + B, share=0.3, temps=[0.8]).check(G)
    Case(B, K, V, dtype, seed=V + B + 1, share=20.0 / V, probs=False).check(G)
    Case(B, K, V, dtype, seed=V + B + 2, temps=[0.0, 1.0]).check(G)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_greedy(G, dtype):
    c = Case(40, 5, 3001, dtype, seed=1, share=0.4)
    best = np.where(c.bits[:, :5], c.logits.float().cpu().numpy()[:, :5], -np.inf).argmax(-1)
    hit = np.random.default_rng(2).random((40, 5)) < 0.8
    c.draft = np.where(hit, best, c.draft).astype(np.int32)
    got = c.check(G, greedy=True)
    assert got[1].max() >= 3
    c.temps = np.zeros(40, np.float32)
    again = c.check(G)
    assert all(np.array_equal(a, b) for a, b in zip(got, again))
    c.temps = np.resize(np.array([-1.0, np.nan], np.float32), 40)
    again = c.run(G)
    assert all(np.array_equal(a, b) for a, b in zip(got, again))


def test_ties_go_to_the_lowest_index(G):
    for V in (9, 5000, 30000):
        c = Case(3, 2, V, "bf16", seed=V, share=0.5)
        c.logits.fill_(1.5)
        c.noise[:] = 0.25
        low = c.bits.argmax(-1)
        assert np.array_equal(c.check(G, greedy=True)[0][:, 0], low[:, 0])
        c.len[:] = 0
        got = c.run(G)
        assert np.array_equal(got[0][:, 0], low[:, 0]) and (got[0][:, 1:] == -1).all()


def test_rows_without_a_distribution(G):
    """nothing allowed, minus infinity everywhere allowed, NaN or infinity at an allowed token: token -1, no draft accepted"""
    for dtype in DT:
        for bad in range(4):
            c = Case(4, 3, 700, dtype, seed=bad, share=0.5, probs=False, ragged=False)
            c.uniform[:] = 0.0  # all drafts are accepted where they can be
            at = [0, 1, 2, 3]
            for b in range(4):
                here = np.flatnonzero(c.bits[b, at[b]])
                if bad == 0:
                    c.bits[b, at[b]] = False
                elif bad == 1:
                    c.logits[b, at[b]] = -math.inf
                elif bad == 2:
                    c.logits[b, at[b], int(here[5])] = math.nan
                else:
                    c.logits[b, at[b], int(here[5])] = math.inf
            for greedy in (False, True):
                if greedy:
                    for b in range(4):
                        for j in range(3):
                            x = np.where(c.bits[b, j], c.logits[b, j].float().cpu().numpy(), -np.inf)
                            c.draft[b, j] = 0 if np.isnan(x).any() else x.argmax()
                got = c.run(G, greedy)
                assert got[1].tolist() == at
                for b in range(4):
                    assert got[0][b].tolist() == c.draft[b, :at[b]].tolist() + [-1] * (4 - at[b])
                assert np.isfinite(got[2]).all()


def test_what_is_masked_has_no_part(G):
    """NaN, infinities and the type's lowest value at masked tokens; the lowest value at allowed ones"""
    for dtype in DT:
        c = Case(6, 3, 1111, dtype, seed=3, share=0.5, temps=[1.0, 0.0])
        clean = c.check(G)
        out = torch.from_numpy(~c.bits).cuda()
        for x in (math.nan, math.inf, -math.inf, torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max):
            c.logits[out] = x
            again = c.run(G)
            assert all(np.array_equal(a, b) for a, b in zip(clean, again))
        c = Case(6, 0, 1111, dtype, seed=4, share=0.5, temps=[1.0, 0.0])
        c.logits.fill_(torch.finfo(DT[dtype]).min)
        c.check(G)


def test_drafts_that_are_no_tokens(G):
    c = Case(5, 3, 400, "f32", seed=5, probs=False, ragged=False)
    c.uniform[:] = 0.0
    c.draft[0, 0], c.draft[1, 1], c.draft[2, 2], c.draft[3, 0] = -1, 400, 1 << 30, -(1 << 31)
    got = c.check(G)
    assert got[1].tolist() == [0, 1, 2, 0, 3]
    assert (got[0][np.arange(5), got[1]] >= 0).all()
    # and with the drafter's probabilities
    c = Case(5, 3, 400, "f32", seed=5, ragged=False)
    c.uniform[:] = 0.0
    c.draft[0, 0], c.draft[1, 1] = -5, 400
    got = c.run(G)
    assert got[1].tolist() == [0, 1, 3, 3, 3]


def test_lengths_outside_the_drafts(G):
    c = Case(4, 3, 300, "f32", seed=6)
    c.len[:] = [-3, 9, 3, 0]
    got = c.check(G)
    assert got[1][0] == 0


def test_temperature_extremes(G):
    c = Case(4, 0, 900, "f32", seed=7, share=0.5, temps=[1e-30, 1e30, math.inf, 1e-3])
    got = c.run(G)
    x = np.where(c.bits, c.logits.cpu().numpy(), -np.inf)[:, 0]
    assert got[0][0, 0] == x[0].argmax()
    flat = np.where(c.bits[:, 0], 1 / c.noise, 0).argmax(-1)  # all allowed tokens alike
    assert got[0][1, 0] == flat[1] and got[0][2, 0] == flat[2]
    assert np.isfinite(got[2]).all()


def test_strides(G):
    c = Case(4, 3, 1001, "bf16", seed=8, share=0.4)
    want = c.check(G)
    wide = torch.full((4, 5, 1013), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, 1:, 3:1004] = c.logits
    mask = torch.full((4, 6, 40), -1, dtype=torch.int32, device="cuda")
    mask[:, 2:, :32] = torch.from_numpy(pack(c.bits)).cuda()
    probs = torch.full((4, 3, 1002), math.nan, device="cuda")
    probs[:, :, 1:] = torch.from_numpy(c.probs).cuda()
    noise = torch.full((4, 1005), math.nan, device="cuda")
    noise[:, 3:1004] = torch.from_numpy(c.noise).cuda()
    c.logits = wide[:, 1:, 3:1004]
    got = c.run(G, mask=mask[:, 2:, :32], draft_probs=probs[:, :, 1:], noise=noise[:, 3:1004])
    assert all(np.array_equal(a, b) for a, b in zip(want, got))


def test_the_target_is_followed(G):
    """The first token's frequencies over many sequences are the target's, whatever the drafter (a bound of five
    standard deviations for each of 11 tokens)."""
    B, V = 40000, 11
    for probs in (True, False):
        c = Case(1, 1, V, "f32", seed=9, std=1.2, ragged=False)
        c.B = B
        c.logits = c.logits.expand(B, 2, V)
        r = np.random.default_rng(10)
        q = r.dirichlet(np.ones(V)).astype(np.float32)
        c.probs = np.broadcast_to(q, (B, 1, V)) if probs else None
        c.draft = r.choice(V, size=(B, 1), p=q.astype(np.float64) / q.sum(dtype=np.float64)).astype(np.int32) if probs else \
            np.full((B, 1), 3, np.int32)
        c.len = np.ones(B, np.int32)
        c.uniform, c.noise = r.random((B, 1), np.float32), r.exponential(size=(B, V)).astype(np.float32)
        tokens, accepted, _ = c.run(G)
        p = torch.softmax(c.logits[0, 0].double(), -1).cpu().numpy()
        freq = np.bincount(tokens[:, 0], minlength=V) / B
        assert (np.abs(freq - p) <= 5 * np.sqrt(p * (1 - p) / B)).all()
        want = np.minimum(p, q).sum() if probs else p[3]
        assert abs(accepted.mean() - want) <= 5 * math.sqrt(want * (1 - want) / B)


def test_same_bits_every_time(G):
    c = Case(3, 4, 151936, "bf16", seed=11, share=0.4)
    first = c.run(G)
    for _ in range(5):
        assert all(np.array_equal(a, b) for a, b in zip(first, c.run(G)))


def test_other_stream_and_graph(G):
    c = Case(6, 3, 50257, "bf16", seed=12, share=0.4, ragged=False)
    want = c.check(G)
    draft, mask, probs, uniform, noise = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in
                                          (c.draft, pack(c.bits), c.probs, c.uniform, c.noise))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = G.verify(c.logits, draft, mask=mask, draft_probs=probs, uniform=uniform, noise=noise, stream=side)
    side.synchronize()
    assert all(np.array_equal(a, b.cpu().numpy()) for a, b in zip(want, got))
    out = [torch.empty_like(x) for x in got]
    workspace = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.verify(c.logits, draft, mask=mask, draft_probs=probs, uniform=uniform, noise=noise, tokens=out[0],
                 accepted=out[1], logprobs=out[2], workspace=workspace)
    for i in range(4):
        uniform.uniform_()
        noise.exponential_()
        workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = G.verify(c.logits, draft, mask=mask, draft_probs=probs, uniform=uniform, noise=noise)
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
