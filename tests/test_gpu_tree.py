"""Trees of drafts on the GPU: grid_tree_masks, grid_kv_append_tree, grid_attend_tree and grid_commit_tree against plain
implementations.  Bounds of computed numbers as for chunks that are no trees: attention with the scores, weights and sums of
the same kernels (|out - ref| <= (u + 2 e + 2^-18) sum p |v| + u |ref| + n 2^-25 max |v| with e = (D + 8) 2^-24 scale sum
|q_i k_i| and u half a unit in the last place; |lse - ref| <= e + 2^-20 (1 + |ref|)); an append is one rounding of 32-bit
arithmetic.  All else is whole numbers and copies, and equal."""

import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attend import DT, U, Batch, rounded_once, tables, turned  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import paper_2607_11951_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    pkg.lib()
    return pkg


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def random_parents(lens, seed, reach=8, roots=0.0):
    """of every chunk's nodes: earlier ones, no further back than `reach`; now and then none"""
    r = random.Random(seed)
    return [i - 1 - r.randrange(min(i, reach)) if i and r.random() >= roots else -1 for n, _ in lens for i in range(n)]


def plain_masks(lens, parent, max_q):
    """(words [T, W], depth [T]) by following parents"""
    W, rows, depth, at = (max_q + 31) // 32, [], [], 0
    for n, _ in lens:
        for i in range(n):
            bits, j, d = 0, i, -1
            while j >= 0:
                bits |= 1 << j
                d += 1
                p = parent[at + j]
                j = p if 0 <= p < j else -1
            rows.append([(bits >> 32 * w & 0xFFFFFFFF) for w in range(W)])
            depth.append(d)
        at += n
    words = np.array(rows, np.uint32).reshape(-1, W).view(np.int32)
    return torch.from_numpy(words).cuda(), ints(depth)


class Trees(Batch):
    def __init__(self, lens, heads, page, dtype, seed=0, reach=8, roots=0.0, words=0, **kw):
        super().__init__(lens, heads, page, dtype, seed=seed, **kw)
        self.parent = random_parents(lens, seed, reach, roots)
        self.tree, self.depth = plain_masks(lens, self.parent, max(self.max_q, 32 * words))

    def attend(self, G, **kw):
        kw.setdefault("max_q", self.max_q)
        kw.setdefault("max_kv", self.max_kv)
        kw.setdefault("depth", self.depth)
        return G.attend_tree(self.q, self.k, self.v, self.table, self.kv_len, self.cu, self.tree, **kw)


def reference(bt, window=0, scale=None):
    """out, lse in 64 bits and the bounds of both, from the bits of bt.tree"""
    scale = bt.D ** -0.5 if scale is None else scale
    group, u = bt.hq // bt.hkv, U[bt.dt]
    out = torch.zeros((bt.T, bt.hq, bt.D), dtype=torch.float64, device="cuda")
    lse = torch.full((bt.T, bt.hq), -math.inf, dtype=torch.float64, device="cuda")
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    for b, (n, kv) in enumerate(bt.lens):
        if n == 0:
            continue
        k, v = bt.gathered(bt.k, b), bt.gathered(bt.v, b)
        at, first = int(bt.cu_host[b]), kv - n
        bits = bt.tree[at:at + n, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32) & 1
        inside = bits.flatten(1)[:, :n].bool()
        key = torch.arange(first, device="cuda")[None]
        pos = first + bt.depth[at:at + n].long()[:, None]
        seen = torch.cat([(key > pos - window) if window else (key >= 0).expand(n, first), inside], 1)
        for h in range(bt.hq):
            g = h // group
            q = bt.q[at:at + n, h].double()
            kg, vg = (torch.nan_to_num(x[:, g], 0, 0, 0) for x in (k, v))
            x = scale * (q @ kg.T.contiguous())
            e = (bt.D + 8) * 2.0 ** -24 * abs(scale) * (q.abs() @ kg.abs().T.contiguous())
            x = torch.where(seen, x, -math.inf)
            e = torch.where(seen, e, 0.0).amax(-1)
            l = torch.logsumexp(x, -1)
            p = torch.where(seen, torch.exp(x - l[:, None].clamp_min(-1e300)), 0.0)
            o, mass = p @ vg, p @ vg.abs()
            out[at:at + n, h], lse[at:at + n, h] = o, l
            out_tol[at:at + n, h] = (u + 2 * e[:, None] + 2.0 ** -18) * mass + u * o.abs() + \
                (kv * 2.0 ** -25 * vg.abs().max() + 2.0 ** -25 if bt.dt == torch.float16 else 0.0)
            lse_tol[at:at + n, h] = e + 2.0 ** -20 * (1 + l.abs())
    return out, lse, out_tol, lse_tol


def agree(got, bt, rows=None, **kw):
    out, lse, out_tol, lse_tol = reference(bt, **kw)
    sel = slice(None) if rows is None else rows
    d = (got[0].double() - out)[sel].abs()
    assert bool((d <= out_tol[sel]).all()), float((d / out_tol[sel].clamp_min(1e-300)).nan_to_num(math.inf).max())
    none = torch.isneginf(lse)
    assert torch.equal(torch.isneginf(got[1])[sel], none[sel])
    d = (got[1].double() - lse).masked_fill(none, 0.0)[sel].abs()
    tol = lse_tol.masked_fill(none, 0.0)[sel]
    assert bool((d <= tol).all()), float((d / tol.clamp_min(1e-300)).nan_to_num(math.inf).max())


# ------------------------------------------------------------------------------------------------------------- masks
@pytest.mark.parametrize("lens", [[(1, 1)], [(5, 9), (0, 3), (64, 64), (1, 7), (33, 40)], [(300, 300), (1000, 1024)],
                                  [(i % 7, 9) for i in range(700)]])
@pytest.mark.parametrize("reach,roots", [(1, 0.0), (8, 0.1), (1000, 0.0)])
def test_tree_masks(G, lens, reach, roots):
    parent = random_parents(lens, len(lens), reach, roots)
    max_q = max(n for n, _ in lens) + 3
    words, depth = plain_masks(lens, parent, max_q)
    cu = ints(np.concatenate([[0], np.cumsum([n for n, _ in lens])]).tolist())
    got = G.tree_masks(ints(parent), cu, max_q)
    assert torch.equal(got[0], words) and torch.equal(got[1], depth)


def test_tree_masks_of_what_is_no_tree(G):
    """parents that are not before their nodes are none; chunks out of order or too long are empty; others' rows are left"""
    parent = [5, 0, 2, -9, 1 << 30, 3, 0, 0, 1, -1]
    masks, depth = torch.full((10, 3), 77, dtype=torch.int32, device="cuda"), torch.full((10,), 77, dtype=torch.int32, device="cuda")
    got = G.tree_masks(ints(parent), ints([1, 5, 9]), 40, masks=masks, depth=depth)
    assert got[0] is masks and got[1] is depth
    #                places 0 .. 3 of tokens 1 .. 4: parents 0 (itself), 2 (later), -9, 2^30; then 3 (later), 0, 0, 1
    assert masks[:, 0].tolist() == [77, 1, 2, 4, 8, 1, 3, 5, 0b1011, 77]
    assert masks[1:9, 1].tolist() == [0] * 8 and bool((masks[:, 2] == 77).all())
    assert depth.tolist() == [77, 0, 0, 0, 0, 0, 1, 1, 2, 77]
    masks.fill_(77), depth.fill_(77)
    G.tree_masks(ints([-1] * 10), ints([0, 2, 7, 5, 10]), 4, masks=masks, depth=depth)
    assert masks[:, 0].tolist() == [1, 2] + [0] * 8  # the second is too long, the third out of order: all after it is its own
    assert depth.tolist() == [0] * 10


# ------------------------------------------------------------------------------------------------------------ attend
MIXED = [(1, 1), (1, 700), (0, 33), (5, 5), (5, 130), (0, 0), (1, 64), (9, 65), (33, 200), (2, 1025)]


@pytest.mark.parametrize("heads", [(28, 4, 128), (4, 4, 64), (15, 5, 64), (8, 1, 256), (32, 8, 128), (6, 2, 256),
                                   (40, 1, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_mixed_lengths(G, heads, dtype):
    bt = Trees(MIXED, heads, 16, dtype, seed=1)
    agree(bt.attend(G), bt)


@pytest.mark.parametrize("page", [1, 3, 16, 24, 64, 100, 256, 4096])
@pytest.mark.parametrize("window", [0, 1, 37, 128, 5000])
def test_pages_and_windows(G, page, window):
    bt = Trees([(1, 777), (7, 300), (70, 333), (3, 3), (0, 9), (1, 129)], (14, 2, 128), page, "bf16", seed=page, roots=0.05)
    agree(bt.attend(G, window=window), bt, window=window)


@pytest.mark.parametrize("n", [1, 2, 7, 8, 16, 31, 32, 33, 63, 64, 65, 127, 129, 300, 513])
@pytest.mark.parametrize("heads", [(8, 1, 128), (3, 3, 64), (10, 2, 256)])
def test_tree_sizes(G, n, heads):
    bt = Trees([(n, n), (n, n + 95), (n, n + 1)], heads, 32, "bf16", seed=n, reach=n)
    agree(bt.attend(G), bt)


@pytest.mark.parametrize("before", [0, 1, 30, 31, 32, 33, 63, 65, 100, 127, 128, 640, 2047, 4097])
def test_trees_anywhere_in_a_stage(G, before):
    for heads in ((28, 4, 128), (4, 4, 64), (2, 1, 256)):
        bt = Trees([(40, before + 40), (3, before + 3)], heads, 16, "bf16", seed=before)
        agree(bt.attend(G), bt)


@pytest.mark.parametrize("lens", [[(1, 40000)], [(4, 70001), (1, 17)], [(40, 33333)], [(200, 20000), (1, 30000)]])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_long_caches(G, lens, dtype):
    bt = Trees(lens, (16, 2, 128), 64, dtype, seed=5)
    agree(bt.attend(G), bt)
    agree(bt.attend(G, window=9000), bt, window=9000)


def test_a_chain_is_a_chunk(G):
    """trees of one branch: what grid_attend gives, whatever the launch"""
    for lens in (MIXED, [(40, 3000), (64, 100)]):
        bt = Trees(lens, (28, 4, 128), 16, "bf16", seed=2, reach=1)
        for window in (0, 50):
            want = G.attend(bt.q, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, bt.max_q, bt.max_kv, window=window)
            if window:  # a window counts ancestors as well there
                continue
            agree(want, bt)
            agree(bt.attend(G), bt)


def test_any_bits_and_rows_that_see_nothing(G):
    """masks that are no tree's: bits at random, later places among them, and rows without any"""
    for lens in ([(9, 9), (40, 40), (3, 3)], [(9, 90), (70, 1000), (3, 3)]):
        for heads in ((8, 2, 64), (28, 4, 128), (2, 1, 256)):
            bt = Trees(lens, heads, 16, "bf16", seed=7, words=4)
            r = np.random.default_rng(3)
            bits = r.integers(-2 ** 31, 2 ** 31, bt.tree.shape).astype(np.int32)
            bits[r.random(bt.T) < 0.4] = 0
            bt.tree = torch.from_numpy(bits).cuda()
            got = bt.attend(G)
            agree(got, bt)
            none = torch.isneginf(got[1])
            assert bool(none.any()) and bool((got[0][none] == 0).all())


@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("lens", [[(5, 130), (1, 31), (33, 90)], [(200, 300)], [(7, 7)], [(12, 900), (40, 1500)]])
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (2, 1, 256)])
def test_what_is_not_seen_has_no_part(G, poison, lens, heads):
    """infinities and NaN in free pages, after a sequence's end, before its window, and in other branches"""
    window = 40
    bt = Trees(lens, heads, 16, "bf16", seed=11, spare=3)
    clean = bt.attend(G, window=window)
    agree(clean, bt, window=window)
    for pages in (bt.k, bt.v):
        pages[torch.from_numpy(bt.free.astype(np.int64)).cuda()] = poison
        for b, (n, kv) in enumerate(lens):
            if kv % bt.page:
                pages[int(bt.table_host[b, kv // bt.page]), kv % bt.page:] = poison
            for s in range(0, max(0, kv - n - window + 1)):
                page, row = bt.rows(b, np.array([s]))
                pages[int(page[0]), int(row[0])] = poison
    got = bt.attend(G, window=window)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    # a node in the middle of each tree: itself and its descendants see it
    sees = torch.zeros(bt.T, dtype=torch.bool)
    for b, (n, kv) in enumerate(lens):
        i, at = n // 2, int(bt.cu_host[b])
        sees[at:at + n] = (bt.tree[at:at + n, i // 32] >> i % 32 & 1).bool().cpu()
        page, row = bt.rows(b, np.array([kv - n + i]))
        for pages in (bt.k, bt.v):
            pages[int(page[0]), int(row[0])] = poison
    got = bt.attend(G, window=window)
    assert torch.equal(got[0][~sees], clean[0][~sees]) and torch.equal(got[1][~sees], clean[1][~sees])
    assert not torch.isfinite(got[0][sees].float()).all(-1).any()


def test_bad_sequences_are_nan(G):
    lens = [(2, 90), (1, 40), (3, 64), (1, 100), (40, 200)]

    def check(change, bad, **kw):
        bt, good = (Trees(lens, (8, 2, 128), 16, "bf16", seed=13) for _ in range(2))
        change(bt)
        got = bt.attend(G, **kw)
        rows = torch.zeros(bt.T, dtype=torch.bool, device="cuda")
        for b in bad:
            rows[int(good.cu_host[b]):int(good.cu_host[b + 1])] = True
        agree(got, good, rows=~rows)
        assert bool(torch.isnan(got[0][rows].float()).all()) and bool(torch.isnan(got[1][rows]).all())

    def put(name, at, x):
        return lambda bt: getattr(bt, name).__setitem__(at, x)

    for kw in ({}, {"max_kv": 2000}):
        check(put("table", (0, 1), 1 << 20), [0], **kw)
        check(put("kv_len", 1, 1 << 30), [1], **kw)
        check(put("kv_len", 2, 2), [2], **kw)
        check(put("cu", 5, 10000), [4], **kw)
        check(put("cu", 4, 2), [3, 4], **kw)
    check(lambda bt: None, [3, 4], max_kv=99)
    check(lambda bt: None, [4], max_q=3)


def test_layouts_streams_and_graphs(G):
    bt = Trees([(12, 5000), (1, 300), (60, 900)], (6, 3, 64), 16, "bf16", seed=17, heads_first=True)
    want = bt.attend(G)
    agree(want, bt)
    wide = bt.rand((bt.T, 20, bt.D))
    wide[:, 5:11] = bt.q
    bt.q = wide[:, 5:11]
    words = torch.full((bt.T, 9), -1, dtype=torch.int32, device="cuda")
    words[:, 2:4] = bt.tree
    bt.tree = words[:, 2:4]
    out, lse = torch.zeros((bt.T, 9, bt.D), dtype=bt.dt, device="cuda"), torch.zeros((bt.T, 6), device="cuda")
    got = bt.attend(G, out=out[:, 2:8], lse=lse)
    assert torch.equal(got[0], want[0]) and got[1] is lse and torch.equal(lse, want[1])
    assert bool((out[:, :2] == 0).all()) and bool((out[:, 8:] == 0).all())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bt.attend(G, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out, workspace = torch.empty_like(want[0]), torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    parent = ints(bt.parent)
    masks, depth = torch.empty((bt.T, 2), dtype=torch.int32, device="cuda"), torch.empty(bt.T, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.tree_masks(parent, bt.cu, bt.max_q, masks=masks, depth=depth)
        G.attend_tree(bt.q, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, masks, bt.max_q, bt.max_kv, out=out, lse=lse,
                      workspace=workspace)
    for i in range(4):
        bt.parent = random_parents(bt.lens, 100 + i)
        parent.copy_(ints(bt.parent))
        bt.tree, bt.depth = plain_masks(bt.lens, bt.parent, bt.max_q)
        workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        agree((out, lse), bt)
        again = bt.attend(G)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_rows_of_no_sequence_are_left(G):
    bt = Trees([(3, 20), (2, 70)], (4, 2, 64), 16, "bf16", seed=14)
    q, tree = bt.q, bt.tree
    bt.q = torch.cat([q[:2], q, q[:4]])
    bt.tree = torch.cat([tree[:2], tree, tree[:4]])
    out, lse = torch.full_like(bt.q, 7.0), torch.full((bt.T + 6, bt.hq), 7.0, device="cuda")
    bt.cu = bt.cu + 2
    bt.attend(G, out=out, lse=lse, depth=None)
    assert bool((out[:2] == 7).all()) and bool((out[bt.T + 2:] == 7).all())
    assert bool((lse[:2] == 7).all()) and bool((lse[bt.T + 2:] == 7).all())
    bt.q, bt.tree = q, tree
    agree((out[2:bt.T + 2], lse[2:bt.T + 2]), bt)
    empty = G.attend_tree(q[:0], bt.k, bt.v, bt.table, bt.kv_len, torch.zeros_like(bt.cu), tree[:0], 1, 100)
    assert empty[0].shape == (0, bt.hq, bt.D)


def test_same_bits_every_time(G):
    bt = Trees([(1, 9000), (25, 3000), (64, 700)], (28, 4, 128), 16, "bf16", seed=16)
    first = bt.attend(G)
    for _ in range(5):
        again = bt.attend(G)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ------------------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_append_at_depths(G, style, dtype):
    lens = [(1, 1), (9, 100), (0, 40), (33, 77), (2, 2)]
    bt = Trees(lens, (6, 2, 128), 24, dtype, seed=3)
    k, v = bt.rand((bt.T, 2, 128), 3.0), bt.rand((bt.T, 2, 128))
    weight = [1 + torch.randn(128, device="cuda") for _ in range(2)]
    first = torch.cat([torch.full((n,), kv - n) for n, kv in lens]).cuda()
    pos = first + bt.depth.long()
    cos, sin = tables(101, 64)
    page, row = (torch.from_numpy(np.concatenate([bt.rows(b, np.arange(kv - n, kv))[i] for b, (n, kv) in enumerate(lens)])
                                  .astype(np.int64)).cuda() for i in range(2))
    old_k, old_v = bt.k.clone(), bt.v.clone()
    status = torch.full((len(lens),), -1, dtype=torch.int32, device="cuda")
    q_out, _ = G.kv_append(k, v, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, q=bt.q, cos=cos, sin=sin, depth=bt.depth,
                           interleaved=style == "pairs", q_norm=weight[0], k_norm=weight[1], eps=1e-5, status=status)
    assert status.tolist() == [0] * len(lens)
    for got, x, w in ((bt.k[page, row], k, weight[1]), (q_out, bt.q, weight[0])):
        want, size = turned(x, pos, w, 1e-5, cos, sin, style == "pairs")
        rounded_once(got, want, size)
    assert torch.equal(bt.v[page, row], v)
    old_k[page, row], old_v[page, row] = bt.k[page, row], bt.v[page, row]
    assert torch.equal(bt.k, old_k) and torch.equal(bt.v, old_v)


def test_append_leaves_out_depths_without_a_position(G):
    lens = [(3, 40), (4, 10), (2, 30)]
    bt = Trees(lens, (2, 1, 64), 16, "bf16", seed=21)
    k, v = bt.rand((bt.T, 1, 64)), bt.rand((bt.T, 1, 64))
    cos, sin = tables(40, 64)
    depth = ints([0, 3, 1, 0, -1, 1, 2, 0, 1 << 30])  # 37 + 3 has no row; -1 is no depth; nor has 2^30 a row
    status = torch.full((3,), -1, dtype=torch.int32, device="cuda")
    old = bt.k.clone()
    G.kv_append(k, v, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, cos=cos, sin=sin, depth=depth, status=status)
    assert status.tolist() == [2, 2, 2]
    for b, (n, kv) in enumerate(lens):
        for i in range(n):
            t, d = int(bt.cu_host[b]) + i, int(depth[int(bt.cu_host[b]) + i])
            page, row = bt.rows(b, np.array([kv - n + i]))
            got = bt.k[int(page[0]), int(row[0])]
            if d < 0 or kv - n + d >= 40:
                assert torch.equal(got, old[int(page[0]), int(row[0])])
            else:
                want, size = turned(k[t:t + 1], torch.tensor([kv - n + d]).cuda(), None, 0, cos, sin, False)
                rounded_once(got[None], want, size)


@pytest.mark.parametrize("at", [0, 15, 16, 63, 64, 127, 128, 500, 999])
def test_append_tells_where_a_depth_has_no_position(G, at):
    """at a place of every tree that has it, in some a negative depth, in the others one past the table of positions"""
    lens = [(1, 3), (64, 70), (128, 200), (129, 129), (0, 5), (1000, 1024), (600, 700), (128, 128), (17, 30)] * 8
    bt = Trees(lens, (1, 1, 64), 16, "bf16", seed=at)
    k = bt.rand((bt.T, 1, 64))
    cos, sin = tables(1024, 64)
    status = torch.full((len(lens),), -1, dtype=torch.int32, device="cuda")
    for bad in (None, -1, 1024):
        depth, want = torch.zeros_like(bt.depth), []
        for b, (n, kv) in enumerate(lens):
            hit = bad is not None and n > at and b % 3 != 0
            want.append(2 if hit else 0)
            if hit:
                depth[int(bt.cu_host[b]) + at] = bad
        G.kv_append(k, k, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, cos=cos, sin=sin, depth=depth, status=status)
        assert status.tolist() == want


# ------------------------------------------------------------------------------------------------------------ commit
def plain_commit(bt, tokens, parent, said, start, max_q):
    paths, nexts = [], []
    for b, (n, _) in enumerate(bt.lens):
        at, path, s = int(bt.cu_host[b]), [], start[b]
        if 0 <= s < n:
            j = s
            while j >= 0:
                path.insert(0, j)
                p = parent[at + j]
                j = p if 0 <= p < j else -1
            while True:
                child = [i for i in range(path[-1] + 1, n)
                         if parent[at + i] == path[-1] and said[at + path[-1]] >= 0 and tokens[at + i] == said[at + path[-1]]]
                if not child:
                    break
                path.append(child[0])
        paths.append(path)
        nexts.append(said[at + path[-1]] if path else -1)
    return paths, nexts


def commit_case(bt, seed, vocabulary=4):
    r = random.Random(seed)
    tokens = [r.randrange(vocabulary) for _ in range(bt.T)]
    said = [r.randrange(-1, vocabulary) for _ in range(bt.T)]
    return tokens, said


@pytest.mark.parametrize("lens", [[(1, 1)], [(16, 200)], [(5, 130), (0, 0), (64, 64), (33, 90), (1, 31), (0, 9)],
                                  [(300, 400), (1000, 1024), (129, 700)]])
@pytest.mark.parametrize("page", [1, 16, 24])
@pytest.mark.parametrize("heads", [(4, 4, 128), (3, 3, 8), (24, 12, 64), (40, 40, 256)])
def test_commit(G, lens, page, heads):
    if sum(kv for _, kv in lens) * heads[1] * heads[2] > 1 << 23:
        lens = [(n, kv) for n, kv in lens if kv < 500]
    L = 3
    bt = Trees(lens, heads, page, "bf16", seed=len(lens), reach=3)
    for seed in range(3):
        tokens, said = commit_case(bt, seed, vocabulary=2 + seed)
        r = random.Random(seed)
        start = None if seed == 0 else [r.randrange(-1, n + 1) if n else 0 for n, _ in lens]
        paths, nexts = plain_commit(bt, tokens, bt.parent, said, start or [0] * len(lens), bt.max_q)
        k, v = (torch.randn((L,) + tuple(bt.k.shape), device="cuda").bfloat16() for _ in range(2))
        want_k, want_v = k.clone(), v.clone()
        for b, (n, kv) in enumerate(lens):
            for i, f in enumerate(paths[b]):
                to, fro = (tuple(int(x[0]) for x in bt.rows(b, np.array([kv - n + j]))) for j in (i, f))
                want_k[:, to[0], to[1]] = want_k[:, fro[0], fro[1]].clone()
                want_v[:, to[0], to[1]] = want_v[:, fro[0], fro[1]].clone()
        args = (bt.cu, ints(tokens), ints(bt.parent), ints(said), bt.max_q)
        kw = {} if start is None else {"start": ints(start)}
        path, length, following = G.commit_tree(k, v, bt.table, bt.kv_len, *args, **kw)
        assert length.tolist() == [len(p) for p in paths] and following.tolist() == nexts
        assert path.tolist() == [p + [-1] * (bt.max_q - len(p)) for p in paths]
        assert torch.equal(k, want_k) and torch.equal(v, want_v)
        # the branches alone, without a cache; and a cache of one layer
        again = G.commit_tree(None, None, None, None, *args, **kw)
        assert torch.equal(again[0], path) and torch.equal(again[1], length) and torch.equal(again[2], following)
    one_k, one_v = bt.k.clone(), bt.v.clone()
    both_k, both_v = one_k[None].clone(), one_v[None].clone()
    G.commit_tree(one_k, one_v, bt.table, bt.kv_len, *args)
    G.commit_tree(both_k, both_v, bt.table, bt.kv_len, *args)
    assert torch.equal(one_k, both_k[0]) and torch.equal(one_v, both_v[0])


@pytest.mark.parametrize("n", [2, 63, 64, 65, 128, 257, 1000])
@pytest.mark.parametrize("reach", [1, 2, 70])
def test_branches_to_the_end(G, n, reach):
    """every child matches, so that the branch is the first children's down to a leaf (of a chain all of it)"""
    lens = [(n, n + 5), (1, 1), (n, n)]
    bt = Trees(lens, (2, 1, 64), 16, "bf16", seed=n + reach, reach=reach)
    tokens, said = [0] * bt.T, [0] * bt.T
    for start in ([0, 0, 0], [n - 1, 0, n // 2]):
        paths, nexts = plain_commit(bt, tokens, bt.parent, said, start, bt.max_q)
        assert reach > 1 or [len(p) for p in paths] == [n, 1, n]
        path, length, following = G.commit_tree(None, None, None, None, bt.cu, ints(tokens), ints(bt.parent), ints(said),
                                                bt.max_q, start=ints(start))
        assert path.tolist() == [p + [-1] * (bt.max_q - len(p)) for p in paths]
        assert length.tolist() == [len(p) for p in paths] and following.tolist() == nexts
    # tokens and targets that are no tokens match nothing
    minus = ints([-1] * bt.T)
    _, length, following = G.commit_tree(None, None, None, None, bt.cu, minus, ints(bt.parent), minus, bt.max_q)
    assert length.tolist() == [1, 1, 1] and following.tolist() == [-1, -1, -1]


def test_commit_layouts_and_outputs(G):
    """heads before rows, layers inside pages, outputs that are given, a graph"""
    lens = [(20, 50), (7, 300)]
    bt = Trees(lens, (4, 2, 64), 16, "f16", seed=4, reach=2, heads_first=True)
    L = 2
    store = torch.randn((bt.P, L, 2, bt.hkv, bt.page, bt.D), device="cuda").half()
    k, v = (store[:, :, i].permute(1, 0, 3, 2, 4) for i in range(2))
    flat_k, flat_v = k.contiguous(), v.contiguous()
    # the target agrees with every node's last child
    tokens, said = list(range(bt.T)), [-1] * bt.T
    for b, (n, _) in enumerate(lens):
        at = int(bt.cu_host[b])
        for i in range(1, n):
            said[at + bt.parent[at + i]] = tokens[at + i]
    args = (bt.table, bt.kv_len, bt.cu, ints(tokens), ints(bt.parent), ints(said), bt.max_q)
    want = G.commit_tree(flat_k, flat_v, *args)
    assert not torch.equal(flat_k, k) and not torch.equal(flat_v, v)
    first = store.clone()
    path, length, following = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty_like(want[2])
    got = G.commit_tree(k, v, *args, path=path, length=length, next=following)
    assert got[0] is path and got[1] is length and got[2] is following
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(k, flat_k) and torch.equal(v, flat_v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.commit_tree(k, v, *args, path=path, length=length, next=following)
    for _ in range(3):
        store.copy_(first)
        path.fill_(5), length.fill_(5), following.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((path, length, following), want))
        assert torch.equal(k, flat_k) and torch.equal(v, flat_v)


def test_commit_of_bad_sequences(G):
    lens = [(4, 40), (6, 33), (5, 50), (3, 10)]
    args = None

    def run(change, **kw):
        bt = Trees(lens, (2, 2, 64), 16, "bf16", seed=6, reach=1)
        token, said = [9] * bt.T, [9] * bt.T
        change(bt)
        k, v = bt.k.clone(), bt.v.clone()
        got = G.commit_tree(k, v, bt.table, bt.kv_len, bt.cu, ints(token), ints(bt.parent), ints(said), kw.get("max_q", bt.max_q),
                            start=kw.get("start"))
        assert torch.equal(k, bt.k) and torch.equal(v, bt.v)  # chains: nothing to move in any case
        return got[1].tolist(), got[2].tolist()

    assert run(lambda bt: None) == ([4, 6, 5, 3], [9] * 4)
    assert run(lambda bt: bt.kv_len.__setitem__(1, 5)) == ([4, 0, 5, 3], [9, -1, 9, 9])
    assert run(lambda bt: bt.kv_len.__setitem__(2, 1 << 30)) == ([4, 6, 0, 3], [9, 9, -1, 9])
    assert run(lambda bt: bt.cu.__setitem__(2, 3)) == ([4, 0, 0, 0], [9, -1, -1, -1])
    assert run(lambda bt: bt.cu.__setitem__(4, 100)) == ([4, 6, 5, 0], [9, 9, 9, -1])
    assert run(lambda bt: None, max_q=5) == ([4, 0, 5, 3], [9, -1, 9, 9])
    assert run(lambda bt: None, start=ints([3, 6, -1, 1])) == ([4, 0, 0, 3], [9, -1, -1, 9])
    # a page that is not in the cache: its rows are not moved
    bt = Trees([(6, 36)], (2, 2, 64), 4, "bf16", seed=7)
    parent = [-1, 0, 0, 1, 2, 4]
    bt.table[0, 8] = bt.P + 5  # places 2 .. 5
    k, v = bt.k.clone(), bt.v.clone()
    got = G.commit_tree(k, v, bt.table, bt.kv_len, bt.cu, ints([1, 2, 3, 4, 5, 6]), ints(parent), ints([3, 0, 5, 0, 6, 8]), 6)
    assert got[0].tolist() == [[0, 2, 4, 5, -1, -1]] and got[2].tolist() == [8]
    assert torch.equal(k, bt.k) and torch.equal(v, bt.v)


def test_a_step_with_trees(G):
    """append at depths, attend over the tree, commit: what follows attends as if the branch had been the chunk"""
    lens = [(13, 60), (20, 33)]
    bt = Trees(lens, (4, 2, 64), 16, "bf16", seed=30, reach=4)
    cos, sin = tables(80, 64)
    k, v = bt.rand((bt.T, 2, 64)), bt.rand((bt.T, 2, 64))
    one, two = (bt.k.clone(), bt.v.clone()), (bt.k.clone(), bt.v.clone())
    masks, depth = G.tree_masks(ints(bt.parent), bt.cu, bt.max_q)
    q, _ = G.kv_append(k, v, *one, bt.table, bt.kv_len, bt.cu, q=bt.q, cos=cos, sin=sin, depth=depth)
    out, lse = G.attend_tree(q, *one, bt.table, bt.kv_len, bt.cu, masks, bt.max_q, bt.max_kv)
    # the target agrees with one branch of each tree
    r, tokens, said = random.Random(1), list(range(bt.T)), [-1] * bt.T
    branch = []
    for b, (n, _) in enumerate(lens):
        at, leaf = int(bt.cu_host[b]), n - 1
        path = [leaf]
        while bt.parent[at + path[0]] >= 0:
            path.insert(0, bt.parent[at + path[0]])
        for x, y in zip(path, path[1:]):
            said[at + x] = tokens[at + y]
        said[at + leaf] = 1000 + b
        branch.append(path)
    path, length, following = G.commit_tree(*one, bt.table, bt.kv_len, bt.cu, ints(tokens), ints(bt.parent), ints(said), bt.max_q)
    assert [p[:n] for p, n in zip(path.tolist(), length.tolist())] == branch and following.tolist() == [1000, 1001]
    # the same tokens as plain chunks
    rows = torch.tensor([int(bt.cu_host[b]) + i for b, p in enumerate(branch) for i in p], device="cuda")
    cu = ints([0, len(branch[0]), len(rows)])
    kv = ints([kv - n + len(p) for (n, kv), p in zip(lens, branch)])
    q2, _ = G.kv_append(k[rows], v[rows], *two, bt.table, kv, cu, q=bt.q[rows], cos=cos, sin=sin)
    assert torch.equal(q2, q[rows])
    want, want_lse = G.attend(q2, *two, bt.table, kv, cu, 40, 80)
    u = U[bt.dt]
    assert bool(((out[rows].double() - want.double()).abs() <= 4 * u * (want.double().abs() + 1)).all())
    for b, ((n, kv_), p) in enumerate(zip(lens, branch)):
        for s in range(kv_ - n + len(p)):
            page, row = (int(x[0]) for x in bt.rows(b, np.array([s])))
            assert torch.equal(one[0][page, row], two[0][page, row]) and torch.equal(one[1][page, row], two[1][page, row])


@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 3, 64), (4, 1, 256)])
@pytest.mark.parametrize("B", [63, 64, 65, 150])
def test_many_sequences(G, heads, B):
    """shares of ragged trees over long and short caches, empty chunks among them"""
    r = random.Random(B)
    lens = []
    for i in range(B):
        n = r.choice([0, 1, 2, 9, 40, 64, 64 // (heads[0] // heads[1]) + 1])
        lens.append((n, n + r.choice([0, 1, 63, 64, 65, 300, r.randint(0, 2500)])))
    lens[B // 2] = (64, 2600)
    bt = Trees(lens, heads, 16, "bf16", seed=B)
    got = bt.attend(G)
    agree(got, bt)
    again = bt.attend(G, max_kv=1 << 20)
    agree(again, bt)
    # a chunk out of order: it and all after it are bad
    bt.cu[B // 2 + 1] = 0
    got = bt.attend(G)
    first = int(bt.cu_host[B // 2])
    assert bool(torch.isnan(got[0][first:].float()).all()) and bool(torch.isfinite(got[0][:first].float()).all())


@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 3, 64), (4, 1, 256), (28, 4, 128)])
@pytest.mark.parametrize("page,window", [(16, 0), (24, 0), (16, 150), (100, 1900)])
def test_many_trees_of_short_texts(G, heads, page, window):
    """so many that whole tiles fill the chip; under a window after longer texts too"""
    r = random.Random(page)
    lens, most = [], 1024 if window == 0 else 3000
    for i in range(190):
        n = r.choice([0, 1, 2, 31, 33, 63, 64])
        lens.append((n, n + r.choice([0, 1, 63, 64, 65, 300, r.randint(0, most - 64)]) if n else 0))
    lens[7], lens[100] = (64, most), (64, 64)
    bt = Trees(lens, heads, page, "bf16", seed=page)
    got = bt.attend(G, window=window)
    agree(got, bt, window=window)
    again = bt.attend(G, window=window)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    # what is not seen has no part: free pages
    used = torch.zeros(bt.k.shape[:2], dtype=torch.bool)
    for b, (n, kv) in enumerate(lens):
        if kv:
            page_of, row = bt.rows(b, np.arange(kv))
            used[torch.from_numpy(np.asarray(page_of)).long(), torch.from_numpy(np.asarray(row)).long()] = True
    used = used.cuda()
    bt.k[~used] = math.nan
    bt.v[~used] = math.nan
    again = bt.attend(G, window=window)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    # a chunk out of order: it and all after it are bad
    bt.cu[101] = 0
    got = bt.attend(G, window=window)
    first = int(bt.cu_host[100])
    assert bool(torch.isnan(got[0][first:].float()).all()) and bool(torch.isfinite(got[0][:first].float()).all())


def test_offsets_past_32_bits(G):
    """a cache of more than 2^32 entries: the sequence's pages lie at its end"""
    page, H, D = 64, 8, 128
    P = (1 << 32) // (page * H * D) + 40
    bt = Trees([(40, 1500)], (16, H, D), page, "bf16", seed=15)
    n = bt.k.shape[0]
    big_k, big_v = (torch.empty((P, page, H, D), dtype=bt.dt, device="cuda") for _ in range(2))
    big_k[-n:], big_v[-n:] = bt.k, bt.v
    want = bt.attend(G)
    table = bt.table + (P - n)
    got = G.attend_tree(bt.q, big_k, big_v, table, bt.kv_len, bt.cu, bt.tree, bt.max_q, bt.max_kv)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    tokens, said = list(range(bt.T)), [-1] * bt.T
    for i in range(1, bt.T):
        said[bt.parent[i]] = tokens[i]
    args = (bt.kv_len, bt.cu, ints(tokens), ints(bt.parent), ints(said), bt.max_q)
    one = G.commit_tree(big_k, big_v, table, *args)
    two = G.commit_tree(bt.k, bt.v, bt.table, *args)
    assert all(torch.equal(x, y) for x, y in zip(one, two))
    assert torch.equal(big_k[-n:], bt.k) and torch.equal(big_v[-n:], bt.v)
