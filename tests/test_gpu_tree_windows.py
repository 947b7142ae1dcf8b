"""Trees deeper than a sliding window: grid_tree_masks_window and grid_attend_tree with its bits.  Bits and depths are whole numbers
and equal; attention is compared with the 64-bit references of test_gpu_tree.py (by bits) and, where a tree is one branch, of
test_gpu_attend.py (by positions), within their bounds."""

import pytest

torch = pytest.importorskip("torch")

import test_gpu_attend  # noqa: E402
from test_gpu_tree import G, Trees, agree, ints, plain_masks, random_parents  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def within(words, depth, cu, window):
    """the bits of places whose depth is above the node's less the window"""
    out = torch.zeros_like(words)
    for at, end in zip(cu[:-1], cu[1:]):
        n = end - at
        if n == 0:
            continue
        bits = (words[at:end, :, None] >> torch.arange(32, dtype=torch.int32, device="cuda") & 1).flatten(1)[:, :n].bool()
        bits &= depth[at:end][None] > depth[at:end, None] - window
        full = torch.zeros((n, out.shape[1] * 32), dtype=torch.int64, device="cuda")
        full[:, :n] = bits.long()
        x = (full.view(n, -1, 32) << torch.arange(32, device="cuda")).sum(-1)
        out[at:end] = torch.where(x >= 1 << 31, x - (1 << 32), x).int()
    return out


@pytest.mark.parametrize("lens", [[(1, 1)], [(5, 9), (0, 3), (64, 64), (1, 7), (33, 40), (130, 200)], [(300, 300), (1024, 1024)]])
@pytest.mark.parametrize("reach,roots", [(1, 0.0), (3, 0.02), (1000, 0.0)])
@pytest.mark.parametrize("window", [1, 2, 3, 31, 32, 33, 63, 64, 65, 127, 500, 1023, 1024, 2 ** 31 - 1])
def test_masks_under_a_window(G, lens, reach, roots, window):  # noqa: F811
    parent = random_parents(lens, window, reach, roots)
    max_q = max(n for n, _ in lens)
    words, depth = plain_masks(lens, parent, max_q)
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    got = G.tree_masks(ints(parent), ints(cu), max_q, window=window)
    assert torch.equal(got[0], within(words, depth, cu, window)) and torch.equal(got[1], depth)
    if int(depth.max()) < window:
        assert torch.equal(got[0], words)


# sequences, nodes, cached tokens, heads, window, such that the launch is of tiles of 32 rows (whole, and shares of them), of 64,
# of 128 (shares, and whole), of 256; the trees are deeper than the window
LAUNCHES = [(2, 40, 300, (28, 4, 128), 25), (300, 20, 90, (2, 2, 64), 9), (150, 40, 90, (2, 2, 64), 17),
            (140, 25, 60, (4, 2, 128), 16), (130, 20, 50, (6, 3, 256), 8), (100, 50, 120, (8, 4, 128), 20),
            (200, 50, 120, (8, 4, 128), 33), (130, 60, 100, (4, 2, 256), 31), (1, 900, 2000, (28, 4, 128), 700),
            (2, 700, 1200, (16, 2, 64), 400), (1, 1000, 1000, (4, 1, 256), 128)]


def ragged(B, n, kv):
    return [(n, kv)] + [(n - b % 3 * (n // 4), kv - b % 5 * 7) for b in range(1, B)]


@pytest.mark.parametrize("B,n,kv,heads,window", LAUNCHES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_branch_is_a_chunk_under_a_window(G, B, n, kv, heads, window, dtype):  # noqa: F811
    bt = Trees(ragged(B, n, kv), heads, 16, dtype, seed=n, reach=1)
    bt.tree, bt.depth = G.tree_masks(ints(bt.parent), bt.cu, bt.max_q, window=window)
    test_gpu_attend.agree(bt.attend(G, window=window), bt, window=window)
    # what the same call says of it as a chunk
    test_gpu_attend.agree(G.attend(bt.q, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, bt.max_q, bt.max_kv, window=window), bt,
                          window=window)


@pytest.mark.parametrize("B,n,kv,heads,window", LAUNCHES)
def test_deep_trees_under_a_window(G, B, n, kv, heads, window):  # noqa: F811
    window = (window + 1) // 2  # (a node's parent is one or two places before it)
    bt = Trees(ragged(B, n, kv), heads, 24, "bf16", seed=n, reach=2)
    whole, depth = bt.tree, bt.depth
    bt.tree, bt.depth = G.tree_masks(ints(bt.parent), bt.cu, bt.max_q, window=window)
    assert torch.equal(bt.tree, within(whole, depth, bt.cu_host.tolist(), window)) and torch.equal(bt.depth, depth)
    assert not torch.equal(bt.tree, whole)
    agree(bt.attend(G, window=window), bt, window=window)
