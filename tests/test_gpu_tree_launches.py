"""Tree attention in every launch that sizes choose: shares of tiles of 32, 64, 128 and 256 rows and whole tiles of 32 and 128, of heads
of 64, 128 and 256, pages of whole runs of 16 rows and others; against the 64-bit reference of test_gpu_tree.py within its
bounds, and what no row sees, and what some see, set to infinities and NaN."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_tree import G, Trees, agree  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def ragged(B, n, kv):
    return [(n, kv)] + [(max(1, n - b % 4 * (n // 4)), kv - b % 7 * (kv // 9)) for b in range(1, B)]


LAUNCHES = {  # sequences, nodes, cached tokens, heads; a window under which the launch is the same one
    "32 shared, 64": (2, 3, 1500, (8, 2, 64), 900), "32 shared, 128": (3, 4, 1100, (16, 2, 128), 800),
    "32 shared, 256": (2, 5, 900, (6, 1, 256), 500), "32 shared by many, 64": (80, 8, 2600, (8, 2, 64), 2100),
    "64 shared, 64": (3, 30, 1200, (6, 3, 64), 800), "64 shared, 128": (2, 12, 1500, (8, 2, 128), 900),
    "64 shared, 256": (2, 12, 900, (4, 1, 256), 500), "64 shared by many, 128": (70, 12, 2600, (20, 4, 128), 2200),
    "64 shared by many, 256": (70, 13, 600, (8, 2, 256), 390),
    "128 shared, 64": (2, 100, 1500, (4, 4, 64), 1100), "128 shared, 128": (3, 25, 1500, (8, 2, 128), 1000),
    "128 shared, 256": (2, 100, 1500, (4, 1, 256), 1200), "128 shared by many, 64": (70, 20, 1300, (20, 4, 64), 2100),
    "256 shared, 64": (6, 64, 4300, (16, 4, 64), 4200), "256 shared, 128": (6, 64, 2300, (32, 8, 128), 2100),
    "256 shared, odd rows, 64": (9, 61, 4000, (15, 5, 64), 2500), "256 shared by many, 64": (90, 45, 2600, (16, 2, 64), 2100),
    "128 whole, 64": (64, 32, 900, (32, 8, 64), 500), "128 whole, 128": (80, 50, 700, (14, 7, 128), 300),
    "128 whole, 256": (130, 60, 500, (4, 2, 256), 250), "32 whole, 64": (2, 40, 500, (15, 5, 64), 100),
    "32 whole, 256": (3, 9, 300, (8, 2, 256), 100)}


@pytest.mark.parametrize("name", list(LAUNCHES))
@pytest.mark.parametrize("page,dtype", [(16, "bf16"), (24, "f16"), (100, "bf16")])
def test_launches(G, name, page, dtype):  # noqa: F811
    B, n, kv, heads, window = LAUNCHES[name]
    bt = Trees(ragged(B, n, kv), heads, page, dtype, seed=B + page, roots=0.02)
    for w in (0, window):
        got = bt.attend(G, window=w)
        agree(got, bt, window=w)
        again = bt.attend(G, window=w)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("name", list(LAUNCHES))
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_what_is_seen_and_what_is_not(G, name, poison):  # noqa: F811
    B, n, kv, heads, window = LAUNCHES[name]
    lens = ragged(B, n, kv)
    bt = Trees(lens, heads, 16, "bf16", seed=B, spare=3)
    clean = bt.attend(G, window=window)
    # free pages, rows after a sequence's end, and before its window
    dead = torch.ones(bt.k.shape[:2], dtype=torch.bool)
    for b, (m, c) in enumerate(lens):
        page, row = bt.rows(b, np.arange(max(0, c - m - window + 1), c))
        dead[torch.from_numpy(page.astype(np.int64)), torch.from_numpy(row)] = False
    dead = dead.cuda()
    for pages in (bt.k, bt.v):
        pages[dead] = poison
    got = bt.attend(G, window=window)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    # a value in the middle of each tree, and one of the text that all see: of one dimension
    for place in ("tree", "text"):
        v, sees, e = bt.v.clone(), torch.zeros(bt.T, dtype=torch.bool, device="cuda"), heads[2] - 5
        for b, (m, c) in enumerate(lens):
            i, at = m // 2, int(bt.cu_host[b])
            sees[at:at + m] = True if place == "text" else (bt.tree[at:at + m, i // 32] >> i % 32 & 1).bool()
            page, row = bt.rows(b, np.array([c - m - 1 if place == "text" else c - m + i]))
            v[int(page[0]), int(row[0]), :, e] = poison
        out, lse = G.attend_tree(bt.q, bt.k, v, bt.table, bt.kv_len, bt.cu, bt.tree, bt.max_q, bt.max_kv, depth=bt.depth,
                                 window=window)
        other = torch.arange(heads[2], device="cuda") != e
        assert torch.equal(out[:, :, other], clean[0][:, :, other]) and torch.equal(lse, clean[1])
        assert torch.equal(out[~sees], clean[0][~sees])
        hit = out[sees][:, :, e].float()
        assert bool((torch.isnan(hit) if math.isnan(poison) else hit == poison).all())
