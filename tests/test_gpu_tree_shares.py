"""Tree attention whose work is cut into shares, where there is nothing to share: no sequence has a new token, or none is good.
Nothing is computed here, so what is compared is equal: rows of bad sequences are NaN, other rows are left as they are."""

import pytest

torch = pytest.importorskip("torch")

from test_gpu_tree import G, Trees  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# sequences, nodes, cached tokens, heads: rows a key head and keys such that the launch is of shares of tiles of 32 and 64 rows
# (one a sequence), 128 and 256 (any number), with a lane a sequence (up to 64) and without
SHARED = [(1, 3, 1500, (8, 2, 128)), (70, 3, 3000, (8, 2, 128)), (1, 12, 1500, (8, 2, 128)), (70, 12, 3000, (6, 2, 256)),
          (1, 16, 1500, (28, 4, 128)), (3, 40, 1200, (4, 2, 64)), (70, 10, 1100, (28, 4, 128)), (66, 20, 1100, (6, 1, 256)),
          (1, 40, 33000, (16, 1, 128)), (2, 40, 33000, (16, 1, 64)), (70, 40, 1100, (28, 4, 128)), (90, 50, 1100, (16, 2, 64))]


def attend(G, bt, out, lse):  # noqa: F811
    out.fill_(7.0), lse.fill_(7.0)
    bt.attend(G, out=out, lse=lse)
    return out, lse


@pytest.mark.parametrize("B,n,kv,heads", SHARED)
def test_nothing_to_share(G, B, n, kv, heads):  # noqa: F811
    bt = Trees([(n, kv)] * min(B, 4), heads, 16, "bf16", seed=B)
    # (the sequences' caches are one another's: nothing writes them)
    of = torch.arange(B, device="cuda") % len(bt.lens)
    token = (of[:, None] * n + torch.arange(n, device="cuda")).flatten()
    bt.q, bt.tree, bt.depth, bt.table, bt.kv_len = bt.q[token], bt.tree[token], bt.depth[token], bt.table[of], bt.kv_len[of]
    bt.cu = torch.arange(0, (B + 1) * n, n, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(bt.q), torch.empty(bt.q.shape[:2], device="cuda")
    good = [x.clone() for x in attend(G, bt, out, lse)]
    assert bool(torch.isfinite(good[0].float()).all()) and bool(torch.isfinite(good[1]).all())
    cu, kv_len = bt.cu.clone(), bt.kv_len.clone()

    def nan(rows):
        bad = torch.zeros(B * n, dtype=torch.bool, device="cuda")
        bad[rows] = True
        assert torch.equal(torch.isnan(out.float()).all(-1).all(-1), bad) and torch.equal(torch.isnan(lse).all(-1), bad)
        assert bool((out[~bad] == 7).all()) and bool((lse[~bad] == 7).all())

    # no sequence has a token, at the rows' beginning and at their end
    for at in (0, B * n):
        bt.cu = torch.full_like(cu, at)
        attend(G, bt, out, lse)
        nan(slice(0, 0))
    bt.cu = cu
    # every sequence bad: more cached tokens than the call or the table allows, fewer than new ones
    for length in (kv + 1, 1 << 30, n - 1, -5):
        bt.kv_len = torch.full_like(kv_len, length)
        attend(G, bt, out, lse)
        nan(slice(None))
    bt.kv_len = kv_len
    # longer chunks than the call allows (the launch is that of the chunks that it does)
    if n > 3:
        out.fill_(7.0), lse.fill_(7.0)
        bt.attend(G, out=out, lse=lse, max_q=n - 1)
        nan(slice(None))
    # out of order from the first on
    bt.cu = cu.clone()
    bt.cu[0] = bt.cu[1] + 1
    attend(G, bt, out, lse)
    nan(slice(n + 1, None))
    bt.cu = cu.clone()
    bt.cu[1] = B * n + 1
    attend(G, bt, out, lse)
    nan(slice(None))
    # some empty, the others bad
    if B > 1:
        bt.cu = torch.minimum(cu, cu[B // 2])
        bt.kv_len = torch.full_like(kv_len, -1)
        attend(G, bt, out, lse)
        nan(slice(0, B // 2 * n))
    bt.cu, bt.kv_len = cu, kv_len
    again = attend(G, bt, out, lse)
    assert torch.equal(again[0], good[0]) and torch.equal(again[1], good[1])


@pytest.mark.parametrize("B,n,kv,heads", [SHARED[4], SHARED[8], SHARED[9]])
def test_a_captured_step_without_work(G, B, n, kv, heads):  # noqa: F811
    """a graph of a full batch, replayed with sequences that have ended"""
    bt = Trees([(n, kv)] * B, heads, 16, "bf16", seed=3)
    out, lse = torch.empty_like(bt.q), torch.empty(bt.q.shape[:2], device="cuda")
    want = [x.clone() for x in attend(G, bt, out, lse)]
    workspace = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    cu = bt.cu.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bt.attend(G, out=out, lse=lse, workspace=workspace)
    for ended in (False, True, True, False, True):
        out.fill_(7.0), lse.fill_(7.0), workspace.fill_(255)
        bt.cu.copy_(torch.zeros_like(cu) if ended else cu)
        graph.replay()
        torch.cuda.synchronize()
        if ended:
            assert bool((out == 7).all()) and bool((lse == 7).all())
        else:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
