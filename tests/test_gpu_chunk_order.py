"""Chunks that are not in order: from the first such sequence on all are bad, whatever the later ones say by themselves.
Those before keep their results, no row is written twice, and statuses and NaN say the same.

Bounds of what is compared are those of test_gpu_attend.py (the sequences before are computed by its reference).
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attend import G, Batch, agree  # noqa: E402,F401

pytestmark = pytest.mark.gpu

# lengths, and which launch they reach: all keys at once; shares and their joining; shares over more sequences than a wave
# has lanes; tiles of 128 rows; the same split and joined
DIRECT = [(2, 90), (4, 40), (3, 64), (1, 100), (5, 77), (2, 30)]
SHARES = [(2, 900), (4, 1400), (3, 64), (1, 2000), (5, 77), (2, 300)]
MANY = [(1 + i % 4, 2500 if i == 5 else 10 + 37 * i % 900) for i in range(150)]
TILES = [(200, 900), (4, 1400), (150, 160), (1, 2000), (90, 777), (2, 300)] * 12
SPLIT = [(70, 4000), (4, 1400), (40, 64), (1, 4000), (50, 777), (2, 300)]
LAUNCHES = {"direct": DIRECT, "shares": SHARES, "many": MANY, "tiles": TILES, "split": SPLIT}


def spoil(cu, T, at, how):
    """entry `at` of cu, in the middle of others that are in order by themselves, and the first sequence that this breaks"""
    cu = cu.copy()
    if how == "large":
        cu[at] = T + 10000
        return cu, at - 1
    if how == "negative":
        cu[at] = -3
        return cu, at - 1
    if how == "back":  # the sequence before ends before its start
        cu[at] = cu[at - 1] - 1
        return cu, at - 1
    cu[at] = cu[at + 1] + 1  # "forward": the sequence from here on does, or the one before leaves the rows
    return cu, at if cu[at] <= T else at - 1


@pytest.mark.parametrize("how", ["large", "negative", "back", "forward"])
@pytest.mark.parametrize("launch", LAUNCHES)
def test_attend(G, launch, how):
    lens = LAUNCHES[launch]
    bt = Batch(lens, (8, 2, 128), 16, "bf16", seed=31)
    out = torch.full_like(bt.q, 7.0)
    lse = torch.full((bt.T, bt.hq), 7.0, device="cuda")
    for at in {2, len(lens) // 2, len(lens) - 1}:
        cu, first = spoil(bt.cu_host, bt.T, at, how)
        bt.cu = torch.from_numpy(cu).cuda()
        got = bt.attend(G, out=out.clone(), lse=lse.clone())
        bad = torch.zeros(bt.T, dtype=torch.bool, device="cuda")
        bad[max(0, int(cu[first])):] = True
        assert bool(torch.isnan(got[0][bad].float()).all()) and bool(torch.isnan(got[1][bad]).all())
        if how == "forward":  # the sequence before ends later than it did: its rows are others
            bad[int(bt.cu_host[first - 1]):] = True
        agree(got, bt, rows=~bad)


@pytest.mark.parametrize("first", [-1, 1 << 30])
def test_the_first_entry(G, first):
    bt = Batch(SHARES, (8, 2, 128), 16, "bf16", seed=32)
    for max_kv in (bt.max_kv, 100):
        bt.cu = torch.from_numpy(bt.cu_host).cuda()
        bt.cu[0] = first
        out, lse = bt.attend(G, out=torch.full_like(bt.q, 7.0), max_kv=max_kv)
        if first < 0:
            assert bool(torch.isnan(out.float()).all()) and bool(torch.isnan(lse).all())
        else:
            assert bool((out == 7.0).all())  # no token comes after it


@pytest.mark.parametrize("n", [6, 700])
@pytest.mark.parametrize("how", ["large", "negative", "back", "forward"])
def test_append(G, n, how):
    lens = [(1 + i % 5, 20 + 3 * i % 50) for i in range(n)]
    bt = Batch(lens, (4, 2, 64), 16, "bf16", seed=33)
    k, v = bt.rand((bt.T, 2, 64)), bt.rand((bt.T, 2, 64))
    place = [bt.rows(b, np.arange(kv - m, kv)) for b, (m, kv) in enumerate(lens)]
    for at in {2, n // 2, n - 1}:
        cu, first = spoil(bt.cu_host, bt.T, at, how)
        bt.k.zero_(), bt.v.zero_()
        q_out, status = torch.full_like(bt.q, 7.0), torch.full((n,), -1, dtype=torch.int32, device="cuda")
        G.kv_append(k, v, bt.k, bt.v, bt.table, bt.kv_len, torch.from_numpy(cu).cuda(), q=bt.q, q_out=q_out, status=status)
        whole = first - 1 if how == "forward" else first  # sequences with their own tokens and places
        assert status.tolist() == [0] * first + [2] * (n - first)
        want_k, want_v, want_q = torch.zeros_like(bt.k), torch.zeros_like(bt.v), torch.full_like(bt.q, 7.0)
        for b in range(first):
            m = int(cu[b + 1] - cu[b])
            s = torch.arange(int(cu[b]), int(cu[b + 1])).cuda()
            page, row = place[b] if b < whole else bt.rows(b, np.arange(lens[b][1] - m, lens[b][1]))
            page, row = torch.from_numpy(page.astype(np.int64)).cuda(), torch.from_numpy(row.astype(np.int64)).cuda()
            want_k[page, row], want_v[page, row], want_q[s] = k[s], v[s], bt.q[s]
        assert torch.equal(bt.k, want_k) and torch.equal(bt.v, want_v) and torch.equal(q_out, want_q)
