"""Statuses of an append at depths: whole numbers, equal."""

import pytest

torch = pytest.importorskip("torch")

from test_gpu_tree import G, Trees, tables  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [1, 5, 300])
def test_sequences_without_a_token_ask_for_no_position(G, B):  # noqa: F811
    """caches longer than the table of positions: no token of theirs is rotated, as in an append without depths"""
    lens = [(0, 200), (3, 64)] + [(0, 101 + i % 7) for i in range(B)] + [(2, 101)]
    bt = Trees(lens, (2, 1, 64), 16, "bf16", seed=B)
    k = bt.rand((bt.T, 1, 64))
    cos, sin = tables(100, 64)
    for depth in (bt.depth, None):
        status = torch.full((len(lens),), -1, dtype=torch.int32, device="cuda")
        G.kv_append(k, k, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, cos=cos, sin=sin, depth=depth, status=status)
        assert status.tolist() == [0] * (len(lens) - 1) + [2]
