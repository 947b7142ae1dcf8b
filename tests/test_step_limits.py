"""Sizes at the limits of what the kernels of a model's step count in: refused on the host, before anything is enqueued.
Through the C ABI, with addresses that are never read."""

import ctypes

import pytest

from test_step_host import S, append, attend, cache, chunks, refused, verify  # noqa: F401

by = ctypes.byref


@pytest.mark.parametrize("V", [(1 << 30) - 2047, 1 << 30, (1 << 31) - 4096 - 1, (1 << 31) - 1])
def test_vocabularies_are_counted_in_32_bits(S, V):  # noqa: F811
    """the pieces of a row and the parts of the race end less than 2^31 after its start"""
    assert S.lib().grid_verify_workspace_bytes(1, 0, V) == 0
    refused(S, S.lib().grid_verify(by(verify(S, V=V, workspace_bytes=1 << 62)), None), "sizes")


def test_the_largest_vocabulary(S):  # noqa: F811
    V = (1 << 30) - 2048
    assert S.lib().grid_verify_workspace_bytes(1, 0, V) > 0
    for steps in (2, 4):  # of 2048 tokens, in a piece of float32 and of 16-bit rows
        piece = steps * 2048
        assert -(-V // piece) * piece < 1 << 31
    for B in (1, 2, 3, 100, 700, 1024, 65535):
        n = min(max(1, 1024 // B), -(-V // 2048))
        race = -(-(-(-V // n)) // 2048) * 2048
        assert -(-V // race) * race < 1 << 31


def test_stages_of_a_sequence_are_counted_in_32_bits(S):  # noqa: F811
    """64 keys a stage and key head: 2^38 keys in all heads are too many, as bounds or as a window's span; fewer are not"""
    c = cache(S, n_kv_heads=1024, page_size=65536, head_dim=64)
    x = chunks(S, table_cols=8192, table_stride=8192)

    def both(**kw):
        a = attend(S, n_heads=1024, **kw)
        size = S.lib().grid_attend_workspace_bytes(by(c), by(x), by(a))
        a.workspace = None  # refused at the latest for this
        return size, S.lib().grid_attend(by(c), by(x), by(a), None)

    for kw in (dict(max_kv=1 << 28), dict(max_kv=1 << 29), dict(max_kv=(1 << 28) - 63),
               dict(max_kv=1 << 30, window=1 << 28)):
        assert both(**kw) == (0, -11), kw  # GRID_E_CAPACITY
        assert "keys" in S.lib().grid_last_error().decode()
    for kw in (dict(max_kv=(1 << 28) - 64), dict(max_kv=1 << 30, window=1 << 27)):
        size, rc = both(**kw)
        assert size > 0 and rc == -1, kw


def test_tiles_are_counted_by_rows(S):  # noqa: F811
    """a launch has 2^23 workgroups: rows that need more are refused, before anything is enqueued"""
    c = cache(S, n_kv_heads=1024, head_dim=64, k_stride=S._THREE(1 << 20, 1 << 16, 64), v_stride=S._THREE(1 << 20, 1 << 16, 64))
    a = attend(S, n_heads=1024, max_q=1 << 24, max_kv=80)
    rc = S.lib().grid_attend(by(c), by(chunks(S, n_tokens=1 << 24)), by(a), None)
    assert rc == -11 and "rows" in S.lib().grid_last_error().decode()


def test_a_style_that_is_neither_true_nor_false(S):  # noqa: F811
    """an error raised while the argument is read is the call's own, not left behind a result"""
    torch = pytest.importorskip("torch")
    pages, table = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 5, dtype=torch.int32)
    k, lens, cu = torch.zeros(7, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for bad in (torch.zeros(2), torch.zeros(0, 3)):
        with pytest.raises(TypeError, match="interleaved"):
            S.G.kv_append(k, k, pages, pages, table, lens, cu, interleaved=bad)
