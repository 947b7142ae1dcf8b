"""What grid_kv_append, grid_attend and grid_verify refuse: every check is made on the host before anything is enqueued,
so it is tested through the C ABI with addresses that are never read."""

import ctypes

import pytest

AT = 1 << 20  # an address of the right alignment


@pytest.fixture(scope="module")
def S():
    pytest.importorskip("torch")
    import paper_2607_11951_amd as pkg
    if not pkg.grid.LIB_PATH.exists():
        from paper_2607_11951_amd import build
        build.build()
    from paper_2607_11951_amd import step
    return step


def cache(S, **kw):
    c = S._Cache(AT, AT, 1, 10, 16, 4, 128, S._THREE(8192, 512, 128), S._THREE(8192, 512, 128))
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def chunks(S, **kw):
    c = S._Chunks(3, 7, AT, 5, 5, AT, AT)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append(S, **kw):
    a = S._Append(AT, AT, AT, AT, 8, S._TWO(512, 128), S._TWO(512, 128), S._TWO(1024, 128), S._TWO(1024, 128), AT, AT, 64,
                  128, 0, None, None, 1e-6, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def attend(S, **kw):
    a = S._Attend(AT, AT, S._TWO(1024, 128), S._TWO(1024, 128), AT, 8, 4, 80, 0, 0.1, AT, 1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def verify(S, **kw):
    a = S._Verify(AT, 1, 2, 3, 1000, S._TWO(4000, 1000), AT, S._TWO(128, 32), AT, None, AT, S._TWO(3000, 1000), AT, AT,
                  1000, None, AT, AT, AT, AT, 1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def refused(S, rc, word):
    assert rc == -1  # GRID_E_ARG
    assert word in S.lib().grid_last_error().decode()


BAD_CACHE = [("k_pages", None), ("v_pages", None), ("k_pages", AT + 8), ("v_pages", AT + 2), ("dtype", 0), ("dtype", 7),
             ("n_pages", 0), ("n_pages", -1), ("page_size", 0), ("page_size", 65537), ("n_kv_heads", 0),
             ("n_kv_heads", 1025), ("head_dim", 0), ("head_dim", 100), ("head_dim", 264), ("k_stride", (8192, 512, 100)),
             ("v_stride", (8192, 4, 128)), ("k_stride", (-8192, 512, 128))]
BAD_CHUNKS = [("n_seqs", 0), ("n_seqs", 65536), ("n_tokens", -1), ("n_tokens", (1 << 24) + 1), ("block_table", None),
              ("table_stride", 4), ("table_cols", 0), ("kv_len", None), ("cu_q", None)]
BAD_APPEND = [("k", None), ("v", None), ("q_out", None), ("n_heads", 0), ("n_heads", 2000), ("k", AT + 4),
              ("v_stride", (512, 100)), ("q_stride", (1024, 4)), ("q_out_stride", (-8, 128)), ("cos", None),
              ("sin", None), ("n_positions", 0), ("rot_dim", 0), ("rot_dim", 24), ("rot_dim", 144), ("eps", -1.0),
              ("eps", float("nan"))]
BAD_ATTEND = [("q", None), ("out", None), ("q", AT + 2), ("q_stride", (1024, 12)), ("out_stride", (1, 128)),
              ("n_heads", 0), ("n_heads", 6), ("n_heads", 1028), ("max_q", 0), ("max_kv", 0), ("window", -1),
              ("scale", float("inf")), ("scale", float("nan")), ("workspace", None), ("workspace", AT + 1),
              ("workspace_bytes", 0)]
BAD_VERIFY = [("logits", None), ("dtype", 3), ("dtype", -1), ("B", 0), ("B", 65536), ("K", -1), ("K", 64), ("V", 0),
              ("draft", None), ("uniform", None), ("noise", None), ("logits_stride", (-1, 1000)),
              ("mask_stride", (128, -32)), ("probs_stride", (-3, 1)), ("noise_stride", -1), ("tokens", None),
              ("accepted", None), ("logprobs", None), ("workspace", None), ("workspace", AT + 4), ("workspace_bytes", 8)]


def value(S, v):
    return S._THREE(*v) if isinstance(v, tuple) and len(v) == 3 else S._TWO(*v) if isinstance(v, tuple) else v


@pytest.mark.parametrize("name,bad", BAD_CACHE)
def test_bad_cache(S, name, bad):
    c, x, L = cache(S, **{name: value(S, bad)}), chunks(S), S.lib()
    refused(S, L.grid_kv_append(ctypes.byref(c), ctypes.byref(x), ctypes.byref(append(S)), None), "grid_kv_append")
    refused(S, L.grid_attend(ctypes.byref(c), ctypes.byref(x), ctypes.byref(attend(S)), None), "grid_attend")


@pytest.mark.parametrize("name,bad", BAD_CHUNKS)
def test_bad_chunks(S, name, bad):
    c, x, L = cache(S), chunks(S, **{name: bad}), S.lib()
    refused(S, L.grid_kv_append(ctypes.byref(c), ctypes.byref(x), ctypes.byref(append(S)), None), "grid_kv_append")
    refused(S, L.grid_attend(ctypes.byref(c), ctypes.byref(x), ctypes.byref(attend(S)), None), "grid_attend")


@pytest.mark.parametrize("name,bad", BAD_APPEND)
def test_bad_append(S, name, bad):
    a = append(S, **{name: value(S, bad)})
    refused(S, S.lib().grid_kv_append(ctypes.byref(cache(S)), ctypes.byref(chunks(S)), ctypes.byref(a), None),
            "grid_kv_append")


@pytest.mark.parametrize("name,bad", BAD_ATTEND)
def test_bad_attend(S, name, bad):
    a = attend(S, **{name: value(S, bad)})
    refused(S, S.lib().grid_attend(ctypes.byref(cache(S)), ctypes.byref(chunks(S)), ctypes.byref(a), None), "grid_attend")


@pytest.mark.parametrize("name,bad", BAD_VERIFY)
def test_bad_verify(S, name, bad):
    refused(S, S.lib().grid_verify(ctypes.byref(verify(S, **{name: value(S, bad)})), None), "grid_verify")


def test_more_refusals(S):
    L = S.lib()
    by = ctypes.byref
    for call in (L.grid_kv_append, L.grid_attend):
        a = append(S) if call is L.grid_kv_append else attend(S)
        assert call(None, by(chunks(S)), by(a), None) == -1
        assert call(by(cache(S)), None, by(a), None) == -1
        assert call(by(cache(S)), by(chunks(S)), None, None) == -1
    assert L.grid_verify(None, None) == -1
    # heads of a size that only the append takes
    refused(S, L.grid_attend(by(cache(S, head_dim=80)), by(chunks(S)), by(attend(S)), None), "head_dim")
    # a table of 2^31 positions
    refused(S, L.grid_attend(by(cache(S, page_size=65536)), by(chunks(S, table_cols=32768, table_stride=32768)),
                             by(attend(S)), None), "positions")
    # interleaved pairs need a multiple of 8 only, halves one of 16
    refused(S, L.grid_kv_append(by(cache(S)), by(chunks(S)), by(append(S, rot_dim=12, interleaved=1)), None), "rot_dim")
    # probabilities of a drafter without random numbers
    refused(S, L.grid_verify(by(verify(S, uniform=None, noise=None)), None), "random")


def test_nothing_to_do(S):
    """no tokens and no statuses: nothing is enqueued, nothing is read"""
    L, by = S.lib(), ctypes.byref
    assert L.grid_kv_append(by(cache(S)), by(chunks(S, n_tokens=0)), by(append(S)), None) == 0
    assert L.grid_attend(by(cache(S)), by(chunks(S, n_tokens=0)), by(attend(S, workspace=None)), None) == 0


def test_workspace_sizes(S):
    L, by = S.lib(), ctypes.byref
    assert L.grid_verify_workspace_bytes(0, 1, 1) == 0 and L.grid_verify_workspace_bytes(1, 64, 1) == 0
    for B, K, V in [(1, 0, 1), (1, 4, 151936), (65535, 63, 151936), (300, 3, 17)]:
        rows, n = B * (K + 1), L.grid_verify_workspace_bytes(B, K, V)
        assert rows * 16 <= n <= 20 * B + 256 + rows * 64 * 16
    size = L.grid_attend_workspace_bytes
    assert size(by(cache(S)), by(chunks(S)), by(attend(S, n_heads=6))) == 0
    assert size(by(cache(S)), by(chunks(S)), None) == 0
    # what a long cache may be split into does not grow without bound
    big = size(by(cache(S)), by(chunks(S, n_seqs=1)), by(attend(S, max_kv=1 << 30)))
    assert 0 < big < 1 << 30


def test_python_refusals(S):
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        S._paged(k, k[:, :, :1])
    with pytest.raises(ValueError):
        S._paged(k.transpose(2, 3), k.transpose(2, 3))
    with pytest.raises(TypeError):
        S._paged(k.float(), k.float())
    table, one = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    four = torch.zeros(4, dtype=torch.int32)
    S._chunks(7, table, one, four, k.device)
    for t, n, c in [(table.long(), one, four), (table[0], one, four), (table, four, four), (table, one, one),
                    (table, one.long(), four), (table.T, one, four)]:
        with pytest.raises(ValueError):
            S._chunks(7, t, n, c, k.device)
    with pytest.raises(ValueError):
        S._vectors(torch.zeros(7, 2, 64), torch.bfloat16, 7, 64, k.device, "q")
    with pytest.raises(ValueError):
        S._vectors(torch.zeros(7, 2, 64).transpose(1, 2), torch.float32, 7, 2, k.device, "q")
    with pytest.raises(TypeError):
        S.verify(torch.zeros(1, 2, 8, dtype=torch.float64), four[:1].view(1, 1))
