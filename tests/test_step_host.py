"""What grid_kv_append, grid_attend and grid_verify refuse: every check is made on the host before anything is enqueued,
so it is tested through the C ABI with addresses that are never read."""

import ctypes
import types

import pytest

AT = 1 << 20  # an address of the right alignment


_vp, _i32, _i64, _f32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
_TWO, _THREE = _i64 * 2, _i64 * 3


class _Cache(ctypes.Structure):
    _fields_ = [("k_pages", _vp), ("v_pages", _vp), ("dtype", _i32), ("n_pages", _i32), ("page_size", _i32),
                ("n_kv_heads", _i32), ("head_dim", _i32), ("k_stride", _THREE), ("v_stride", _THREE)]


class _Chunks(ctypes.Structure):
    _fields_ = [("n_seqs", _i32), ("n_tokens", _i32), ("block_table", _vp), ("table_stride", _i64), ("table_cols", _i32),
                ("kv_len", _vp), ("cu_q", _vp)]


class _Append(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("q", _vp), ("q_out", _vp), ("n_heads", _i32), ("k_stride", _TWO),
                ("v_stride", _TWO), ("q_stride", _TWO), ("q_out_stride", _TWO), ("cos", _vp), ("sin", _vp),
                ("n_positions", _i32), ("rot_dim", _i32), ("interleaved", _i32), ("q_norm", _vp), ("k_norm", _vp),
                ("eps", _f32), ("status", _vp)]


class _Attend(ctypes.Structure):
    _fields_ = [("q", _vp), ("out", _vp), ("q_stride", _TWO), ("out_stride", _TWO), ("lse", _vp), ("n_heads", _i32),
                ("max_q", _i32), ("max_kv", _i32), ("window", _i32), ("scale", _f32), ("workspace", _vp),
                ("workspace_bytes", _sz)]


class _Verify(ctypes.Structure):
    _fields_ = [("logits", _vp), ("dtype", _i32), ("B", _i32), ("K", _i32), ("V", _i32), ("logits_stride", _TWO),
                ("mask", _vp), ("mask_stride", _TWO), ("draft", _vp), ("draft_len", _vp), ("draft_probs", _vp),
                ("probs_stride", _TWO), ("uniform", _vp), ("noise", _vp), ("noise_stride", _i64), ("temperature", _vp),
                ("tokens", _vp), ("accepted", _vp), ("logprobs", _vp), ("workspace", _vp), ("workspace_bytes", _sz)]


@pytest.fixture(scope="module")
def S():
    pytest.importorskip("torch")
    import paper_2607_11951_amd as pkg
    if not pkg.grid.LIB_PATH.exists() or not (pkg.grid.PKG / "_step.so").exists():
        from paper_2607_11951_amd import build
        build.build()
    return types.SimpleNamespace(lib=pkg.lib, G=pkg, _Cache=_Cache, _Chunks=_Chunks, _Append=_Append, _Attend=_Attend,
                                 _Verify=_Verify, _TWO=_TWO, _THREE=_THREE)


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
    """wrong types, shapes, layouts and devices, through the package's functions: on tensors in host memory everything
    else is checked before their device is"""
    torch = pytest.importorskip("torch")
    half, zeros = torch.bfloat16, torch.zeros
    pages = zeros(4, 16, 2, 64, dtype=half)
    table, lens, cu = zeros(3, 5, dtype=torch.int32), zeros(3, dtype=torch.int32), zeros(4, dtype=torch.int32)
    k, q = zeros(7, 2, 64, dtype=half), zeros(7, 6, 64, dtype=half)

    def append(**kw):
        a = dict(k=k, v=k, k_pages=pages, v_pages=pages, block_table=table, kv_len=lens, cu_q=cu, q=q)
        S.G.kv_append(**{**a, **kw})

    def attend(**kw):
        a = dict(q=q, k_pages=pages, v_pages=pages, block_table=table, kv_len=lens, cu_q=cu, max_q=7, max_kv=80)
        S.G.attend(**{**a, **kw})

    def refused(call, error, word, **kw):
        with pytest.raises(error, match=word):
            call(**kw)

    for call in (append, attend):
        refused(call, ValueError, "GPU")  # nothing else is wrong
        refused(call, ValueError, "alike", v_pages=pages[:, :, :1])
        refused(call, ValueError, "alike", v_pages=pages.half())
        refused(call, ValueError, "dense", k_pages=pages.transpose(2, 3), v_pages=pages.transpose(2, 3))
        refused(call, TypeError, "bfloat16", k_pages=pages.float(), v_pages=pages.float())
        refused(call, TypeError, "tensor", k_pages=None)
        refused(call, ValueError, "block_table", block_table=table.long())
        refused(call, ValueError, "block_table", block_table=table[0])
        refused(call, ValueError, "block_table", block_table=table.T)
        refused(call, ValueError, "kv_len", kv_len=cu)
        refused(call, ValueError, "kv_len", kv_len=lens.long())
        refused(call, ValueError, "cu_q", cu_q=lens)
    for bad in (k.float(), k[:, :, :32], k[:5], k[0], zeros(7, 64, 2, dtype=half).transpose(1, 2)):
        refused(append, ValueError, "v: ", v=bad)
        refused(attend, ValueError, "q: ", q=bad) if bad.shape[0] == 7 else None
    refused(append, ValueError, "heads", k=q, v=q)
    table_f = zeros(9, 32)
    refused(append, ValueError, "together", cos=table_f)
    refused(append, ValueError, "cos", cos=table_f.double(), sin=table_f)
    refused(append, ValueError, "sin", cos=table_f, sin=table_f[:5])
    refused(append, ValueError, "q_norm", q_norm=zeros(32))
    refused(append, ValueError, "k_norm", k_norm=zeros(64, dtype=half))
    refused(append, ValueError, "status", status=zeros(3))
    refused(append, TypeError, "eps", eps="x")
    refused(attend, ValueError, "lse", lse=zeros(7, 5))
    refused(attend, TypeError, "max_q", max_q=1.5)
    refused(attend, TypeError, "max_kv", max_kv=None)
    refused(attend, TypeError, "scale", scale="x")

    draft, logits = zeros(2, 3, dtype=torch.int32), zeros(2, 4, 40)

    def verify(**kw):
        S.G.verify(**{**dict(logits=logits, draft=draft), **kw})

    refused(verify, ValueError, "GPU")
    refused(verify, TypeError, "float32", logits=logits.double())
    refused(verify, ValueError, "logits", logits=logits[0])
    refused(verify, ValueError, "logits", logits=zeros(2, 40, 4).transpose(1, 2))
    refused(verify, ValueError, "draft", draft=draft.long())
    refused(verify, ValueError, "draft", draft=draft[:, :2])
    refused(verify, ValueError, "draft_len", draft_len=zeros(3, dtype=torch.int32))
    refused(verify, ValueError, "mask", mask=zeros(2, 4, 1, dtype=torch.int32))
    refused(verify, ValueError, "mask", mask=zeros(2, 3, 2, dtype=torch.int32))
    refused(verify, ValueError, "draft_probs", draft_probs=zeros(2, 4, 40))
    refused(verify, ValueError, "uniform", uniform=zeros(2, 4))
    refused(verify, ValueError, "noise", noise=zeros(2, 39))
    refused(verify, ValueError, "temperature", temperature=zeros(1))
    refused(verify, ValueError, "tokens", tokens=zeros(2, 4))
    refused(verify, ValueError, "accepted", accepted=zeros(3, dtype=torch.int32))
    refused(verify, ValueError, "logprobs", logprobs=zeros(2, 3))
