"""What the calls of trees, pages and sampling refuse: every check is made on the host before anything is enqueued, so it is
tested through the C ABI with addresses that are never read, and through the package's functions on tensors in host memory."""

import ctypes

import pytest

from test_step_host import (AT, BAD_CACHE, BAD_CHUNKS, S, _Cache, _i32, _i64, _sz, _vp, append, attend, cache,  # noqa: F401
                            chunks, refused, value)


class _TreeArgs(ctypes.Structure):
    _fields_ = [("n_seqs", _i32), ("n_tokens", _i32), ("cu_q", _vp), ("parent", _vp), ("max_q", _i32), ("stride_words", _i64),
                ("masks", _vp), ("depth", _vp)]


class _Tree(ctypes.Structure):
    _fields_ = [("masks", _vp), ("stride_words", _i64), ("depth", _vp)]


class _Commit(ctypes.Structure):
    _fields_ = [("tokens", _vp), ("parent", _vp), ("sampled", _vp), ("start", _vp), ("max_q", _i32), ("n_layers", _i32),
                ("k_layer_stride", _i64), ("v_layer_stride", _i64), ("path", _vp), ("path_stride", _i64), ("length", _vp),
                ("next", _vp)]


class _Copy(ctypes.Structure):
    _fields_ = [("src", _vp), ("dst", _vp), ("rows", _vp), ("n", _i32), ("n_layers", _i32), ("k_layer_stride", _i64),
                ("v_layer_stride", _i64)]


class _Fork(ctypes.Structure):
    _fields_ = [("table", _vp), ("table_stride", _i64), ("held", _vp), ("n_in", _i32), ("n_rows", _i32), ("table_cols", _i32),
                ("n_pages", _i32), ("page_size", _i32), ("parent", _vp), ("keep", _vp), ("room", _vp), ("refs", _vp),
                ("table_out", _vp), ("table_out_stride", _i64), ("held_out", _vp), ("refs_out", _vp), ("copies", _vp),
                ("status", _vp), ("workspace", _vp), ("workspace_bytes", _sz)]


class _Sample(ctypes.Structure):
    _fields_ = [("logits", _vp), ("dtype", _i32), ("B", _i32), ("V", _i32), ("logits_stride", _i64), ("mask", _vp),
                ("mask_stride", _i64), ("temperature", _vp), ("top_k", _vp), ("top_p", _vp), ("min_p", _vp), ("noise", _vp),
                ("noise_stride", _i64), ("tokens", _vp), ("logprobs", _vp), ("workspace", _vp), ("workspace_bytes", _sz)]


GOOD = {
    "tree_masks": lambda: _TreeArgs(3, 7, AT, AT, 7, 1, AT, AT),
    "tree": lambda: _Tree(AT, 1, AT),
    "commit": lambda: _Commit(AT, AT, AT, None, 7, 2, 1 << 20, 1 << 20, AT, 7, AT, AT),
    "copy": lambda: _Copy(AT, AT, None, 3, 2, 1 << 20, 1 << 20),
    "fork": lambda: _Fork(AT, 5, AT, 3, 4, 5, 100, 16, AT, AT, AT, AT, 2 * AT, 5, 2 * AT, 2 * AT, AT, AT, AT, 1 << 20),
    "sample": lambda: _Sample(AT, 1, 2, 1000, 1000, AT, 32, None, AT, AT, AT, AT, 1000, AT, AT, AT, 1 << 30),
}


def made(kind, **kw):
    a = GOOD[kind]()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def by(x):
    return ctypes.byref(x) if x is not None else None


@pytest.mark.parametrize("name,bad", [("n_seqs", 0), ("n_seqs", 65536), ("n_tokens", -1), ("n_tokens", (1 << 24) + 1),
                                      ("max_q", 0), ("max_q", 1025), ("stride_words", 0), ("cu_q", None), ("parent", None),
                                      ("masks", None), ("depth", None)])
def test_bad_tree_masks(S, name, bad):  # noqa: F811
    refused(S, S.lib().grid_tree_masks(by(made("tree_masks", **{name: bad})), None), "grid_tree_masks")


@pytest.mark.parametrize("name,bad", [("masks", None), ("masks", AT + 2), ("stride_words", 0), ("stride_words", 1 << 31)])
def test_bad_trees(S, name, bad):  # noqa: F811
    rc = S.lib().grid_attend_tree(by(cache(S)), by(chunks(S)), by(attend(S)), by(made("tree", **{name: bad})), None)
    refused(S, rc, "grid_attend_tree")


@pytest.mark.parametrize("name,bad", [("tokens", None), ("parent", None), ("sampled", None), ("max_q", 0), ("max_q", 1025),
                                      ("n_layers", -1), ("n_layers", 1025), ("k_layer_stride", 4), ("v_layer_stride", -8),
                                      ("k_layer_stride", 0), ("v_layer_stride", 1 << 48), ("path", None), ("path_stride", 6),
                                      ("length", None), ("next", None)])
def test_bad_commit(S, name, bad):  # noqa: F811
    rc = S.lib().grid_commit_tree(by(cache(S)), by(chunks(S)), by(made("commit", **{name: bad})), None)
    refused(S, rc, "grid_commit_tree")


@pytest.mark.parametrize("name,bad", [("src", None), ("dst", None), ("n", -1), ("n", (1 << 20) + 1), ("n_layers", 0),
                                      ("n_layers", 1025), ("k_layer_stride", 12), ("v_layer_stride", 0)])
def test_bad_copy(S, name, bad):  # noqa: F811
    refused(S, S.lib().grid_kv_copy(by(cache(S)), by(made("copy", **{name: bad})), None), "grid_kv_copy")


@pytest.mark.parametrize("name,bad", [("table", None), ("held", None), ("parent", None), ("keep", None), ("room", None),
                                      ("refs", None), ("table_out", None), ("held_out", None), ("refs_out", None),
                                      ("copies", None), ("status", None), ("workspace", None), ("workspace", AT + 8),
                                      ("workspace_bytes", 100), ("n_in", 0), ("n_in", 65536), ("n_rows", 0),
                                      ("n_rows", 65536), ("table_cols", 0), ("table_cols", 1 << 28), ("n_pages", 0),
                                      ("n_pages", (1 << 26) + 1), ("page_size", 0), ("page_size", 65537),
                                      ("table_stride", 4), ("table_out_stride", 4), ("table_out", AT), ("held_out", AT)])
def test_bad_fork(S, name, bad):  # noqa: F811
    refused(S, S.lib().grid_kv_fork(by(made("fork", **{name: bad})), None), "grid_kv_fork")


@pytest.mark.parametrize("name,bad", [("logits", None), ("dtype", 3), ("dtype", -1), ("B", 0), ("B", (1 << 20) + 1), ("V", 0),
                                      ("V", (1 << 30) - 2047), ("logits_stride", -1), ("mask_stride", -1),
                                      ("noise_stride", -8), ("tokens", None), ("logprobs", None), ("workspace", None),
                                      ("workspace", AT + 8), ("workspace_bytes", 4096)])
def test_bad_sample(S, name, bad):  # noqa: F811
    refused(S, S.lib().grid_sample(by(made("sample", **{name: bad})), None), "grid_sample")


@pytest.mark.parametrize("name,bad", BAD_CACHE)
def test_bad_cache(S, name, bad):  # noqa: F811
    c, x, L = cache(S, **{name: value(S, bad)}), chunks(S), S.lib()
    refused(S, L.grid_kv_append_tree(by(c), by(x), by(append(S)), AT, None), "grid_kv_append_tree")
    refused(S, L.grid_attend_tree(by(c), by(x), by(attend(S)), by(made("tree")), None), "grid_attend_tree")
    refused(S, L.grid_commit_tree(by(c), by(x), by(made("commit")), None), "grid_commit_tree")
    refused(S, L.grid_kv_copy(by(c), by(made("copy")), None), "grid_kv_copy")


@pytest.mark.parametrize("name,bad", BAD_CHUNKS)
def test_bad_chunks(S, name, bad):  # noqa: F811
    c, x, L = cache(S), chunks(S, **{name: bad}), S.lib()
    refused(S, L.grid_kv_append_tree(by(c), by(x), by(append(S)), AT, None), "grid_kv_append_tree")
    refused(S, L.grid_attend_tree(by(c), by(x), by(attend(S)), by(made("tree")), None), "grid_attend_tree")
    refused(S, L.grid_commit_tree(by(c), by(x), by(made("commit")), None), "grid_commit_tree")
    if name in ("n_seqs", "n_tokens", "cu_q"):
        rc = L.grid_commit_tree(None, by(x), by(made("commit", n_layers=0)), None)
        assert rc == -1 and "grid_commit_tree" in L.grid_last_error().decode()


def test_null_arguments_and_windows(S):  # noqa: F811
    L = S.lib()
    for rc in (L.grid_tree_masks(None, None), L.grid_kv_copy(by(cache(S)), None, None), L.grid_kv_copy(None, by(made("copy")), None),
               L.grid_kv_fork(None, None), L.grid_sample(None, None), L.grid_commit_tree(by(cache(S)), by(chunks(S)), None, None),
               L.grid_commit_tree(None, by(chunks(S)), by(made("commit")), None),
               L.grid_commit_tree(None, None, by(made("commit", n_layers=0)), None),
               L.grid_attend_tree(by(cache(S)), by(chunks(S)), by(attend(S)), None, None),
               L.grid_kv_append_tree(by(cache(S)), by(chunks(S)), by(append(S)), None, None)):
        assert rc == -1
    tree = made("tree", depth=None)
    refused(S, L.grid_attend_tree(by(cache(S)), by(chunks(S)), by(attend(S, window=9)), by(tree), None), "depth")
    # 33 tokens of a chunk need two words
    refused(S, L.grid_attend_tree(by(cache(S)), by(chunks(S, n_tokens=50)), by(attend(S, max_q=33)), by(made("tree")), None), "words")


def test_nothing_to_do(S):  # noqa: F811
    """no tokens, no pairs: nothing is enqueued, nothing is read"""
    L = S.lib()
    assert L.grid_tree_masks(by(made("tree_masks", n_tokens=0, parent=None, masks=None, depth=None)), None) == 0
    assert L.grid_attend_tree(by(cache(S)), by(chunks(S, n_tokens=0)), by(attend(S, workspace=None)), by(made("tree")), None) == 0
    assert L.grid_kv_append_tree(by(cache(S)), by(chunks(S, n_tokens=0)), by(append(S)), AT, None) == 0
    assert L.grid_kv_copy(by(cache(S)), by(made("copy", n=0, src=None, dst=None)), None) == 0


def test_capacities(S):  # noqa: F811
    L = S.lib()
    assert L.grid_commit_tree(by(cache(S, n_kv_heads=1024, head_dim=256)), by(chunks(S, n_seqs=65535)), by(made("commit")), None) == -11
    assert L.grid_kv_copy(by(cache(S, n_kv_heads=1024, head_dim=256, page_size=65536)), by(made("copy")), None) == -11
    size = L.grid_kv_fork_workspace_bytes
    assert size(0, 1) == 0 and size(65536, 1) == 0 and size(1, 0) == 0 and size(1, (1 << 26) + 1) == 0
    assert 0 < size(1, 1) <= 1024 and size(65535, 1 << 26) <= (1 << 26) // 8 + 65535 * 32 + (1 << 17)
    size = L.grid_sample_workspace_bytes
    assert size(0, 9) == 0 and size(1, 0) == 0 and size((1 << 20) + 1, 9) == 0 and size(1, 1 << 30) == 0
    assert 0 < size(1, 1) < 1 << 14 and (1 << 27) < size(1 << 20, 151936) <= 1 << 28 and size(1 << 20, 9) < 1 << 28
    assert L.grid_attend_tree_workspace_bytes(by(cache(S)), by(chunks(S)), None) == 0


def test_python_refusals(S):  # noqa: F811
    torch = pytest.importorskip("torch")
    G, half, zeros, i32 = S.G, torch.bfloat16, torch.zeros, torch.int32
    pages = zeros(4, 16, 2, 64, dtype=half)
    table, lens, cu, seven = zeros(3, 5, dtype=i32), zeros(3, dtype=i32), zeros(4, dtype=i32), zeros(7, dtype=i32)
    k, q = zeros(7, 2, 64, dtype=half), zeros(7, 6, 64, dtype=half)
    good = {
        G.kv_append: dict(k=k, v=k, k_pages=pages, v_pages=pages, block_table=table, kv_len=lens, cu_q=cu, q=q, depth=seven),
        G.attend_tree: dict(q=q, k_pages=pages, v_pages=pages, block_table=table, kv_len=lens, cu_q=cu, max_q=7, max_kv=80,
                            tree=zeros(7, 1, dtype=i32), depth=seven),
        G.tree_masks: dict(parent=seven, cu_q=cu, max_q=7),
        G.commit_tree: dict(k_pages=pages, v_pages=pages, block_table=table, kv_len=lens, cu_q=cu, tokens=seven, parent=seven,
                            sampled=seven, max_q=7),
        G.kv_copy: dict(k_pages=pages, v_pages=pages, src=lens, dst=lens),
        G.kv_fork: dict(block_table=table, held=lens, parent=lens, keep=lens, room=lens, refs=seven, page_size=16),
        G.sample: dict(logits=zeros(3, 40)),
    }

    def refuses(call, error, word, **kw):
        with pytest.raises(error, match=word):
            call(**{**good[call], **kw})

    for call in good:
        refuses(call, ValueError, "GPU")  # nothing else is wrong
    wrong = zeros(3)
    refuses(G.kv_append, ValueError, "depth", depth=lens)
    refuses(G.kv_append, ValueError, "depth", depth=seven.long())
    refuses(G.attend_tree, ValueError, "tree", tree=zeros(6, 1, dtype=i32))
    refuses(G.attend_tree, ValueError, "tree", tree=zeros(7, 1, dtype=torch.int64))
    refuses(G.attend_tree, ValueError, "tree", tree=zeros(7, 0, dtype=i32))
    refuses(G.attend_tree, ValueError, "tree", tree=zeros(9, 7, dtype=i32).T)
    refuses(G.attend_tree, TypeError, "tree", tree=None)
    refuses(G.attend_tree, ValueError, "depth", depth=lens)
    refuses(G.tree_masks, ValueError, "parent", parent=table)
    refuses(G.tree_masks, ValueError, "parent", parent=seven.long())
    refuses(G.tree_masks, ValueError, "cu_q", cu_q=wrong)
    refuses(G.tree_masks, ValueError, "max_q", max_q=0)
    refuses(G.tree_masks, TypeError, "max_q", max_q="x")
    refuses(G.tree_masks, ValueError, "masks", masks=zeros(7, 0, dtype=i32))
    refuses(G.tree_masks, ValueError, "depth", depth=lens)
    refuses(G.commit_tree, ValueError, "together", v_pages=None)
    refuses(G.commit_tree, ValueError, "alike", v_pages=pages[:, :8])
    refuses(G.commit_tree, ValueError, "alike", k_pages=zeros(2, 4, 16, 2, 64, dtype=half))
    refuses(G.commit_tree, TypeError, "block_table", block_table=None)
    for name in ("parent", "sampled", "cu_q", "kv_len"):
        refuses(G.commit_tree, ValueError, name, **{name: wrong})
    refuses(G.commit_tree, ValueError, "start", start=seven)
    refuses(G.commit_tree, ValueError, "path", path=zeros(3, 6, dtype=i32))
    refuses(G.commit_tree, ValueError, "length", length=wrong)
    refuses(G.commit_tree, ValueError, "next", next=seven)
    refuses(G.commit_tree, ValueError, "max_q", max_q=0)
    refuses(G.kv_copy, ValueError, "dst", dst=cu)
    refuses(G.kv_copy, ValueError, "src", src=table)
    refuses(G.kv_copy, ValueError, "rows", rows=wrong)
    refuses(G.kv_copy, TypeError, "bfloat16", k_pages=pages.float(), v_pages=pages.float())
    for name in ("held", "keep", "room"):
        refuses(G.kv_fork, ValueError, name, **{name: cu})
    refuses(G.kv_fork, ValueError, "block_table", block_table=table.long())
    refuses(G.kv_fork, ValueError, "refs", refs=wrong)
    refuses(G.kv_fork, ValueError, "table_out", table_out=zeros(3, 4, dtype=i32))
    refuses(G.kv_fork, ValueError, "copies", copies=zeros(2, 3, dtype=i32))
    refuses(G.kv_fork, ValueError, "status", status=cu)
    refuses(G.sample, TypeError, "float32", logits=zeros(3, 40).double())
    refuses(G.sample, ValueError, "logits", logits=zeros(40, 3).T)
    refuses(G.sample, ValueError, "mask", mask=zeros(3, 1, dtype=i32))
    for name in ("temperature", "top_p", "min_p"):
        refuses(G.sample, ValueError, name, **{name: zeros(2)})
    refuses(G.sample, ValueError, "top_k", top_k=wrong)
    refuses(G.sample, ValueError, "noise", noise=zeros(3, 39))
    refuses(G.sample, ValueError, "tokens", tokens=wrong)
    refuses(G.sample, ValueError, "logprobs", logprobs=zeros(2))


def test_tensors_that_require_a_gradient(S):  # noqa: F811
    torch = pytest.importorskip("torch")
    half, zeros, i32 = torch.bfloat16, torch.zeros, torch.int32
    pages = zeros(4, 16, 2, 64, dtype=half)
    table, lens, cu, seven = zeros(3, 5, dtype=i32), zeros(3, dtype=i32), zeros(4, dtype=i32), zeros(7, dtype=i32)
    calls = [(S.G.sample, dict(logits=zeros(3, 40), temperature=zeros(3), top_p=zeros(3), min_p=zeros(3), noise=zeros(3, 40),
                               logprobs=zeros(3)), ["logits", "temperature", "top_p", "min_p", "noise", "logprobs"]),
             (S.G.attend_tree, dict(q=zeros(7, 6, 64, dtype=half), k_pages=pages, v_pages=pages.clone(), block_table=table,
                                    kv_len=lens, cu_q=cu, tree=zeros(7, 1, dtype=i32), max_q=7, max_kv=80,
                                    out=zeros(7, 6, 64, dtype=half), lse=zeros(7, 6)), ["q", "k_pages", "v_pages", "out", "lse"]),
             (S.G.commit_tree, dict(k_pages=pages, v_pages=pages.clone(), block_table=table, kv_len=lens, cu_q=cu, tokens=seven,
                                    parent=seven, sampled=seven, max_q=7), ["k_pages", "v_pages"]),
             (S.G.kv_copy, dict(k_pages=pages, v_pages=pages.clone(), src=lens, dst=lens), ["k_pages", "v_pages"])]
    for call, args, names in calls:
        for name in names:
            kw = {**args, name: args[name].clone().requires_grad_()}
            with pytest.raises(RuntimeError, match="gradient"):
                call(**kw)
            with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
                call(**kw)
