"""The model's side of a decoding step: paged cache, attention over it, verification of drafted tokens.

Argument marshalling only, as in grid.py: the work is done by the kernels of libgrid.so (the calls' contracts are in
include/grid.h).  Arrays of chunks are packed: sequence b's new tokens are rows cu_q[b] .. cu_q[b + 1] of q, k and v;
kv_len[b] counts the sequence's cached tokens with the chunk; position s of sequence b is row s % page_size of page
block_table[b, s // page_size].  Pages are [pages, page_size, heads, head_dim] of any strides with dense vectors.

Outputs and workspaces that are not given are allocated on the stream that the call runs on.
"""

import ctypes

import torch

from .grid import DTYPE_BF16, DTYPE_F16, DTYPE_F32, _check, lib

_vp, _i32, _i64, _f32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
_TWO, _THREE = _i64 * 2, _i64 * 3
_HALVES = {torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}
_FLOATS = {torch.float32: DTYPE_F32, **_HALVES}


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


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on(stream):
    """(the stream's handle, a context in which allocations belong to it)"""
    if stream is None:
        return torch.cuda.current_stream().cuda_stream, None
    return stream.cuda_stream, torch.cuda.stream(stream)


def _empty(ctx, shape, dtype, device):
    if ctx is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with ctx:
        return torch.empty(shape, dtype=dtype, device=device)


def _dense(t, dtype, shape, device, what):
    """Checks an optional dense tensor."""
    if t is not None and (t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous()):
        raise ValueError(f"{what}: a contiguous {dtype} tensor {tuple(shape)} on {device} is wanted")


def _paged(k_pages, v_pages):
    _need(k_pages.dim() == 4 and k_pages.shape == v_pages.shape and k_pages.dtype == v_pages.dtype and
          k_pages.device == v_pages.device, "pages: [pages, page_size, heads, head_dim], keys and values alike")
    if k_pages.dtype not in _HALVES:
        raise TypeError("pages must be bfloat16 or float16")
    ks, vs = k_pages.stride(), v_pages.stride()
    _need(ks[3] == 1 and vs[3] == 1, "pages: vectors must be dense")
    P, rows, H, D = k_pages.shape
    return _Cache(k_pages.data_ptr(), v_pages.data_ptr(), _HALVES[k_pages.dtype], P, rows, H, D, _THREE(*ks[:3]),
                  _THREE(*vs[:3]))


def _chunks(n_tokens, block_table, kv_len, cu_q, device):
    _need(block_table.dim() == 2 and block_table.dtype == torch.int32 and block_table.device == device and
          block_table.stride(1) == 1, "block_table: an int32 tensor [B, pages] with dense rows, on the cache's device")
    B, cols = block_table.shape
    _dense(kv_len, torch.int32, (B,), device, "kv_len")
    _dense(cu_q, torch.int32, (B + 1,), device, "cu_q")
    stride = block_table.stride(0) if B > 1 else cols
    return _Chunks(B, n_tokens, block_table.data_ptr(), stride, cols, kv_len.data_ptr(), cu_q.data_ptr())


def _vectors(t, dtype, n, D, device, what):
    """Checks a packed array of heads' vectors [n, heads, D] with dense vectors; its strides."""
    _need(t.dim() == 3 and t.dtype == dtype and t.shape[0] == n and t.shape[2] == D and t.device == device and
          t.stride(2) == 1, f"{what}: a {dtype} tensor [{n}, heads, {D}] with dense vectors on {device} is wanted")
    return _TWO(*t.stride()[:2])


def kv_append(k, v, k_pages, v_pages, block_table, kv_len, cu_q, *, q=None, q_out=None, cos=None, sin=None,
              interleaved=False, q_norm=None, k_norm=None, eps=1e-6, status=None, stream=None):
    """grid_kv_append: writes the chunks' keys and values [tokens, heads, head_dim] into the cache, after the optional
    norm of each head (k_norm, q_norm: float32 [head_dim]) and the optional rotation by position (cos, sin: float32
    [positions, rot_dim / 2]; interleaved: pairs side by side).  With q its vectors get the same and go to q_out (may be
    q itself).  Returns (q_out or None, status); status, an int32 tensor [B], is written where it is given."""
    cache = _paged(k_pages, v_pages)
    dev, dt, n, D = k_pages.device, k_pages.dtype, k.shape[0], cache.head_dim
    chunks = _chunks(n, block_table, kv_len, cu_q, dev)
    handle, ctx = _on(stream)
    ks, vs = _vectors(k, dt, n, D, dev, "k"), _vectors(v, dt, n, D, dev, "v")
    _need(k.shape[1] == cache.n_kv_heads and v.shape[1] == cache.n_kv_heads, "k and v have the cache's heads")
    qs = os = _TWO()
    heads = 0
    if q is not None:
        qs, heads = _vectors(q, dt, n, D, dev, "q"), q.shape[1]
        if q_out is None:
            q_out = _empty(ctx, q.shape, dt, dev)
        _need(q_out.shape == q.shape, "q_out has the shape of q")
        os = _vectors(q_out, dt, n, D, dev, "q_out")
    positions = half = 0
    if cos is not None:
        positions, half = cos.shape
        _dense(cos, torch.float32, cos.shape, dev, "cos")
        _need(sin is not None, "cos and sin come together")
        _dense(sin, torch.float32, cos.shape, dev, "sin")
    _dense(q_norm, torch.float32, (D,), dev, "q_norm")
    _dense(k_norm, torch.float32, (D,), dev, "k_norm")
    _dense(status, torch.int32, (chunks.n_seqs,), dev, "status")
    args = _Append(k.data_ptr(), v.data_ptr(), _ptr(q), _ptr(q_out), heads, ks, vs, qs, os, _ptr(cos), _ptr(sin),
                   positions, 2 * half, int(interleaved), _ptr(q_norm), _ptr(k_norm), eps, _ptr(status))
    _check(lib().grid_kv_append(ctypes.byref(cache), ctypes.byref(chunks), ctypes.byref(args), handle))
    return q_out, status


def attend(q, k_pages, v_pages, block_table, kv_len, cu_q, max_q, max_kv, *, scale=None, window=0, out=None, lse=None,
           workspace=None, stream=None):
    """grid_attend: causal attention of the chunks' queries [tokens, heads, head_dim] over the cache, over the last
    `window` positions only where that is not 0.  max_q and max_kv bound the chunks' lengths and kv_len; scale is
    head_dim ** -0.5 unless given.  Returns (out like q, lse float32 [tokens, heads])."""
    cache = _paged(k_pages, v_pages)
    dev, n, D = k_pages.device, q.shape[0], cache.head_dim
    chunks = _chunks(n, block_table, kv_len, cu_q, dev)
    handle, ctx = _on(stream)
    qs, heads = _vectors(q, k_pages.dtype, n, D, dev, "q"), q.shape[1]
    if out is None:
        out = _empty(ctx, (n, heads, D), q.dtype, dev)
    _need(out.shape == q.shape, "out has the shape of q")
    os = _vectors(out, q.dtype, n, D, dev, "out")
    if lse is None:
        lse = _empty(ctx, (n, heads), torch.float32, dev)
    else:
        _dense(lse, torch.float32, (n, heads), dev, "lse")
    args = _Attend(q.data_ptr(), out.data_ptr(), qs, os, lse.data_ptr(), heads, max_q, max_kv, window,
                   D ** -0.5 if scale is None else scale)
    if workspace is None:
        workspace = _empty(ctx, lib().grid_attend_workspace_bytes(ctypes.byref(cache), ctypes.byref(chunks),
                                                                  ctypes.byref(args)), torch.uint8, dev)
    args.workspace, args.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(lib().grid_attend(ctypes.byref(cache), ctypes.byref(chunks), ctypes.byref(args), handle))
    return out, lse


def verify(logits, draft, *, draft_len=None, mask=None, draft_probs=None, uniform=None, noise=None, temperature=None,
           tokens=None, accepted=None, logprobs=None, workspace=None, stream=None):
    """grid_verify: drafted tokens draft (int32 [B, K]) against the target's logits [B, K + 1, V] under the mask rows
    (int32 [B, K + 1, words], as Grid.mask writes them; None: all tokens allowed).  uniform (float32 [B, K], from
    U[0, 1)) and noise (float32 [B, V], from Exp(1)) are the random numbers; without them the verification is greedy.
    draft_probs (float32 [B, K, V]) is the drafter's distribution; without it each draft is taken as certain.  Returns
    (tokens int32 [B, K + 1]: accepted drafts, the next token, -1; accepted int32 [B]; logprobs float32 [B, K + 1])."""
    _need(logits.dim() == 3 and logits.stride(2) == 1, "logits: [B, K + 1, V] with dense rows")
    if logits.dtype not in _FLOATS:
        raise TypeError("logits must be float32, bfloat16 or float16")
    B, K, V = logits.shape[0], logits.shape[1] - 1, logits.shape[2]
    dev, words = logits.device, (V + 31) // 32
    handle, ctx = _on(stream)
    _dense(draft, torch.int32, (B, K), dev, "draft")
    _dense(draft_len, torch.int32, (B,), dev, "draft_len")
    _dense(uniform, torch.float32, (B, K), dev, "uniform")
    _dense(temperature, torch.float32, (B,), dev, "temperature")
    ms = ps = _TWO()
    ns = 0
    if mask is not None:
        _need(mask.dim() == 3 and mask.dtype == torch.int32 and mask.device == dev and mask.shape[:2] == (B, K + 1) and
              mask.shape[2] >= words and mask.stride(2) == 1, f"mask: an int32 tensor [{B}, {K + 1}, >= {words}]")
        ms = _TWO(*mask.stride()[:2])
    if draft_probs is not None:
        _need(draft_probs.dtype == torch.float32 and draft_probs.device == dev and draft_probs.shape == (B, K, V) and
              (K == 0 or draft_probs.stride(2) == 1), f"draft_probs: a float32 tensor [{B}, {K}, {V}] with dense rows")
        ps = _TWO(*draft_probs.stride()[:2])
    if noise is not None:
        _need(noise.dtype == torch.float32 and noise.device == dev and noise.shape == (B, V) and noise.stride(1) == 1,
              f"noise: a float32 tensor [{B}, {V}] with dense rows")
        ns = noise.stride(0)
    if tokens is None:
        tokens = _empty(ctx, (B, K + 1), torch.int32, dev)
    if accepted is None:
        accepted = _empty(ctx, (B,), torch.int32, dev)
    if logprobs is None:
        logprobs = _empty(ctx, (B, K + 1), torch.float32, dev)
    _dense(tokens, torch.int32, (B, K + 1), dev, "tokens")
    _dense(accepted, torch.int32, (B,), dev, "accepted")
    _dense(logprobs, torch.float32, (B, K + 1), dev, "logprobs")
    if workspace is None:
        workspace = _empty(ctx, lib().grid_verify_workspace_bytes(B, K, V), torch.uint8, dev)
    args = _Verify(logits.data_ptr(), _FLOATS[logits.dtype], B, K, V, _TWO(*logits.stride()[:2]), _ptr(mask), ms,
                   draft.data_ptr(), _ptr(draft_len), _ptr(draft_probs), ps, _ptr(uniform), _ptr(noise), ns,
                   _ptr(temperature), tokens.data_ptr(), accepted.data_ptr(), logprobs.data_ptr(), workspace.data_ptr(),
                   workspace.numel() * workspace.element_size())
    _check(lib().grid_verify(ctypes.byref(args), handle))
    return tokens, accepted, logprobs
