"""The model's side of a decoding step: paged cache, attention over it, verification of drafted tokens.

The work is done by the kernels of libgrid.so; the module _step checks the tensors and passes them on (the calls'
contracts are in include/grid.h).  Arrays of chunks are packed: sequence b's new tokens are rows cu_q[b] .. cu_q[b + 1] of
q, k and v; kv_len[b] counts the sequence's cached tokens with the chunk; position s of sequence b is row s % page_size
of page block_table[b, s // page_size].  Pages are [pages, page_size, heads, head_dim] of any strides with dense vectors.

Calls run on `stream`, or on the current stream; outputs and workspaces that are not given are allocated there.  They have
no gradients: tensors that require one are refused while torch records them.
"""

import torch  # before _step, which links its libraries

from .grid import PKG, _check

if not (PKG / "_step.so").exists():
    raise RuntimeError(f"{PKG / '_step.so'} is missing: build it with __graft_entry__.build()")
from . import _step  # noqa: E402


def _done(result):
    if type(result) is int:
        _check(result)
    return result


def kv_append(k, v, k_pages, v_pages, block_table, kv_len, cu_q, *, q=None, q_out=None, cos=None, sin=None,
              interleaved=False, q_norm=None, k_norm=None, eps=1e-6, status=None, stream=None):
    """grid_kv_append: writes the chunks' keys and values [tokens, heads, head_dim] into the cache, after the optional
    norm of each head (k_norm, q_norm: float32 [head_dim]) and the optional rotation by position (cos, sin: float32
    [positions, rot_dim / 2]; interleaved: pairs side by side).  With q its vectors get the same and go to q_out (may be
    q itself).  Returns (q_out or None, status); status, an int32 tensor [B], is written where it is given."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_append(k, v, k_pages, v_pages, block_table, kv_len, cu_q, q=q, q_out=q_out, cos=cos, sin=sin,
                             interleaved=interleaved, q_norm=q_norm, k_norm=k_norm, eps=eps, status=status)
    return _done(_step.kv_append(k, v, k_pages, v_pages, block_table, kv_len, cu_q, q, q_out, cos, sin, interleaved,
                                 q_norm, k_norm, eps, status))


def attend(q, k_pages, v_pages, block_table, kv_len, cu_q, max_q, max_kv, *, scale=None, window=0, out=None, lse=None,
           workspace=None, stream=None):
    """grid_attend: causal attention of the chunks' queries [tokens, heads, head_dim] over the cache, over the last
    `window` positions only where that is not 0.  max_q and max_kv bound the chunks' lengths and kv_len; scale is
    head_dim ** -0.5 unless given.  Returns (out like q, lse float32 [tokens, heads])."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return attend(q, k_pages, v_pages, block_table, kv_len, cu_q, max_q, max_kv, scale=scale, window=window,
                          out=out, lse=lse, workspace=workspace)
    return _done(_step.attend(q, k_pages, v_pages, block_table, kv_len, cu_q, max_q, max_kv, scale, window, out, lse,
                              workspace))


def verify(logits, draft, *, draft_len=None, mask=None, draft_probs=None, uniform=None, noise=None, temperature=None,
           tokens=None, accepted=None, logprobs=None, workspace=None, stream=None):
    """grid_verify: drafted tokens draft (int32 [B, K]) against the target's logits [B, K + 1, V] under the mask rows
    (int32 [B, K + 1, words], as Grid.mask writes them; None: all tokens allowed).  uniform (float32 [B, K], from
    U[0, 1)) and noise (float32 [B, V], from Exp(1)) are the random numbers; without them the verification is greedy.
    draft_probs (float32 [B, K, V]) is the drafter's distribution; without it each draft is taken as certain.  Returns
    (tokens int32 [B, K + 1]: accepted drafts, the next token, -1; accepted int32 [B]; logprobs float32 [B, K + 1])."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return verify(logits, draft, draft_len=draft_len, mask=mask, draft_probs=draft_probs, uniform=uniform,
                          noise=noise, temperature=temperature, tokens=tokens, accepted=accepted, logprobs=logprobs,
                          workspace=workspace)
    return _done(_step.verify(logits, draft, draft_len, mask, draft_probs, uniform, noise, temperature, tokens, accepted,
                              logprobs, workspace))
