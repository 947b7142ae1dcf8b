"""The model's side of a decoding step: paged cache, attention over it, sampling, drafts in a row or in a tree.

The work is done by the kernels of libgrid.so; the module _step checks the tensors and passes them on (the calls'
contracts are in include/grid.h).  Arrays of chunks are packed: sequence b's new tokens are rows cu_q[b] .. cu_q[b + 1] of
q, k and v; kv_len[b] counts the sequence's cached tokens with the chunk; position s of sequence b is row s % page_size
of page block_table[b, s // page_size].  Pages are [pages, page_size, heads, head_dim] of any strides with dense vectors;
calls that work on all layers of a cache take [layers, pages, page_size, heads, head_dim] too.

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
              interleaved=False, q_norm=None, k_norm=None, eps=1e-6, status=None, depth=None, stream=None):
    """grid_kv_append: writes the chunks' keys and values [tokens, heads, head_dim] into the cache, after the optional
    norm of each head (k_norm, q_norm: float32 [head_dim]) and the optional rotation by position (cos, sin: float32
    [positions, rot_dim / 2]; interleaved: pairs side by side).  With q its vectors get the same and go to q_out (may be
    q itself).  With depth (int32 [tokens], as tree_masks writes it) the chunks are trees: a token is rotated by the position of
    the chunk's first and its depth.  Returns (q_out or None, status); status, an int32 tensor [B], is written where it is
    given."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_append(k, v, k_pages, v_pages, block_table, kv_len, cu_q, q=q, q_out=q_out, cos=cos, sin=sin,
                             interleaved=interleaved, q_norm=q_norm, k_norm=k_norm, eps=eps, status=status,
                             depth=depth)
    return _done(_step.kv_append(k, v, k_pages, v_pages, block_table, kv_len, cu_q, q, q_out, cos, sin, interleaved,
                                 q_norm, k_norm, eps, status, depth))


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


def sample(logits, *, mask=None, temperature=None, top_k=None, top_p=None, min_p=None, noise=None, tokens=None,
           logprobs=None, workspace=None, stream=None):
    """grid_sample: one token of every row of logits [B, V] under the mask rows (int32 [B, words], as Grid.mask writes them;
    None: all tokens allowed), at the rows' temperature (float32 [B]), of the top_k (int32 [B]) largest, of these the ones
    that hold top_p (float32 [B]) of the mass, of these the ones with at least min_p (float32 [B]) of the largest
    probability.  noise (float32 [B, V], from Exp(1)) are the random numbers, drawn by the caller for all V whatever is kept;
    without them the token is the largest logit's.
    Returns (tokens int32 [B], -1 where there is none; logprobs float32 [B], of the token among those that are kept)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return sample(logits, mask=mask, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, noise=noise,
                          tokens=tokens, logprobs=logprobs, workspace=workspace)
    return _done(_step.sample(logits, mask, temperature, top_k, top_p, min_p, noise, tokens, logprobs, workspace))


def tree_masks(parent, cu_q, max_q, *, window=0, masks=None, depth=None, stream=None):
    """grid_tree_masks: of every node of the chunks' trees (parent int32 [tokens]: the place of a node's parent in its
    chunk, before its own; -1: none) the places of itself and its ancestors as bits, and its depth.  A chunk has max_q places
    at most, max_q is at most 1024.  With a window only the nearest ancestors have bits, `window` places with the node
    itself: attend_tree under a window asks for such masks where trees may be deeper than it.  Returns (masks int32 [tokens, ceil(max_q / 32)], depth int32 [tokens])."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_masks(parent, cu_q, max_q, window=window, masks=masks, depth=depth)
    return _done(_step.tree_masks(parent, cu_q, max_q, masks, depth, window))


def attend_tree(q, k_pages, v_pages, block_table, kv_len, cu_q, tree, max_q, max_kv, *, depth=None, scale=None, window=0,
                out=None, lse=None, workspace=None, stream=None):
    """grid_attend_tree: attend for chunks that are trees.  A token sees what is cached before its chunk, and of its chunk
    the places whose bits are set in its row of tree (int32 [tokens, words], as tree_masks writes them).  With a window
    depth (int32 [tokens]) says where the tokens are; it bounds what is cached before the chunk, the bits the chunk itself
    (tree_masks with the same window).  Returns (out like q, lse float32 [tokens, heads])."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return attend_tree(q, k_pages, v_pages, block_table, kv_len, cu_q, tree, max_q, max_kv, depth=depth,
                               scale=scale, window=window, out=out, lse=lse, workspace=workspace)
    return _done(_step.attend_tree(q, k_pages, v_pages, block_table, kv_len, cu_q, max_q, max_kv, scale, window, out, lse,
                                   workspace, tree, depth))


def commit_tree(k_pages, v_pages, block_table, kv_len, cu_q, tokens, parent, sampled, max_q, *, start=None, path=None,
                length=None, next=None, stream=None):
    """grid_commit_tree: the branch of every chunk's tree that the target's tokens follow, moved together in the cache, in
    all layers of it.  tokens, parent and sampled (int32 [tokens]) are the nodes' drafted tokens, their parents and the
    target's tokens after them; the branch begins at place start[b] (int32 [B]; None: 0) with its ancestors.  k_pages and
    v_pages may be None (then so may block_table and kv_len): nothing is moved.  Returns (path int32 [B, max_q]: the
    branch's places, then -1; length int32 [B]; next int32 [B]: the target's token after the branch)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return commit_tree(k_pages, v_pages, block_table, kv_len, cu_q, tokens, parent, sampled, max_q, start=start,
                               path=path, length=length, next=next)
    return _done(_step.commit_tree(k_pages, v_pages, block_table, kv_len, cu_q, tokens, parent, sampled, max_q, start, path,
                                   length, next))


def kv_copy(k_pages, v_pages, src, dst, *, rows=None, stream=None):
    """grid_kv_copy: the first rows[i] rows (int32 [n]; None: all) of page src[i] to page dst[i] (int32 [n]), keys and
    values, in all layers; pairs with an id that is not a page (-1) are left out."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_copy(k_pages, v_pages, src, dst, rows=rows)
    code = _step.kv_copy(k_pages, v_pages, src, dst, rows)
    if code is not None:
        _check(code)


def kv_fork(block_table, held, parent, keep, room, refs, page_size, *, table_out=None, held_out=None, refs_out=None,
            copies=None, status=None, workspace=None, stream=None):
    """grid_kv_fork: the block table of the next step's rows.  Row b goes on from row parent[b] (-1: from nothing) with its
    first keep[b] tokens and gets room for room[b]; held (int32 [rows]) counts the pages of the old rows, refs (int32
    [pages]) who holds each page.  Returns (table like block_table, held, refs, copies int32 [3, rows], status int32
    [rows]); kv_copy(k_pages, v_pages, copies[0], copies[1], rows=copies[2]) then copies the pages that rows no longer
    share."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_fork(block_table, held, parent, keep, room, refs, page_size, table_out=table_out, held_out=held_out,
                           refs_out=refs_out, copies=copies, status=status, workspace=workspace)
    return _done(_step.kv_fork(block_table, held, parent, keep, room, refs, page_size, table_out, held_out, refs_out, copies,
                               status, workspace))
