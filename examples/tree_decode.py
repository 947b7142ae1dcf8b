"""Sampling several continuations of SQL prompts under a grammar, with trees of drafted tokens and shared pages.

    python examples/tree_decode.py [--rows 4] [--samples 2] [--tokens 40] [--branches 3] [--depth 4] [--temperature 0.8]
                                   [--top-k 50] [--top-p 0.95]

A prompt goes through the model once; its continuations share its pages (kv_fork), each with a copy of the last one that it
writes into (kv_copy).  A step of them all:
 1. drafts: what followed the last token earlier in the sequence, up to `branches` continuations, as a tree; Grid.accept and
    Grid.mask give the configuration and the mask after every node, and nodes that the grammar refuses are dropped;
 2. kv_fork: room for the chunk of pending tokens and tree, and the pages of ended rows back;
 3. the model, once, over all nodes: per layer kv_append at their depths and attend_tree;
 4. sample: a token at every node, under its mask and the usual filters;
 5. commit_tree: the branch that these tokens follow, moved together in the cache; the token after it is the next.
"""

import argparse
import sys
from pathlib import Path

import numpy as np
import torch

HERE = Path(__file__).resolve().parent
for p in (HERE, HERE.parent):
    if str(p) not in sys.path:
        sys.path.insert(0, str(p))

import paper_2607_11951_amd as G  # noqa: E402
from draft_decode import CAP, Model, tokenize  # noqa: E402
from workloads import make_workload  # noqa: E402

PAGE = 16
NODES = 1024  # of a tree, at most; longer prompts go through the model in such pieces
OFFSET = G.CONFIG_DTYPE.fields["stk_off"][1] // 4  # of a configuration's words: where its stack begins


class TreeModel(Model):
    """The model of draft_decode.py over chunks that are trees; keys and values of all layers in one tensor each."""

    def pages(self, n):
        shape = (len(self.layers), n, PAGE, self.kv_heads, self.head_dim)
        return [torch.zeros(shape, dtype=torch.float16, device=self.cos.device) for _ in range(2)]

    def forward(self, tokens, pages, table, kv_len, cu_q, masks, depth, max_q, max_kv):
        x = self.embed[tokens]
        h, kh = self.heads, self.kv_heads
        for w, k_pages, v_pages in zip(self.layers, *pages):
            qkv = (self._normed(x) @ w["qkv"]).half().view(len(tokens), h + 2 * kh, self.head_dim)
            q, _ = G.kv_append(qkv[:, h:h + kh], qkv[:, h + kh:], k_pages, v_pages, table, kv_len, cu_q, q=qkv[:, :h],
                               cos=self.cos, sin=self.sin, q_norm=w["q_norm"], k_norm=w["k_norm"], depth=depth)
            o, _ = G.attend_tree(q, k_pages, v_pages, table, kv_len, cu_q, masks, max_q, max_kv)
            x = x + o.float().flatten(1) @ w["out"]
            x = x + torch.relu(self._normed(x) @ w["up"]) @ w["down"]
        return self._normed(x)


class Cache:
    """The pages of all rows: who holds which, and what they hold."""

    def __init__(self, model, pages, cols, device):
        self.k, self.v = model.pages(pages)
        self.table = torch.full((1, cols), -1, dtype=torch.int32, device=device)
        self.held = torch.zeros(1, dtype=torch.int32, device=device)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)

    def go_on(self, parent, keep, room):
        """The next step's rows: from which row they go on, with how many of its tokens, and room for how many."""
        parent, keep, room = (torch.tensor(x, dtype=torch.int32, device=self.refs.device) for x in (parent, keep, room))
        self.table, self.held, self.refs, copies, status = G.kv_fork(self.table, self.held, parent, keep, room, self.refs, PAGE,
                                                                     refs_out=self.refs)
        G.kv_copy(self.k, self.v, copies[0], copies[1], rows=copies[2])
        return status


def draft_tree(history, branches, depth):
    """(token, parent) of the nodes below the last token: what followed its last `branches` earlier places, merged."""
    nodes, child, found = [], {}, 0
    for i in range(len(history) - 2, -1, -1):
        if found == branches:
            break
        if history[i] != history[-1]:
            continue
        found += 1
        at = -1
        for t in history[i + 1:i + 1 + depth]:
            if (at, t) not in child:
                child[at, t] = len(nodes)
                nodes.append((t, at))
            at = child[at, t]
    return nodes


class Grammar:
    """Configurations of any number of rows, advanced together."""

    def __init__(self, grid):
        self.grid = grid

    def rows(self, state, index):
        """rows `index` of a state, in an order of their own"""
        cfg, stack = state
        index = torch.as_tensor(index, device=cfg.device)
        cfg = cfg.view(-1, 32)[index].contiguous()
        cfg.view(torch.int32)[:, OFFSET] = torch.arange(len(index), dtype=torch.int32, device=cfg.device) * CAP
        return cfg.reshape(-1), stack.view(-1, CAP)[index].reshape(-1).contiguous()

    def accept(self, state, tokens):
        tokens = torch.as_tensor(tokens, dtype=torch.int32, device=state[0].device)
        cfg, stack, status = self.grid.accept(*state, tokens, len(tokens), CAP)
        return (cfg, stack), status

    @staticmethod
    def joined(states):
        cfgs = torch.cat([c.view(-1, 32) for c, _ in states])
        cfgs.view(torch.int32)[:, OFFSET] = torch.arange(len(cfgs), dtype=torch.int32, device=cfgs.device) * CAP
        return cfgs.reshape(-1), torch.cat([s for _, s in states])


def decode(model, wl, rows=4, samples=2, new_tokens=40, branches=3, depth=4, temperature=0.0, top_k=0, top_p=1.0, min_p=0.0,
           seed=0, device="cuda"):
    """Decodes `samples` continuations of `rows` prompts until each has new_tokens tokens more or its sentence ends.  Returns
    a dict: prompts and histories (of row b * samples + i), steps, and how many nodes were drafted and accepted."""
    grid, slots = G.from_workload(wl)
    grid.to_device(device)
    grammar = Grammar(grid)
    ids = {s: i for i, s in reversed(list(enumerate(wl.vocab))) if s}
    longest = max(map(len, ids))
    texts = [w or b"S" for w in wl.prefixes[:rows]]
    prompts = [tokenize(ids, longest, w) for w in texts]
    R, B, V = len(prompts), len(prompts) * samples, wl.V
    of = [b // samples for b in range(B)]
    cfgs, _ = grid.configs(texts, [slots[s] for s in wl.slots[:R]])
    pool = np.zeros((R, CAP), np.uint16)
    for b, w in enumerate(texts):
        st = grid.config(w, slots[wl.slots[b]])[1]
        pool[b, :len(st)], cfgs["stk_off"][b] = st, b * CAP
    state = grammar.rows(grid.configs_to_device(cfgs, pool.reshape(-1), device), of)
    room = max(map(len, prompts)) + new_tokens + 2 * branches * depth + 2
    cols = -(-room // PAGE)
    cache = Cache(model, R * cols + B * cols, cols, device)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=device)

    def run(chunks, parents, cached):
        """hidden states of the chunks' nodes, whose keys and values are appended; also cu_q and kv_len"""
        n = [len(c) for c in chunks]
        cu, kv, max_q = ints(np.concatenate([[0], np.cumsum(n)]).tolist()), ints([c + m for c, m in zip(cached, n)]), max(n)
        masks, deep = G.tree_masks(ints(sum(parents, [])), cu, max_q)
        tokens = torch.tensor(sum(chunks, []), device=device)
        max_kv = max(c + m for c, m in zip(cached, n))
        return model.forward(tokens, (cache.k, cache.v), cache.table, kv, cu, masks, deep, max_q, max_kv), cu, kv

    # the prompts, but for their last tokens, once; then the continuations from them
    head = [p[:-1] or p for p in prompts]
    cache.go_on([-1] * R, [0] * R, [len(p) for p in head])
    for at in range(0, max(map(len, head)), NODES):
        piece = [p[at:at + NODES] for p in head]
        run(piece, [list(range(-1, len(p) - 1)) for p in piece], [min(at, len(p)) for p in head])
    start = [len(p) - 1 for p in prompts]
    cache.go_on(of, [start[r] for r in of], [start[r] for r in of])
    gen = torch.Generator(device=device).manual_seed(seed)
    history = [list(prompts[r]) for r in of]
    pending = [[prompts[r][-1]] for r in of]  # tokens the cache does not hold yet
    cached, done = [start[r] for r in of], [False] * B
    count = {"steps": 0, "drafted": 0, "accepted": 0}
    while not all(done):
        # trees, as far as the grammar goes, level by level; the states of the roots and of the nodes that are left
        trees = [[] if done[b] else draft_tree(history[b], branches, depth) for b in range(B)]
        states, row = [state], {(b, -1): b for b in range(B)}
        made = {(b, i): p for b in range(B) for i, (_, p) in enumerate(trees[b])}
        level = [k for k, p in made.items() if p == -1]
        while level:
            nodes, ok = grammar.accept(grammar.rows(grammar.joined(states), [row[b, trees[b][i][1]] for b, i in level]),
                                       [trees[b][i][0] for b, i in level])
            at = sum(len(c) for c, _ in states) // 32
            row.update({k: at + j for j, (k, s) in enumerate(zip(level, ok.tolist())) if s == G.ROW_OK})
            states.append(nodes)
            here = set(level)
            level = [k for k, p in made.items() if (k[0], p) in here and (k[0], p) in row]
        every = grammar.joined(states)
        left = [[i for i in range(len(trees[b])) if (b, i) in row] for b in range(B)]
        # the chunk of a row: pending tokens, a node below the other, and the tree below the last of them
        chunk, parent, start = [], [], []
        for b in range(B):
            n = len(pending[b])
            place = {-1: n - 1, **{i: n + j for j, i in enumerate(left[b])}}
            chunk.append([] if done[b] else pending[b] + [trees[b][i][0] for i in left[b]])
            parent.append([] if done[b] else list(range(-1, n - 1)) + [place[trees[b][i][1]] for i in left[b]])
            start.append(n - 1)
        status = cache.go_on([-1 if d else b for b, d in enumerate(done)], cached, [c + len(x) for c, x in zip(cached, chunk)])
        assert not bool(status.any())
        hidden, cu, kv = run(chunk, parent, cached)
        # a token at the last pending one and at every node
        first = cu.tolist()
        at = [first[b] + start[b] + j for b in range(B) if not done[b] for j in range(1 + len(left[b]))]
        of_row = [row[b, i] for b in range(B) if not done[b] for i in [-1] + left[b]]
        mask = grid.mask(*grammar.rows(every, of_row), len(of_row))[0]
        filters = {}
        if temperature > 0:
            def full(x, dtype):
                return torch.full((len(at),), x, dtype=dtype, device=device)

            noise = torch.empty((len(at), V), device=device).exponential_(generator=gen).clamp_min_(1e-20)
            filters = {"noise": noise, "temperature": full(temperature, torch.float32), "top_k": full(top_k, torch.int32),
                       "top_p": full(top_p, torch.float32), "min_p": full(min_p, torch.float32)}
        drawn, _ = G.sample(model.logits(hidden[torch.tensor(at, device=device)]), mask=mask, **filters)
        sampled = torch.full((len(hidden),), -1, dtype=torch.int32, device=device)
        sampled[torch.tensor(at, device=device)] = drawn
        path, length, following = G.commit_tree(cache.k, cache.v, cache.table, kv, cu, ints(sum(chunk, [])),
                                                ints(sum(parent, [])), sampled, max(map(len, chunk)), start=ints(start))
        path, length, following = path.tolist(), length.tolist(), following.tolist()
        # each row goes on from the configuration after its branch and the next token
        last = [row[b, -1] if done[b] or path[b][length[b] - 1] == start[b] else
                row[b, left[b][path[b][length[b] - 1] - start[b] - 1]] for b in range(B)]
        state, ok = grammar.accept(grammar.rows(every, last), [max(t, 0) for t in following])
        ok = ok.tolist()
        for b in range(B):
            if done[b]:
                continue
            branch = [chunk[b][i] for i in path[b][start[b] + 1:length[b]]]
            assert following[b] >= 0 and ok[b] in (G.ROW_OK, G.ROW_FINISHED), (b, following[b], ok[b])
            history[b] += branch + [following[b]]
            cached[b] += length[b]
            pending[b] = [following[b]]
            count["drafted"] += len(left[b])
            count["accepted"] += len(branch)
            done[b] = ok[b] == G.ROW_FINISHED or len(history[b]) - len(prompts[of[b]]) >= new_tokens
        count["steps"] += 1
    return {"prompts": [prompts[r] for r in of], "histories": history, **count}


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, kind, value in (("rows", int, 4), ("samples", int, 2), ("tokens", int, 40), ("branches", int, 3),
                              ("depth", int, 4), ("temperature", float, 0.8), ("top-k", int, 50), ("top-p", float, 0.95)):
        ap.add_argument(f"--{name}", type=kind, default=value)
    a = ap.parse_args()
    wl = make_workload(2, rows=a.rows)
    got = decode(TreeModel(wl.V), wl, a.rows, a.samples, a.tokens, a.branches, a.depth, a.temperature, a.top_k, a.top_p)
    for p, h in zip(got["prompts"], got["histories"]):
        text = [b"".join(wl.vocab[t] for t in x).decode("utf-8", "replace") for x in (p, h[len(p):])]
        print(f"{text[0]!r} -> {text[1]!r}")
    made = sum(len(h) - len(p) for p, h in zip(got["prompts"], got["histories"]))
    print(f"{made} tokens in {got['steps']} steps of the model: {got['accepted']} of {got['drafted']} drafted nodes accepted")


if __name__ == "__main__":
    main()
