"""Decoding SQL under a grammar with forced spans and drafted tokens, a small model of random weights in the loop.

    python examples/draft_decode.py [--rows 8] [--tokens 48] [--drafts 4] [--temperature 0.8]

A step of a sequence:
 1. Grid.forced_span: the tokens the grammar leaves no choice about (jump-forward), and the mask after them;
 2. drafts: what followed the same two tokens earlier in the sequence, as far as the grammar allows it; Grid.accept and
    Grid.mask give the configuration and the mask after every draft;
 3. the model, once, over the chunk of all these tokens: per layer kv_append (rotation on the way into the paged cache)
    and attend;
 4. verify: how many drafts are accepted, and the next token, under the masks.

What the cache holds of refused drafts is overwritten by the next chunk: kv_len counts the accepted tokens only.
"""

import argparse
import sys
from pathlib import Path

import numpy as np
import torch

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

import paper_2607_11951_amd as G  # noqa: E402
from workloads import make_workload  # noqa: E402

CAP = 1024  # stack entries of a row
PAGE = 16
SPAN = 8    # forced tokens a step, at most


class Model:
    """A decoder of random weights: grouped heads, head norms, rotary positions, float16 cache."""

    def __init__(self, V, layers=2, width=256, heads=8, kv_heads=2, head_dim=64, positions=4096, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=g) / shape[0] ** 0.5).to(device)

        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.embed, self.unembed = weight(V, width) * V ** 0.5, weight(width, V) * 3
        self.layers = [{"qkv": weight(width, (heads + 2 * kv_heads) * head_dim), "out": weight(heads * head_dim, width),
                        "up": weight(width, 4 * width), "down": weight(4 * width, width),
                        "q_norm": torch.ones(head_dim, device=device), "k_norm": torch.ones(head_dim, device=device)}
                       for _ in range(layers)]
        angle = torch.arange(positions)[:, None] * 10000.0 ** (-torch.arange(head_dim // 2) * 2 / head_dim)
        self.cos, self.sin = angle.cos().to(device), angle.sin().to(device)

    def pages(self, n):
        """The paged cache: keys and values of every layer."""
        shape = (n, PAGE, self.kv_heads, self.head_dim)
        return [tuple(torch.zeros(shape, dtype=torch.float16, device=self.cos.device) for _ in range(2))
                for _ in self.layers]

    @staticmethod
    def _normed(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def forward(self, tokens, pages, table, kv_len, cu_q, max_q, max_kv):
        """Hidden states of the chunks' packed tokens, whose keys and values are appended to the cache."""
        x = self.embed[tokens]
        h, kh = self.heads, self.kv_heads
        for w, (k_pages, v_pages) in zip(self.layers, pages):
            qkv = (self._normed(x) @ w["qkv"]).half().view(len(tokens), h + 2 * kh, self.head_dim)
            q, _ = G.kv_append(qkv[:, h:h + kh], qkv[:, h + kh:], k_pages, v_pages, table, kv_len, cu_q, q=qkv[:, :h],
                               cos=self.cos, sin=self.sin, q_norm=w["q_norm"], k_norm=w["k_norm"])
            o, _ = G.attend(q, k_pages, v_pages, table, kv_len, cu_q, max_q, max_kv)
            x = x + o.float().flatten(1) @ w["out"]
            x = x + torch.relu(self._normed(x) @ w["up"]) @ w["down"]
        return self._normed(x)

    def logits(self, hidden):
        return hidden @ self.unembed


def tokenize(vocab_ids, longest, text):
    """Greedy longest match."""
    out, i = [], 0
    while i < len(text):
        n = next(n for n in range(min(longest, len(text) - i), 0, -1) if text[i:i + n] in vocab_ids)
        out.append(vocab_ids[text[i:i + n]])
        i += n
    return out


def lookup(history, k):
    """Up to k tokens that followed the last earlier place of the final two tokens."""
    for i in range(len(history) - 3, 0, -1):
        if history[i - 1:i + 1] == history[-2:]:
            return history[i + 1:i + 1 + k]
    return []


def decode(model, wl, rows=8, new_tokens=48, drafts=4, temperature=0.0, seed=0, device="cuda"):
    """Decodes `rows` rows of a workload until each has new_tokens tokens more or its sentence ends.  Returns a dict:
    prompts and histories (lists of token ids), steps, and how many tokens were forced, drafted and accepted."""
    grid, slots = G.from_workload(wl)
    grid.to_device(device)
    ids = {s: i for i, s in reversed(list(enumerate(wl.vocab))) if s}
    longest = max(map(len, ids))
    texts = [w or b"S" for w in wl.prefixes[:rows]]
    prompts = [tokenize(ids, longest, w) for w in texts]
    B, K, V = len(prompts), drafts, wl.V
    cfgs, _ = grid.configs(texts, [slots[s] for s in wl.slots[:B]])
    pool = np.zeros((B, CAP), np.uint16)
    for b, w in enumerate(texts):
        st = grid.config(w, slots[wl.slots[b]])[1]
        pool[b, :len(st)], cfgs["stk_off"][b] = st, b * CAP
    cfg, stack = grid.configs_to_device(cfgs, pool.reshape(-1), device)
    room = max(map(len, prompts)) + new_tokens + 2 * SPAN + K + 2
    cols = -(-room // PAGE)
    pages = model.pages(B * cols)
    table = torch.randperm(B * cols, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(B, cols).to(device)
    gen = torch.Generator(device=device).manual_seed(seed)
    history = [list(p) for p in prompts]
    pending = [list(p) for p in prompts]  # tokens the cache does not hold yet
    cached, done = [0] * B, [False] * B
    count = {"steps": 0, "forced": 0, "drafted": 0, "accepted": 0}

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=device)

    while not all(done):
        # forced tokens, and the mask after them
        span, span_len, mask, _, _ = grid.forced_span(cfg, stack, B, CAP, SPAN)
        span, span_len = span.tolist(), span_len.tolist()
        for b in range(B):
            if not done[b]:
                new = span[b][:span_len[b]]
                history[b] += new
                pending[b] += new
                count["forced"] += len(new)
                done[b] = (bool(new) and new[-1] == wl.eos_id) or len(history[b]) - len(prompts[b]) >= new_tokens
        if all(done):
            break
        # drafts as far as the grammar goes, with the configuration and the mask after each
        draft = [[] if done[b] else lookup(history[b], K) for b in range(B)]
        draft_dev = ints([d + [-1] * (K - len(d)) for d in draft]).view(B, K)
        masks, states, alive, length = [mask], [(cfg, stack)], torch.ones(B, dtype=torch.bool, device=device), ints([0] * B)
        for j in range(K):
            c, s, status = grid.accept(*states[-1], draft_dev[:, j].contiguous(), B, CAP)
            alive = alive & (status == G.ROW_OK)
            length += alive
            states.append((c, s))
            masks.append(grid.mask(c, s, B)[0])
        lens = length.tolist()
        # the model over all of it
        chunk = [[] if done[b] else pending[b] + draft[b][:lens[b]] for b in range(B)]
        n = [len(c) for c in chunk]
        cu = np.concatenate([[0], np.cumsum(n)])
        kv = [cached[b] + n[b] for b in range(B)]
        hidden = model.forward(torch.tensor(sum(chunk, []), device=device), pages, table, ints(kv), ints(cu.tolist()), max(n),
                               max(kv))
        # logits after the last pending token and after each draft (rows past a sequence's drafts are not read)
        at = [[min(int(cu[b]) + max(n[b] - lens[b] - 1, 0) + min(j, lens[b]), len(hidden) - 1) for j in range(K + 1)]
              for b in range(B)]
        logits = model.logits(hidden[torch.tensor(at, device=device)])
        random = {}
        if temperature > 0:
            random = {"uniform": torch.rand((B, K), generator=gen, device=device),
                      "noise": torch.empty((B, V), device=device).exponential_(generator=gen).clamp_min_(1e-20),
                      "temperature": torch.full((B,), temperature, device=device)}
        tokens, accepted, _ = G.verify(logits, draft_dev, draft_len=length, mask=torch.stack(masks, 1), **random)
        # each row goes on from the configuration after its accepted drafts
        row, a = torch.arange(B, device=device), accepted.long()
        cfg = torch.stack([c.view(B, 32) for c, _ in states])[a, row].reshape(-1).contiguous()
        stack = torch.stack([s.view(B, CAP) for _, s in states])[a, row].reshape(-1).contiguous()
        cfg, stack, status = grid.accept(cfg, stack, tokens[row, a].contiguous(), B, CAP)
        tokens, accepted, status = tokens.tolist(), accepted.tolist(), status.tolist()
        for b in range(B):
            if done[b]:
                continue
            new = tokens[b][:accepted[b] + 1]
            assert new[-1] >= 0 and status[b] in (G.ROW_OK, G.ROW_FINISHED), (b, new, status[b])
            history[b] += new
            cached[b] += n[b] - lens[b] + accepted[b]
            pending[b] = [new[-1]]
            count["drafted"] += lens[b]
            count["accepted"] += accepted[b]
            done[b] = status[b] == G.ROW_FINISHED or len(history[b]) - len(prompts[b]) >= new_tokens
        count["steps"] += 1
    return {"prompts": prompts, "histories": history, **count}


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rows", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--temperature", type=float, default=0.8)
    a = ap.parse_args()
    wl = make_workload(2, rows=a.rows)
    got = decode(Model(wl.V), wl, a.rows, a.tokens, a.drafts, a.temperature)
    for p, h in zip(got["prompts"], got["histories"]):
        text = [b"".join(wl.vocab[t] for t in x).decode("utf-8", "replace") for x in (p, h[len(p):])]
        print(f"{text[0]!r} -> {text[1]!r}")
    made = sum(len(h) - len(p) for p, h in zip(got["prompts"], got["histories"]))
    print(f"{made} tokens in {got['steps']} steps of the model: {got['forced']} forced, {got['accepted']} of "
          f"{got['drafted']} drafts accepted")


if __name__ == "__main__":
    main()
