"""A step with a tree of drafts under a grammar, and the pages of its cache: sampling, tree attention, commit, fork, copy.

Where a grammar leaves a few continuations open, a program drafts several at once: a tree of tokens, of which a model's
one pass scores every branch.  Each token of the tree attends over the cache and over its own ancestors (`attend_tree`);
at every node a token is drawn from the masked, filtered distribution (`sample`); the branch that these tokens follow is
kept, and what the cache holds of it moves together behind the text (`commit_tree`).  Sequences that go on from the same
text share its pages: `kv_fork` hands pages on, frees and gives out pages, and says which have to be copied; `kv_copy`
copies them, in all layers.

`run` makes these calls where `own` is true; otherwise it computes the same in elementary torch operations.  Layouts:
chunks are packed, sequence b's nodes are rows cu_q[b] .. cu_q[b + 1] (a node comes after its parent); kv_len[b] counts
the cached tokens with the chunk; position s of sequence b is row s % page of page block_table[b, s // page].
"""

import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------------------ cases
def _sample(name, B, V, dtype, masked, filters, shape=0):
    c = {"kind": "sample", "B": B, "V": V, "dtype": dtype, "masked": masked, "filters": filters, "shape": shape}
    return {"name": name, **c} if name else c


def _attend(name, B, q, kv, heads, page, dtype="bf16", window=0, ragged=False, shape=0):
    hq, hkv, d = heads
    c = {"kind": "attend", "B": B, "q": q, "kv": kv, "hq": hq, "hkv": hkv, "d": d, "page": page, "dtype": dtype,
         "window": window, "ragged": ragged, "shape": shape}
    return {"name": name, **c} if name else c


def _commit(name, layers, B, q, kv, heads, page, dtype="bf16", ragged=False, shape=0):
    hkv, d = heads
    c = {"kind": "commit", "layers": layers, "B": B, "q": q, "kv": kv, "hkv": hkv, "d": d, "page": page, "dtype": dtype,
         "ragged": ragged, "shape": shape}
    return {"name": name, **c} if name else c


def _copy(name, layers, pages, n, heads, page, dtype="bf16", partial=False, shape=0):
    hkv, d = heads
    c = {"kind": "copy", "layers": layers, "pages": pages, "n": n, "hkv": hkv, "d": d, "page": page, "dtype": dtype,
         "partial": partial, "shape": shape}
    return {"name": name, **c} if name else c


def _fork(name, B, kv, page, pages, grow, forked, shape=0):
    c = {"kind": "fork", "B": B, "kv": kv, "page": page, "pages": pages, "grow": grow, "forked": forked, "shape": shape}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one user's next token over the full vocabulary, the usual filters: the call is latency
        _sample("sample_b1", 1, 151936, "bf16", True, "k"),
        # the ordinary batch under masks, every user with filters of their own
        _sample("sample_b32_mixed", 32, 151936, "bf16", True, "mixed", 1),
        # a large batch without a grammar on an odd vocabulary, float32 logits, nucleus and smallest probability
        _sample("sample_b256_f32", 256, 50257, "f32", False, "p", 2),
        # one user's tree of sixteen nodes after a page of text: latency
        _attend("attend_b1_tree", 1, 16, 1500, (28, 4, 128), 16),
        # the ordinary batch of trees, users at lengths of their own
        _attend("attend_b32_trees", 32, 64, 8192, (32, 8, 128), 64, ragged=True, shape=3),
        # float16, small heads shared by three, a window, pages that are no power of two, trees of any size
        _attend("attend_trees_window_f16", 7, 61, 1900, (15, 5, 64), 24, "f16", window=300, ragged=True, shape=4),
        # one user's accepted branch moved together in every layer
        _commit("commit_b1", 28, 1, 16, 200, (4, 128), 16),
        # a batch of large trees
        _commit("commit_b64", 32, 64, 64, 300, (8, 128), 64, ragged=True, shape=5),
        # the last pages of a few forked sequences
        _copy("copy_few", 28, 256, 3, (4, 128), 16, partial=True, shape=6),
        # pages moved for defragmentation
        _copy("copy_many", 32, 1100, 500, (8, 128), 16, shape=7),
        # eight beams go on from one text
        _fork("fork_b8_beams", 8, 700, 16, 2048, 8, 1.0),
        # a server's step: most sequences grow, some fork, some end and make room
        _fork("fork_b512", 512, 8192, 16, 200003, 40, 0.15, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(28, 4, 128), (32, 8, 128), (16, 16, 64), (15, 5, 64), (8, 1, 256), (40, 8, 128), (12, 12, 64), (24, 2, 128)]


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """One more case: kinds by how often a program makes them, sizes over the logarithm of their ranges."""
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), _cost(c))
    while True:
        kind = rng.choice(["sample", "sample", "sample", "attend", "attend", "attend", "commit", "copy", "fork"])
        shape, ragged = rng.randrange(1 << 20), rng.random() < 0.7
        heads, page = rng.choice(HEADS), rng.choice([1, 16, 16, 24, 32, 64, 64, 100, 128, 256])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        if kind == "sample":
            c = _sample(None, _log_int(rng, 1, 256), _log_int(rng, 1000, 151936), rng.choice(["bf16", "bf16", "f32", "f16"]),
                        rng.random() < 0.6, rng.choice(["mixed", "mixed", "k", "p", "none"]), shape)
        elif kind == "attend":
            q, B = rng.choice([rng.randint(2, 16), rng.randint(9, 64), _log_int(rng, 16, 200)]), _log_int(rng, 1, 64)
            kv = q + _log_int(rng, 1, 65536)
            c = _attend(None, B, q, kv, heads, page, dtype, rng.choice([0, 0, 0, _log_int(rng, 16, 4096)]), ragged, shape)
            # what the plain form holds at once has to fit
            if B * kv * heads[1] * heads[2] > 1 << 29 or B * heads[0] * q * kv > 1 << 30:
                continue
        elif kind == "commit":
            q = rng.randint(1, 64)
            c = _commit(None, _log_int(rng, 1, 48), _log_int(rng, 1, 96), q, q + _log_int(rng, 1, 1000), heads[1:], page, dtype,
                        ragged, shape)
            if c["layers"] * c["B"] * (c["kv"] + page) * heads[1] * heads[2] > 1 << 30:
                continue
        elif kind == "copy":
            n = _log_int(rng, 1, 1000)
            c = _copy(None, _log_int(rng, 1, 48), 2 * n + rng.randint(0, 2 * n), n, heads[1:], page, dtype, rng.random() < 0.5,
                      shape)
            if c["layers"] * c["pages"] * page * heads[1] * heads[2] > 1 << 30:
                continue
        else:
            B, kv, grow = _log_int(rng, 1, 700), _log_int(rng, 1, 16384), rng.choice([1, 5, 8, 64, 700])
            need = B * (2 * -(-kv // page) + -(-grow // page) + 2)
            if need > 1 << 21:
                continue
            c = _fork(None, B, kv, page, need + _log_int(rng, 1, 1 << 17), grow, rng.choice([0.0, 0.1, 0.5, 1.0]), shape)
        if _cost(c) <= most[kind]:
            return c


def _lens(c):
    """(new tokens, cached tokens with them) of every sequence: fixed by the case."""
    if not c["ragged"]:
        return [(c["q"], c["kv"])] * c["B"]
    r = random.Random(c["shape"])
    got = [(c["q"], c["kv"])]
    for _ in range(c["B"] - 1):
        n = 0 if r.random() < 0.04 else r.randint(1, c["q"])
        before = 0 if r.random() < 0.04 else r.randint(1, max(1, c["kv"] - n))
        got.append((n, min(c["kv"], n + before)))
    r.shuffle(got)
    return got


def _filters(c):
    """(top_k, top_p, min_p) of every row: fixed by the case; top_k 0, top_p 1 and min_p 0 keep all."""
    r = random.Random(c["shape"])
    kinds = {"none": lambda: (0, 1.0, 0.0), "k": lambda: (50, 0.9, 0.0), "p": lambda: (0, r.choice([0.8, 0.9, 0.95]), 0.001),
             "mixed": lambda: (r.choice([0, 1, 20, 50, 200, 1000]), r.choice([1.0, 0.9, 0.95]), r.choice([0.0, 0.0, 0.05]))}
    return [kinds[c["filters"]]() for _ in range(c["B"])]


def _fork_plan(c):
    """Lengths, parents, kept lengths and room of every row: fixed by the case."""
    r = random.Random(c["shape"])
    B, whole = c["B"], c["forked"] == 1.0
    lens = [c["kv"] if whole else r.randint(1, c["kv"]) for _ in range(B)]
    parent, keep = [], []
    for b in range(B):
        if whole:
            parent.append(r.randrange(B) if c["shape"] else r.randrange(min(B, 3)))
        elif r.random() < c["forked"]:
            parent.append(r.choice([-1, r.randrange(B), r.randrange(B)]))
        else:
            parent.append(b)
        p = parent[b]
        keep.append(0 if p < 0 else lens[p] if r.random() < 0.8 else r.randint(0, lens[p]))
    room = [0 if parent[b] < 0 and r.random() < 0.5 else keep[b] + r.randint(0, c["grow"]) for b in range(B)]
    return lens, parent, keep, room


def work(c):
    if c["kind"] == "sample":
        V, W = c["V"], (c["V"] + 31) // 32
        # every row of logits and masks; noise where any token may be drawn, otherwise of as many as are kept at most
        noise = sum(k if k else 0 if p < 1 or m > 0 else V for k, p, m in _filters(c))
        return {"bytes": c["B"] * (V * SIZE[c["dtype"]] + (4 * W if c["masked"] else 0) + 24) + 4 * noise, "flops": 4 * c["B"] * V}
    if c["kind"] == "copy":
        row = 2 * c["layers"] * c["hkv"] * c["d"] * SIZE[c["dtype"]]
        return {"bytes": 2 * row * sum(_rows(c)) + 12 * c["n"], "flops": 1}
    if c["kind"] == "fork":
        lens, parent, keep, room = _fork_plan(c)
        held = sum(-(-n // c["page"]) for n in lens)
        now = sum(-(-max(k, n) // c["page"]) for k, n in zip(keep, room))
        return {"bytes": 4 * (held + now + 2 * c["pages"]) + 32 * c["B"], "flops": 1}
    s, lens = SIZE[c["dtype"]], _lens(c)
    T = sum(n for n, _ in lens)
    if c["kind"] == "commit":
        # the branch that moves is not known before; of a tree of n nodes here about as many rows as its depth
        rows = sum(min(n, 4) for n, _ in lens)
        return {"bytes": 4 * rows * c["layers"] * c["hkv"] * c["d"] * s + 12 * T + 20 * c["B"], "flops": 1}
    keys = pairs = 0
    for n, kv in lens:
        first = kv - n
        before = min(first, c["window"]) if c["window"] else first
        keys += before + n if n else 0
        pairs += n * before + 4 * n
    b = 2 * keys * c["hkv"] * c["d"] * s + 2 * T * c["hq"] * c["d"] * s + 4 * T * c["hq"] + T * 4 * (2 + c["q"] // 32)
    return {"bytes": b, "flops": 4 * c["d"] * c["hq"] * pairs}


# ----------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _bits(masks, V):
    """int32 [..., words] -> bool [..., V]"""
    return ((masks[..., None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1).bool().flatten(-2)[..., :V]


def _words(bits):
    """bool [..., V] -> int32 [..., words]"""
    W = (bits.shape[-1] + 31) // 32
    full = torch.nn.functional.pad(bits, (0, W * 32 - bits.shape[-1]))
    return (full.unflatten(-1, (W, 32)).long() << torch.arange(32, device=DEV)).sum(-1).to(torch.int32)


def _prepare_sample(c, gen):
    B, V = c["B"], c["V"]
    # logits of a model: a broad bulk and a handful of tokens that stand out, less or more
    z = 1.5 * torch.randn((B, V), generator=gen, device=DEV)
    z.scatter_add_(1, torch.randint(V, (B, 12), generator=gen, device=DEV), 6 + 12 * torch.rand((B, 12), generator=gen, device=DEV))
    s = {"case": c, "logits": z.to(DTYPES[c["dtype"]]), "mask": None}
    if c["masked"]:
        # what a grammar allows: a handful of tokens, a class of words, or nearly everything inside a string
        u, v = (torch.rand((B, 1), generator=gen, device=DEV) for _ in range(2))
        share = torch.where(u < 0.3, 8.0 / V, torch.where(u < 0.7, 0.005 + 0.05 * v, 0.5 + 0.45 * v))
        s["mask"] = _words(torch.rand((B, V), generator=gen, device=DEV) < share)
    s["temperature"] = 0.5 + torch.rand(B, generator=gen, device=DEV)
    s["temperature"][torch.rand(B, generator=gen, device=DEV) < 0.1] = 0.0
    k, p, m = zip(*_filters(c))
    s["top_k"], s["top_p"], s["min_p"] = _ints(k), torch.tensor(p, device=DEV), torch.tensor(m, device=DEV)
    s["noise"] = torch.empty((B, V), device=DEV).exponential_(generator=gen).clamp_min(1e-20)
    return s


def _trees(lens, seed, tokens=False):
    """Random trees: every node's parent among the eight before it (the first is the root), and, with tokens, a few
    children's tokens as what the target says after a node."""
    r = random.Random(seed)
    parent, token, said = [], [], []
    for n, _ in lens:
        up = [-1] + [i - 1 - r.randrange(min(i, 8)) for i in range(1, n)]
        parent += up[:n]
        if tokens:
            mine = [r.randrange(40) for _ in range(n)]
            next_of = [[] for _ in range(n)]
            for i in range(1, n):
                next_of[up[i]].append(mine[i])
            token += mine
            said += [r.choice(x) if x and r.random() < 0.8 else r.randrange(40) for x in next_of]
    return parent, token, said


def _prepare_chunks(c, gen):
    lens, page = _lens(c), c["page"]
    need = [-(-kv // page) for _, kv in lens]
    P, M = sum(need) + 1, max(need + [1])
    # pages are handed out as they come free: in no order
    order = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)
    starts = _ints([sum(need[:b]) for b in range(len(need))])
    col = torch.arange(M, device=DEV, dtype=torch.int32)
    table = torch.where(col[None] < _ints(need)[:, None], order[(starts[:, None] + col[None]).clamp(max=P - 1).long()], 0)
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    return {"case": c, "P": P, "table": table.to(torch.int32).contiguous(), "kv_len": _ints([kv for _, kv in lens]),
            "cu_q": _ints(cu), "T": cu[-1], "max_q": max(n for n, _ in lens), "max_kv": max(kv for _, kv in lens)}


def _padded(s, x, fill):
    """[T] -> [B, max_q], of every sequence its own."""
    b, i = _places(s)
    y = torch.full((s["case"]["B"], s["max_q"]), fill, dtype=x.dtype, device=DEV)
    y[b, i] = x
    return y


def _ancestors(parent):
    """[B, n] parents -> bool [B, n, n]: j is i or one of its ancestors."""
    B, n = parent.shape
    step = torch.eye(n, dtype=torch.float64, device=DEV).repeat(B, 1, 1)
    step += (parent[..., None] == torch.arange(n, device=DEV)).double()
    return torch.linalg.matrix_power(step, n) > 0


def prepare(case, seed):
    c, gen = dict(case), _generator(seed)
    c.pop("name", None)
    if c["kind"] == "sample":
        return _prepare_sample(c, gen)
    if c["kind"] == "copy":
        return _prepare_copy(c, gen)
    if c["kind"] == "fork":
        return _prepare_fork(c, gen)
    s, dt = _prepare_chunks(c, gen), DTYPES[c["dtype"]]
    parent, token, said = _trees(_lens(c), seed, c["kind"] == "commit")
    s["parent"] = _ints(parent)
    if c["kind"] == "commit":
        s["tokens"], s["sampled"] = _ints(token), _ints(said)
        shape = (2, c["layers"], s["P"], c["page"], c["hkv"], c["d"])
        s["pages"] = torch.randn(shape, generator=gen, device=DEV, dtype=dt)
        return s
    shape = (s["P"], c["page"], c["hkv"], c["d"])
    s["k_pages"], s["v_pages"] = (torch.randn(shape, generator=gen, device=DEV, dtype=dt) for _ in range(2))
    s["q"] = (2 * torch.randn((s["T"], c["hq"], c["d"]), generator=gen, device=DEV)).to(dt)
    # once a step: what every layer's attention is given of the tree
    above = _ancestors(_padded(s, s["parent"], -1))
    b, i = _places(s)
    s["tree"], s["depth"] = _words(above[b, i]), (above[b, i].sum(-1) - 1).to(torch.int32)
    return s


def _rows(c):
    r = random.Random(c["shape"])
    return [r.randint(1, c["page"]) if c["partial"] else c["page"] for _ in range(c["n"])]


def _prepare_copy(c, gen):
    order = torch.randperm(c["pages"], generator=gen, device=DEV).to(torch.int32)
    src, dst = order[:c["n"]].contiguous(), order[c["n"]:2 * c["n"]].contiguous()
    shape = (2, c["layers"], c["pages"], c["page"], c["hkv"], c["d"])
    return {"case": c, "pages": torch.randn(shape, generator=gen, device=DEV, dtype=DTYPES[c["dtype"]]), "src": src,
            "dst": dst, "rows": _ints(_rows(c)) if c["partial"] else None}


def _prepare_fork(c, gen):
    lens, parent, keep, room = _fork_plan(c)
    held = [-(-n // c["page"]) for n in lens]
    cols = max(max(held), max(-(-max(k, n) // c["page"]) for k, n in zip(keep, room)))
    order = torch.randperm(c["pages"], generator=gen, device=DEV).to(torch.int32)
    col, starts = torch.arange(cols, device=DEV), torch.tensor([0] + held, device=DEV).cumsum(0)[:-1]
    mine = col[None] < _ints(held)[:, None]
    table = torch.where(mine, order[(starts[:, None] + col[None]).clamp(max=c["pages"] - 1)], -1).to(torch.int32)
    refs = torch.zeros(c["pages"], dtype=torch.int32, device=DEV)
    refs[order[:sum(held)].long()] = 1
    # some pages are held by others too
    refs[order[sum(held):].long()] = (torch.rand(c["pages"] - sum(held), generator=gen, device=DEV) < 0.1).to(torch.int32)
    need = sum(-(-max(k, n) // c["page"]) + 1 for k, n in zip(keep, room))
    refs[order[sum(held):sum(held) + need].long()] = 0
    return {"case": c, "table": table, "held": _ints(held), "parent": _ints(parent), "keep": _ints(keep), "room": _ints(room),
            "refs": refs}


# -------------------------------------------------------------------------------------------------------------- run
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"sample": _own_sample, "attend": _own_attend, "commit": _own_commit, "copy": _own_copy, "fork": _own_fork}[kind](s)
    return {"sample": _plain_sample, "attend": _plain_attend, "commit": _plain_commit, "copy": _plain_copy,
            "fork": _plain_fork}[kind](s)


def _own_sample(s):
    import paper_2607_11951_amd as G
    tokens, logprobs = G.sample(s["logits"], mask=s["mask"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                min_p=s["min_p"], noise=s["noise"])
    return {"tokens": tokens, "logprobs": logprobs}


def _own_attend(s):
    import paper_2607_11951_amd as G
    out, lse = G.attend_tree(s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["cu_q"], s["tree"], s["max_q"],
                             s["max_kv"], depth=s["depth"], window=s["case"]["window"])
    return {"out": out, "lse": lse}


def _own_commit(s):
    import paper_2607_11951_amd as G
    path, length, following = G.commit_tree(s["pages"][0], s["pages"][1], s["table"], s["kv_len"], s["cu_q"], s["tokens"],
                                            s["parent"], s["sampled"], s["max_q"])
    return {"path": path, "length": length, "next": following, "pages": s["pages"]}


def _own_copy(s):
    import paper_2607_11951_amd as G
    G.kv_copy(s["pages"][0], s["pages"][1], s["src"], s["dst"], rows=s["rows"])
    return {"pages": s["pages"]}


def _own_fork(s):
    import paper_2607_11951_amd as G
    table, held, refs, copies, status = G.kv_fork(s["table"], s["held"], s["parent"], s["keep"], s["room"], s["refs"],
                                                  s["case"]["page"])
    return {"table": table, "held": held, "refs": refs, "copies": copies, "status": status}


def _plain_sample(s):
    B, V = s["logits"].shape
    l = s["logits"].float()
    if s["mask"] is not None:
        l = l.masked_fill(~_bits(s["mask"], V), -math.inf)
    cold = s["temperature"] <= 0
    T = torch.where(cold, 1.0, s["temperature"]).double()
    m = l.amax(-1)
    alive = m > -math.inf
    at = torch.arange(V, device=DEV)
    best = torch.where(l == m[:, None], at, V).amin(-1)
    # in order: the larger logits first, of equal ones the lower index
    x, order = l.sort(dim=-1, descending=True, stable=True)
    w = ((x.double() - torch.where(alive, m, 0.0)[:, None].double()) / T[:, None]).exp()
    k = torch.where((s["top_k"] > 0) & ~cold, s["top_k"], V)
    kept = at < k[:, None]
    upto = torch.where(kept, w, 0.0).cumsum(-1)
    kept &= (upto - w < s["top_p"].double()[:, None] * upto[:, -1:]) | ((s["top_p"] >= 1) | cold)[:, None] | (at == 0)
    kept &= (w >= s["min_p"].double()[:, None]) | cold[:, None]
    w = torch.where(kept, w, 0.0)
    score = w / s["noise"].gather(-1, order).double()
    top = score.amax(-1, keepdim=True)
    new = torch.where((score == top) & (score > 0), order, V).amin(-1)
    new = torch.where(alive, torch.where(cold, best, new), -1)
    chosen = l.gather(-1, new.clamp(0, V - 1)[:, None])[:, 0]
    logp = (chosen.double() - m.double()) / T - w.sum(-1).clamp_min(1e-300).log()
    return {"tokens": new.to(torch.int32), "logprobs": torch.where(alive, logp, 0.0).float()}


def _places(s):
    """Of every chunk token: its sequence and its place in the chunk."""
    t = torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(s["cu_q"].long(), t, right=True) - 1
    return b, t - s["cu_q"].long()[b]


def _plain_attend(s):
    c = s["case"]
    B, H, G, D, n = c["B"], c["hkv"], c["hq"] // c["hkv"], c["d"], s["max_q"]
    k = s["k_pages"][s["table"].long()].flatten(1, 2)[:, :s["max_kv"]].float()            # [B, S, H, D]
    v = s["v_pages"][s["table"].long()].flatten(1, 2)[:, :s["max_kv"]].float()
    b, i = _places(s)
    q = torch.zeros((B, n, c["hq"], D), device=DEV)
    q[b, i] = s["q"].float()
    q = q.view(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(D ** -0.5).view(B, H, G, n, -1)
    first = (s["kv_len"] - (s["cu_q"][1:] - s["cu_q"][:-1]))[:, None, None]
    key = torch.arange(x.shape[-1], device=DEV)
    before = key < first
    if c["window"]:
        depth = _padded(s, s["depth"], 0)
        before = before & (key > first + depth[..., None] - c["window"])
    above = torch.zeros((B, n, n), dtype=torch.bool, device=DEV)
    above[b, i] = _bits(s["tree"], n)
    inside = above.gather(-1, (key - first).clamp(0, n - 1).expand(B, n, -1)) & (key >= first) & (key < s["kv_len"][:, None, None])
    x.masked_fill_(~(before | inside)[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-1e30)
    x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, H, G * n, -1), v.permute(0, 2, 1, 3).contiguous()).view(B, H, G, n, D) / z.clamp_min(1e-30)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, c["hq"], D)
    lse = (m + z.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, c["hq"])
    return {"out": o[b, i].to(s["q"].dtype), "lse": lse[b, i]}


def _plain_commit(s):
    c = s["case"]
    B, n, page = c["B"], s["max_q"], c["page"]
    size = s["cu_q"][1:] - s["cu_q"][:-1]
    parent, token, said = (_padded(s, s[x], -1).long() for x in ("parent", "tokens", "sampled"))
    at = torch.arange(n, device=DEV)
    real = at < size[:, None]
    above = _ancestors(parent)
    # a node is right when the target says its token after its parent, and it is the first child with that token
    right = (token == said.gather(-1, parent.clamp_min(0))) & (parent >= 0)
    twin = (parent[:, :, None] == parent[:, None]) & (token[:, :, None] == token[:, None]) & (at[None] < at[:, None])
    right &= ~twin.any(-1)
    right[:, 0] = True
    kept = (right[:, None] | ~above).all(-1) & above[..., 0] & real
    length = kept.sum(-1)
    path = torch.where(kept, at, n).sort(-1).values
    path = torch.where(path < n, path, -1)
    last = path.gather(-1, (length - 1).clamp_min(0)[:, None])[:, 0]
    following = torch.where(length > 0, said.gather(-1, last.clamp_min(0)[:, None])[:, 0], -1)
    # the branch's rows, together behind the text
    b, i = (path >= 0).nonzero(as_tuple=True)
    first = (s["kv_len"] - size).long()[b]
    table, to, fro = s["table"].long(), first + i, first + path[b, i]
    s["pages"][:, :, table[b, to // page], to % page] = s["pages"][:, :, table[b, fro // page], fro % page]
    return {"path": path.to(torch.int32), "length": length.to(torch.int32), "next": following.to(torch.int32), "pages": s["pages"]}


def _plain_copy(s):
    src, dst, page = s["src"].long(), s["dst"].long(), s["case"]["page"]
    if s["rows"] is None:
        s["pages"][:, :, dst] = s["pages"][:, :, src]
    else:
        i, r = (torch.arange(page, device=DEV) < s["rows"][:, None]).nonzero(as_tuple=True)
        s["pages"][:, :, dst[i], r] = s["pages"][:, :, src[i], r]
    return {"pages": s["pages"]}


def _plain_fork(s):
    page, table = s["case"]["page"], s["table"].long()
    cols, P, R = table.shape[1], len(s["refs"]), len(s["parent"])
    parent, keep, room = (s[x].long() for x in ("parent", "keep", "room"))
    col, row = torch.arange(cols, device=DEV), torch.arange(R, device=DEV)
    keep = torch.where(parent >= 0, keep, 0)
    kept = -(-keep // page)
    mine = col < kept[:, None]
    new = torch.where(mine, table[parent.clamp_min(0)], -1)
    # who holds what, once the kept pages have been handed on
    refs = s["refs"].long()
    refs = refs.scatter_add(0, table[col < s["held"][:, None]], torch.full_like(table, -1)[col < s["held"][:, None]])
    refs = refs.scatter_add(0, new[mine], torch.ones_like(new)[mine])
    # a row that goes on writing into its last page needs it for itself: of those who only write the first may keep it
    writes = (room > keep) & (keep % page > 0)
    last = new.gather(-1, (kept - 1).clamp_min(0)[:, None])[:, 0].clamp_min(0)
    spare = torch.where(writes, last, P)
    writers = torch.zeros(P + 1, dtype=torch.long, device=DEV).scatter_add(0, spare, torch.ones_like(spare))
    lowest = torch.full((P + 1,), R, device=DEV).scatter_reduce(0, spare, row, "amin")
    copy = writes & ~((refs[last] == writers[last]) & (lowest[last] == row))
    grow = -(-torch.maximum(room, keep) // page) - kept
    need = grow + copy
    upto = need.cumsum(0)
    free = (refs == 0).nonzero()[:, 0]
    ok = (upto <= len(free)) | (need == 0)
    free = torch.nn.functional.pad(free, (0, 1), value=-1)
    before = (upto - need).clamp(max=len(free) - 1)
    given = ok[:, None] & (col >= kept[:, None]) & (col < (kept + grow)[:, None])
    new = torch.where(given, free[(before[:, None] + copy[:, None] + col - kept[:, None]).clamp(0, len(free) - 1)], new)
    copy &= ok
    to = torch.where(copy, free[before], -1)
    new = torch.where(copy[:, None] & (col == kept[:, None] - 1), to[:, None], new)
    refs = refs.scatter_add(0, last, -copy.long())
    taken = torch.cat([new[given], to[copy]])
    refs = refs.scatter(0, taken, torch.ones_like(taken))
    copies = torch.stack([torch.where(copy, last, -1), to, torch.where(copy, keep % page, 0)])
    return {"table": new.to(torch.int32), "held": (kept + torch.where(ok, grow, 0)).to(torch.int32), "refs": refs.to(torch.int32),
            "copies": copies.to(torch.int32), "status": torch.where(ok, 0, 4).to(torch.int32)}


# ------------------------------------------------------------------------------------------- the definition, 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind = s["case"]["kind"]
    if kind == "fork":  # whole numbers only
        return None
    return {"sample": _exact_sample, "attend": _exact_attend, "commit": _exact_commit, "copy": _exact_copy}[kind](s)


def _exact_sample(s):
    B, V = s["logits"].shape
    temps, ks, ps, ms = (s[x].double().tolist() for x in ("temperature", "top_k", "top_p", "min_p"))
    out = torch.zeros(B, dtype=torch.float64, device=DEV)
    for b in range(B):
        x = s["logits"][b].double()
        ids = torch.arange(V, device=DEV) if s["mask"] is None else _bits(s["mask"][b], V).nonzero()[:, 0]
        if len(ids) == 0:
            continue
        x = x[ids]
        if temps[b] <= 0:
            out[b] = x.max() - torch.logsumexp(x, 0)
            continue
        down = torch.argsort(-x, stable=True)[:int(ks[b]) if ks[b] > 0 else V]
        ids, x = ids[down], x[down]
        p = torch.softmax(x / temps[b], 0)
        n = len(p)
        if ps[b] < 1:
            n = max(1, int(((p.cumsum(0) - p) < ps[b]).sum()))
        n = min(n, int((p >= ms[b] * p[0]).sum()))
        p = p[:n] / p[:n].sum()
        out[b] = p[torch.argmax(p / s["noise"][b, ids[:n]].double())].log()
    return {"tokens": None, "logprobs": out}


def _exact_attend(s):
    c, out, lse = s["case"], [], []
    cu, kv, parent, group = s["cu_q"].tolist(), s["kv_len"].tolist(), s["parent"].tolist(), c["hq"] // c["hkv"]
    for b in range(c["B"]):
        n, S = cu[b + 1] - cu[b], kv[b]
        if n == 0:
            continue
        low = max(0, S - n - c["window"] + 1) if c["window"] else 0
        seen = torch.zeros((n, S), dtype=torch.bool)
        depth = []
        for i in range(n):
            up = parent[cu[b] + i]
            depth.append(0 if up < 0 else depth[up] + 1)
            if up >= 0:
                seen[i, S - n:] = seen[up, S - n:]
            seen[i, S - n + i] = True
            seen[i, max(0, S - n + depth[i] - c["window"] + 1) if c["window"] else 0:S - n] = True
        seen = seen[:, low:].repeat_interleave(group, 0).to(DEV)
        pages = s["table"][b, :-(-S // c["page"])].long()
        k, v = (x[pages].reshape(-1, c["hkv"], c["d"])[low:S].double() for x in (s["k_pages"], s["v_pages"]))
        q = s["q"][cu[b]:cu[b + 1]].double().view(n, c["hkv"], group, c["d"])
        o = torch.empty((n, c["hkv"], group, c["d"]), dtype=torch.float64, device=DEV)
        e = torch.empty((n, c["hkv"], group), dtype=torch.float64, device=DEV)
        for g in range(c["hkv"]):
            x = q[:, g].reshape(n * group, c["d"]) @ k[:, g].T.contiguous() / math.sqrt(c["d"])
            x[~seen] = -math.inf
            z = torch.logsumexp(x, -1)
            e[:, g] = z.view(n, group)
            o[:, g] = (torch.exp(x - z[:, None]) @ v[:, g].contiguous()).view(n, group, c["d"])
        out.append(o.flatten(1, 2))
        lse.append(e.flatten(1, 2))
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def _exact_commit(s):
    c, pages = s["case"], s["pages"].double()
    cu, kv, parent, token, said = (s[x].tolist() for x in ("cu_q", "kv_len", "parent", "tokens", "sampled"))
    for b in range(c["B"]):
        n, first = cu[b + 1] - cu[b], kv[b] - cu[b + 1] + cu[b]
        at, fro = 0, [0]
        while True:
            after = [i for i in range(at + 1, n) if parent[cu[b] + i] == at and token[cu[b] + i] == said[cu[b] + at]]
            if not after:
                break
            at = after[0]
            fro.append(at)
        place = [(int(s["table"][b, p // c["page"]]), p % c["page"]) for p in range(first, kv[b])]
        for i, f in enumerate(fro):
            if f != i:
                pages[:, :, place[i][0], place[i][1]] = pages[:, :, place[f][0], place[f][1]]
    return {"path": None, "length": None, "next": None, "pages": pages}


def _exact_copy(s):
    pages = s["pages"].double()
    for i, (a, b) in enumerate(zip(s["src"].tolist(), s["dst"].tolist())):
        n = s["case"]["page"] if s["rows"] is None else int(s["rows"][i])
        pages[:, :, b, :n] = pages[:, :, a, :n]
    return {"pages": pages}
