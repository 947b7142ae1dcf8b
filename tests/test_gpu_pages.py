"""grid_kv_copy and grid_kv_fork on the GPU against plain implementations: whole numbers and copies, so all is equal."""

import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

OK, BAD, OVER = 0, 2, 4


@pytest.fixture(scope="module")
def G():
    import paper_2607_11951_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    pkg.lib()
    return pkg


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# -------------------------------------------------------------------------------------------------------------- copy
@pytest.mark.parametrize("page", [1, 3, 16, 64, 300])
@pytest.mark.parametrize("heads", [(4, 128), (1, 8), (12, 64), (3, 24), (40, 256)])
@pytest.mark.parametrize("layers", [1, 3])
def test_copy(G, page, heads, layers):
    P, n = 40, 17
    if page * heads[0] * heads[1] > 1 << 18:
        P, n = 9, 4
    r = random.Random(page)
    k, v = (torch.randn((layers, P, page) + heads, device="cuda").bfloat16() for _ in range(2))
    order = r.sample(range(P), 2 * n)
    for rows in (None, [r.randrange(-1, page + 2) for _ in range(n)]):
        want_k, want_v = k.clone(), v.clone()
        for i in range(n):
            m = page if rows is None else min(max(rows[i], 0), page)
            want_k[:, order[n + i], :m] = k[:, order[i], :m]
            want_v[:, order[n + i], :m] = v[:, order[i], :m]
        got_k, got_v = k.clone(), v.clone()
        assert G.kv_copy(got_k, got_v, ints(order[:n]), ints(order[n:]), rows=None if rows is None else ints(rows)) is None
        assert torch.equal(got_k, want_k) and torch.equal(got_v, want_v)
        if layers == 1:
            got_k, got_v = k[0].clone(), v[0].clone()
            G.kv_copy(got_k, got_v, ints(order[:n]), ints(order[n:]), rows=None if rows is None else ints(rows))
            assert torch.equal(got_k, want_k[0]) and torch.equal(got_v, want_v[0])


def test_copy_layouts_and_what_is_left_out(G):
    """heads before rows, keys and values side by side, layers innermost; ids that are no pages; the same page twice"""
    P, L, page, H, D = 11, 3, 10, 2, 64
    store = torch.randn((P, H, page, L, 2, D), device="cuda").half()
    k, v = (store[:, :, :, :, i].permute(3, 0, 2, 1, 4) for i in range(2))
    want = store.clone()
    want[7], want[1, :, :4] = store[2], store[0, :, :4]
    G.kv_copy(k, v, ints([2, 0, -1, 3, 5, P, 4]), ints([7, 1, 8, -1, 5, 9, 1 << 30]), rows=ints([10, 4, 10, 10, 10, 10, 10]))
    assert torch.equal(store, want)
    G.kv_copy(k, v, ints([]), ints([]))
    assert torch.equal(store, want)


def test_copy_of_large_pages_graph_and_stream(G):
    k, v = (torch.randn((2, 9, 256, 8, 128), device="cuda").bfloat16() for _ in range(2))
    first = k.clone(), v.clone()
    src, dst, rows = ints([0, 1, 2]), ints([3, 4, 5]), ints([256, 100, 0])
    G.kv_copy(k, v, src, dst, rows=rows)
    want = k.clone(), v.clone()
    assert torch.equal(k[:, 3], first[0][:, 0]) and torch.equal(k[:, 4, :100], first[0][:, 1, :100])
    assert torch.equal(k[:, 4, 100:], first[0][:, 4, 100:]) and torch.equal(v[:, 5], first[1][:, 5])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.kv_copy(k, v, src, dst, rows=rows)
    for _ in range(3):
        k.copy_(first[0]), v.copy_(first[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    k.copy_(first[0]), v.copy_(first[1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    G.kv_copy(k, v, src, dst, rows=rows, stream=side)
    side.synchronize()
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_copy_past_32_bits(G):
    """a cache of more than 2^32 entries: from its end to its beginning"""
    page, H, D = 64, 8, 128
    P = (1 << 32) // (page * H * D) + 40
    k, v = (torch.empty((P, page, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[P - 2], v[P - 2] = (torch.randn((page, H, D), device="cuda").bfloat16() for _ in range(2))
    k[3], v[P - 1] = k[P - 2] + 1, 2
    G.kv_copy(k, v, ints([P - 2, 3]), ints([0, P - 1]))
    assert torch.equal(k[0], k[P - 2]) and torch.equal(v[0], v[P - 2])
    assert torch.equal(k[P - 1], k[3]) and torch.equal(v[P - 1], v[3])


# -------------------------------------------------------------------------------------------------------------- fork
def plain_fork(table, held, parent, keep, room, refs, page):
    """the definition, a row after the other"""
    cols, P, R, n_in = len(table[0]), len(refs), len(parent), len(table)
    refs, up = list(refs), lambda n: -(-n // page)
    clamped = [min(max(h, 0), cols) for h in held]
    for r in range(n_in):
        for p in table[r][:clamped[r]]:
            if 0 <= p < P:
                refs[p] -= 1
    rows, status, kept, grow = [], [], [], []
    for b in range(R):
        k = keep[b] if parent[b] >= 0 else 0
        bad = parent[b] < -1 or parent[b] >= n_in or (parent[b] >= 0 and keep[b] < 0)
        n = g = 0
        if not bad:
            n, g = up(k), up(max(room[b], k)) - up(k)
            bad = (parent[b] >= 0 and n > clamped[parent[b]]) or n + g > cols
        mine = list(table[parent[b]][:n]) if not bad and parent[b] >= 0 else []
        bad = bad or any(not 0 <= p < P for p in mine)
        mine = [] if bad else mine
        rows.append(mine)
        status.append(BAD if bad else OK)
        kept.append(len(mine))
        grow.append(0 if bad else g)
        for p in mine:
            refs[p] += 1
    last = [rows[b][-1] if status[b] == OK and kept[b] and room[b] > keep[b] and keep[b] % page else -1 for b in range(R)]
    copies, free, left = [[-1] * R, [-1] * R, [0] * R], [p for p in range(P) if refs[p] == 0], True
    after = list(refs)
    for b in range(R):
        writers = [r for r in range(R) if last[r] == last[b]]
        copy = last[b] >= 0 and not (len(writers) == refs[last[b]] and writers[0] == b)
        need = grow[b] + copy
        if need == 0:
            continue
        left = left and need <= len(free)
        if not left:
            status[b] = OVER
            continue
        new, free = free[:need], free[need:]
        for p in new:
            after[p] = 1
        if copy:
            after[last[b]] -= 1
            rows[b][-1] = new[0]
            copies[0][b], copies[1][b], copies[2][b] = last[b], new[0], keep[b] % page
        rows[b] += new[copy:]
    return ([r + [-1] * (cols - len(r)) for r in rows], [len(r) for r in rows], after, copies, status)


def world(R, page, cols, P, seed, longest):
    """rows that hold pages of a pool, some of them shared, some held by others too"""
    r = random.Random(seed)
    refs, table, held, lens = [0] * P, [], [], []
    free = r.sample(range(P), P)
    for b in range(R):
        n = r.randint(0, longest)
        pages = -(-n // page)
        if b and r.random() < 0.4:
            base = r.randrange(b)
            share = r.randint(0, min(pages, held[base]))
            mine = table[base][:share]
        else:
            mine = []
        while len(mine) < pages and free:
            mine = mine + [free.pop()]
        n = min(n, len(mine) * page)
        for p in mine:
            refs[p] += 1
        table.append(mine + [r.choice([-1, -7, 1 << 30])] * (cols - len(mine)))
        held.append(len(mine))
        lens.append(n)
    for p in free:
        if r.random() < 0.1:
            refs[p] += 1
    for p in range(P):
        if refs[p] and r.random() < 0.1:
            refs[p] += r.randint(1, 3)
    return table, held, lens, refs


def check_fork(G, table, held, parent, keep, room, refs, page, **kw):
    want = plain_fork(table, held, parent, keep, room, refs, page)
    got = G.kv_fork(ints(table), ints(held), ints(parent), ints(keep), ints(room), ints(refs), page, **kw)
    for x, y, name in zip(got, want, ("table", "held", "refs", "copies", "status")):
        assert x.tolist() == y, name
    return want


@pytest.mark.parametrize("page", [1, 4, 16, 100])
@pytest.mark.parametrize("R", [1, 3, 40, 300])
@pytest.mark.parametrize("seed", range(4))
def test_fork(G, page, R, seed):
    r = random.Random(1000 * seed + R)
    longest, grow = 20 * page, [1, 3 * page, 3 * page, page][seed]
    P = R * 20 + [R * 30, R * 30, 5, 4500][seed]
    table, held, lens, refs = world(R, page, 30, P, seed, longest)
    n = [R, R, max(1, R // 2), R + 5][seed]
    parent = [r.choice([b if b < R else -1, b if b < R else -1, r.randrange(R), -1]) for b in range(n)]
    keep = [0 if p < 0 else r.choice([lens[p], lens[p], r.randint(0, lens[p])]) for p in parent]
    room = [k + r.choice([0, 1, r.randint(0, grow)]) for k in keep]
    check_fork(G, table, held, parent, keep, room, refs, page)


def test_beams(G):
    """eight rows go on from one or two texts: the first writes on in the last page, the others get copies"""
    table = [[5, 3, 9, -1], [5, 3, 8, -1], [0, 0, 0, 0]]
    refs = [0, 0, 0, 2, 0, 2, 0, 0, 1, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1]
    got = check_fork(G, table, [3, 3, 0], [0, 0, 1, 0, -1], [9, 9, 10, 6, 0], [13, 10, 12, 8, 3], refs, 4)
    assert got[3][0][:4] == [-1, 9, -1, 3] and got[4] == [OK] * 5


def test_fork_gives_pages_back_and_out_again(G):
    refs = [1] * 6
    got = check_fork(G, [[0, 1, 2], [3, 4, 5]], [3, 3], [-1, 1], [0, 2], [0, 24], refs, 8)
    assert got[0] == [[-1, -1, -1], [3, 0, 1]] and got[2] == [1, 1, 0, 1, 0, 0]


def test_fork_when_pages_run_out(G):
    """from the first row on that is too long none gets any; what the others keep stays as it was, shared or not"""
    table = [[0, 1, -1, -1, -1, -1], [2, -1, -1, -1, -1, -1]]
    refs = [1, 1, 1, 0, 0, 0]
    got = check_fork(G, table, [2, 1], [0, 1, 0, 1, 1], [8, 2, 7, 3, 4], [12, 17, 8, 3, 4], refs, 4)
    assert got[4] == [OK, OVER, OVER, OK, OK]
    check_fork(G, table, [2, 1], [0, 0, 0], [5, 5, 5], [6, 6, 6], [2, 1, 1, 1, 1, 1], 4)


def test_fork_of_bad_rows(G):
    table = [[0, 1, 9, -1], [2, -3, 4, 5]]
    refs = [1, 1, 1, 0, 1, 1, 0, 0]
    got = check_fork(G, table, [3, 9], [0, 1, 2, -2, 0, 0, 1, 0, -1], [8, 16, 0, 0, -1, 20, 4, 4, -5], [9, 17, 1, 1, 4, 20, 17, 8, 4],
                     refs, 4)
    assert got[4] == [OK, BAD, BAD, BAD, BAD, BAD, BAD, OK, OK]
    # a kept entry that is no page, a longer row than the table
    check_fork(G, table, [3, 4], [0, 0], [9, 12], [9, 12], refs, 4)
    check_fork(G, table, [-5, 4], [0, 1], [1, 4], [1, 4], refs, 4)


@pytest.mark.parametrize("P", [63, 64, 65, 4095, 4096, 4097, 300000])
def test_pools_of_any_size(G, P):
    r = random.Random(P)
    refs = [int(r.random() < 0.5) for _ in range(P)]
    free = refs.count(0)
    for ask in (free // 3, free // 3 + 1):
        check_fork(G, [[-1] * (ask + 1)], [0], [-1, -1, -1], [0, 0, 0], [ask, ask, ask], refs, 1)


def test_many_rows(G):
    R = 3000
    table, held, lens, refs = world(R, 4, 6, 20000, 1, 16)
    r = random.Random(5)
    parent = [r.choice([b, b, b, r.randrange(R), -1]) for b in range(R)]
    keep = [0 if p < 0 else lens[p] for p in parent]
    room = [k + r.randint(0, 6) for k in keep]
    check_fork(G, table, held, parent, keep, room, refs, 4)


def test_fork_strides_given_outputs_in_place_and_graph(G):
    page, R, cols = 4, 24, 12
    table, held, lens, refs = world(R, page, cols, 600, 3, 30)
    r = random.Random(2)
    parent = [r.choice([b, r.randrange(R)]) for b in range(R)]
    keep = [lens[p] for p in parent]
    room = [k + r.randint(0, 9) for k in keep]
    want = plain_fork(table, held, parent, keep, room, refs, page)
    wide = torch.full((R, 20), -9, dtype=torch.int32, device="cuda")
    wide[:, 3:15] = ints(table)
    out = torch.full((R, 30), 77, dtype=torch.int32, device="cuda")
    counts = ints(refs)
    args = (wide[:, 3:15], ints(held), ints(parent), ints(keep), ints(room))
    made = dict(held_out=torch.empty(R, dtype=torch.int32, device="cuda"), copies=torch.empty((3, R), dtype=torch.int32, device="cuda"),
                status=torch.empty(R, dtype=torch.int32, device="cuda"), workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    got = G.kv_fork(*args, counts, page, table_out=out[:, 5:17], refs_out=counts, **made)
    assert got[2] is counts and got[1] is made["held_out"]
    for x, y in zip(got, want):
        assert x.tolist() == y
    assert bool((out[:, :5] == 77).all()) and bool((out[:, 17:] == 77).all())
    graph, refs_out = torch.cuda.CUDAGraph(), torch.empty_like(counts)
    before = ints(refs)
    with torch.cuda.graph(graph):
        G.kv_fork(*args, before, page, table_out=out[:, 5:17], refs_out=refs_out, **made)
    for _ in range(4):
        for x in (out, refs_out, *made.values()):
            x.fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out[:, 5:17], made["held_out"], refs_out, made["copies"], made["status"]), want):
            assert x.tolist() == y


def test_forked_rows_read_what_they_wrote(G):
    """a cache through several steps of forks and copies: every row's text is what it would be without sharing"""
    page, P, cols, H, D = 4, 200, 12, 1, 8
    r, R = random.Random(7), 6
    k, v = (torch.zeros((2, P, page, H, D), device="cuda").bfloat16() for _ in range(2))
    table, held, refs = torch.full((R, cols), -1, dtype=torch.int32, device="cuda"), ints([0] * R), ints([0] * P)
    text = [[] for _ in range(R)]
    for step in range(9):
        parent = [r.choice([b, b, r.randrange(R), -1 if step % 4 == 3 else b]) for b in range(R)]
        keep = [0 if p < 0 else r.choice([len(text[p]), max(0, len(text[p]) - r.randint(0, 3))]) for p in parent]
        new = [[float(r.randrange(200)) for _ in range(r.randint(0, 5))] for _ in range(R)]
        text = [(text[p][:n] if p >= 0 else []) + x for p, n, x in zip(parent, keep, new)]
        table, held, refs, copies, status = G.kv_fork(table, held, ints(parent), ints(keep), ints([len(t) for t in text]), refs, page)
        assert status.tolist() == [0] * R
        G.kv_copy(k, v, copies[0], copies[1], rows=copies[2])
        host = table.tolist()
        for b in range(R):
            for i, x in enumerate(new[b]):
                s = keep[b] + i
                k[:, host[b][s // page], s % page] = x
                v[:, host[b][s // page], s % page] = -x
        for b in range(R):
            at = [(host[b][s // page], s % page) for s in range(len(text[b]))]
            assert [float(k[1, p, i, 0, 3]) for p, i in at] == text[b]
            assert [float(v[0, p, i, 0, 7]) for p, i in at] == [-x for x in text[b]]
        count = np.zeros(P, int)
        for b in range(R):
            for p in host[b][:int(held[b])]:
                count[p] += 1
        assert refs.tolist() == count.tolist()


@pytest.mark.parametrize("R,P", [(32, 16384), (33, 16384), (32, 16385), (300, 9000)])
def test_fork_in_place_in_either_launch(G, R, P):
    """one workgroup or four launches: reference counts in place, rows inside larger tables, replayed graphs"""
    page, cols = 8, 14
    table, held, lens, refs = world(R, page, cols, P, R, 80)
    r = random.Random(R)
    parent = [r.choice([b, b, r.randrange(R), -1]) for b in range(R)]
    keep = [0 if p < 0 else r.choice([lens[p], lens[p] // 2]) for p in parent]
    room = [k + r.choice([0, 1, 20]) for k in keep]
    want = plain_fork(table, held, parent, keep, room, refs, page)
    wide = torch.full((R, 20), -9, dtype=torch.int32, device="cuda")
    wide[:, 3:3 + cols] = ints(table)
    out = torch.full((R, 30), 77, dtype=torch.int32, device="cuda")
    counts, start = ints(refs), ints(refs)
    args = (wide[:, 3:3 + cols], ints(held), ints(parent), ints(keep), ints(room), counts, page)
    kw = dict(table_out=out[:, 5:5 + cols], refs_out=counts)
    got = G.kv_fork(*args, **kw)
    for x, y in zip(got, want):
        assert x.tolist() == y
    assert bool((out[:, :5] == 77).all()) and bool((out[:, 5 + cols:] == 77).all())
    kw.update(held_out=got[1], copies=got[3], status=got[4], workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.kv_fork(*args, **kw)
    for _ in range(4):
        counts.copy_(start)
        for x in (out, *got[1:2], *got[3:]):
            x.fill_(55)
        kw["workspace"].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out[:, 5:5 + cols], got[1], counts, got[3], got[4]), want):
            assert x.tolist() == y
    side = torch.cuda.Stream()
    counts.copy_(start)
    torch.cuda.synchronize()
    got = G.kv_fork(*args[:6], page, stream=side)
    side.synchronize()
    for x, y in zip(got, want):
        assert x.tolist() == y
