"""row_start entries that are not in order, run out of the arrays or give two sequences the same rows: every sequence that is valid gets exactly
what it gets alone, in all of its rows, and rows that nobody has stay as they were."""
import pytest
import torch

import cache_util as U
import tree_util as V
from test_gpu_tree import BF, DEV, F32, HEADS, Case, _ctx, _i32
from tree_plans import kind, owned, tree_plan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    assert torch.cuda.is_available()
    return T


def _far(B, at, value):
    """Trees of three rows in order, but for entry `at`."""
    s = [3 * b for b in range(B + 1)]
    s[at] = value
    return s


STARTS = [[0, 4, 2, 8], [0, 4, -5, 8], [0, 4, 99, 8, 12], [0, 99, 8, 12], [-3, 4, 8, 12], [0, 4, 8, 99], [0, 4, 8, -5], [50, 60, 70, 80], [8, 12, 0, 4],
          [8, 12, 0, 9], [0, 10, 5, 15, 12, 20], [0, 300, 20, 40], [20, 40, 0, 300], [0, 257, 100, 280], [5, 5, 3, 9, 9, 4, 7], [0, 6, 6, 3, 9, 12],
          [12, 300, -(1 << 31), (1 << 31) - 1, 4, 9], _far(100, 70, 20), _far(300, 200, 0), _far(300, 1, 600), _far(300, 290, 3), _far(130, 129, 387)]


@pytest.mark.parametrize("start", STARTS)
@pytest.mark.parametrize("bad", [None, 0])
def test_plan(T, start, bad):
    """bad: a sequence whose parents are not valid."""
    print(f"plan starts {start[:6]} bad={bad}", flush=True)
    B, n_rows, pad = len(start) - 1, max([24] + [x for x in start if x <= 900]), 6
    parent, trees = torch.full((n_rows + pad,), 9999, dtype=torch.int32), owned(start, n_rows)
    g = torch.Generator().manual_seed(B)
    for b in range(B - 1, -1, -1):                                           # (where nobody's range is another's, all of them are trees)
        r = range(max(start[b], 0), min(start[b + 1], n_rows, max(start[b], 0) + 256))
        if len(r):
            parent[r.start:r.stop] = torch.tensor(V.random_tree(g, len(r), 3), dtype=torch.int32)
    for r in trees:
        if r:
            parent[r.start:r.stop] = torch.tensor(V.random_tree(g, len(r), 3), dtype=torch.int32)
    if bad is not None and trees[bad]:
        parent[trees[bad].stop - 1] = len(trees[bad])
    lens = [(37 * b) % 1000 for b in range(B)]
    pos, anc = torch.full((n_rows + pad,), -7, dtype=torch.int32, device=DEV), torch.full((n_rows + pad, 8), -7, dtype=torch.int32, device=DEV)
    ctx = _ctx(T, HEADS["tiny"], F32, B)
    T.tidar_tree_plan(ctx, B, _i32(lens), _i32(start), n_rows, parent.to(DEV)[:n_rows], pos[:n_rows], anc[:n_rows])
    torch.cuda.synchronize()
    T.tidar_destroy(ctx)
    pos, anc, mine = pos.cpu(), anc.cpu(), torch.zeros(n_rows + pad, dtype=torch.bool)
    for b, r in enumerate(trees):
        if not r:
            continue
        mine[r.start:r.stop] = True
        if b == bad:
            assert bool((pos[r.start:r.stop] == -1).all()) and not bool(anc[r.start:r.stop].any())
            continue
        see = V.ancestors(parent[r.start:r.stop].tolist())
        assert pos[r.start:r.stop].tolist() == (lens[b] + see.sum(1) - 1).tolist(), b
        assert torch.equal(anc[r.start:r.stop], V.words(see)), b
    # of the others, rows from the first one within the arrays on are reported, up to the next that another sequence's range has
    ranges = [range(s, e) if 0 <= s <= e <= n_rows and e - s <= 256 else range(0) for s, e in zip(start, start[1:])]
    told = torch.zeros_like(mine)
    for b in range(B):
        if trees[b] is None:
            s = min(max(start[b], 0), n_rows)
            for r in range(s, min(max(start[b + 1], s), n_rows)):
                if any(r in x for i, x in enumerate(ranges) if i != b):
                    break
                told[r] = True
    assert not bool((told & mine).any())
    assert bool((pos[told] == -1).all()) and not bool(anc[told].any())
    rest = ~told & ~mine
    assert bool((pos[rest] == -7).all()) and bool((anc[rest] == -7).all())


# what: heads, type, prefixes, rows of a tree, the plan's kind with exact and with 4-bit pages
CALLS = {
    "few": ("gqa", BF, [40, 100, 55, 60], 7, ("few", "few")),
    "few, cut": ("gqa", BF, [900, 2600, 1500, 1300], 9, ("few, cut", "few, cut")),
    "fp32": ("odd", F32, [40, 100, 55, 60], 9, ("few", "few")),
    "fp32, cut": ("gqa", F32, [400, 1000, 550, 600], 30, ("few, cut", "few, cut")),
    "many, cut": ("8b", BF, [1300, 900, 1100, 1200], 100, ("many, cut", "many, cut")),
    "many, some cut": ("8b", BF, [40, 30] * 32 + [500, 400, 300, 200], 30, ("many, some cut", "many, some cut")),
}


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("what", list(CALLS))
def test_attention(T, four, what):
    """Sequences whose range begins within an earlier one's, beside such that have nobody's rows."""
    heads, dtype, Ls, n, plans = CALLS[what]
    B = len(Ls)
    sizes = [n, 5, n, 7] * (B // 4)
    hint = 4000 if "some" in what else max(Ls)
    print(f"attention starts four={four} {what}", flush=True)
    c = Case(T, four, HEADS[heads], dtype, Ls, sizes, seed=B, max_nodes=n + 24)
    pps = -(-hint // 16) + 1
    c.hint, c.pps, c.n_pages = hint, pps, B * pps + 2
    c.ids = torch.randperm(c.n_pages, generator=torch.Generator().manual_seed(1))[:B * pps].view(B, pps)
    c.build()
    assert kind(tree_plan(c)) == plans[four], kind(tree_plan(c))
    c.call()
    c.check()
    good, s = c.out.clone(), c.start
    last = B - 4
    for at, value in ((2, n - 3), (last + 2, s[last + 1] - 1), (last + 2, s[last] - 2), (B, c.rows), (1, n + 20), (3, s[2] + n + 20), (0, -1)):
        start = list(s)
        start[at] = value
        have = owned(start, c.rows, c.max_nodes)
        c.start_d.copy_(_i32(start))
        for again in range(2):
            c.out.fill_(77)
            c.ws.fill_(255)
            c.call()
            torch.cuda.synchronize()
            touched = torch.zeros(c.rows, dtype=torch.bool, device=DEV)
            for b in range(B):
                r = have[b]
                if r is None:
                    continue
                touched[r.start:r.stop] = True
                if r == range(s[b], s[b + 1]):
                    assert torch.equal(c.out[r.start:r.stop], good[r.start:r.stop]), (at, value, b)
            assert bool((c.out[~touched] == 77).all()), (at, value)
    c.close()


@pytest.mark.parametrize("four", [False, True])
def test_accept_and_commit(T, four):
    """A sequence that has another's rows is reported and stores nothing."""
    heads, B, path, pps, n_pages, rows = (4, 2, 128), 4, 6, 4, 20, 30
    ctx = _ctx(T, heads, BF, B, 2)
    start, lens = [0, 6, 3, 12, 20], [3, 5, 15, 30]                          # sequence 1: 6 .. 3; 2: rows 3 .. 11, three of them sequence 0's
    parent = [-1, 0, 1, 2, 3, 4] + [-1, 0, 1, 2, 3, 4] + [-1, 0, 0, 2, 2, 3, 1, 6] + [0] * 10
    tokens, choice = [1] * rows, [1] * rows
    g = torch.Generator().manual_seed(3)
    table = torch.randperm(n_pages, generator=g)[:B * pps].view(B, pps).to(torch.int32)
    P, new, n, nxt = _i32(lens), _i32([-7] * B), _i32([-7] * B), _i32([-7] * B)
    at, said = torch.full((B, path), -7, dtype=torch.int32, device=DEV), torch.full((B, path), -7, dtype=torch.int32, device=DEV)
    td, st = table.to(DEV), _i32(start)
    T.tidar_tree_accept(ctx, B, P, st, rows, _i32(parent), _i32(tokens), _i32(choice), td, n_pages, path, new, n, at, said, nxt)
    torch.cuda.synchronize()
    for b in range(B):
        s, e = start[b], start[b + 1]
        want = V.accept(lens[b], parent[s:e], tokens[s:e], choice[s:e], 512, table[b].tolist(), n_pages, path) if b in (0, 3) else None
        rows_, toks, last = want if want else ([], [], -1)
        fill = [-1] * (path - len(rows_))
        assert [int(new[b]), int(n[b]), at[b].tolist(), said[b].tolist(), int(nxt[b])] == [
            lens[b] + len(rows_), len(rows_), rows_ + fill, toks + fill, last], b
    k, v = (torch.randn(2, rows, 2, 128, generator=g).to(BF) for _ in range(2))
    n.fill_(3)                                                               # as if all had three rows accepted: 1 and 2 have none
    at[:, :3] = _i32([0, 1, 2])
    new.copy_(P + 3)
    if four:
        pool = torch.full((2, n_pages, 2, 544 * 4), 0xa5, dtype=torch.uint8)
        held = (pool.to(DEV),)
        T.tidar_kv4_tree_commit(ctx, T.tidar_kv4_cache(held[0].data_ptr(), td.data_ptr(), pps, n_pages), B, new, n, at, path, st, rows, k.to(DEV), v.to(DEV))
    else:
        pool = [torch.randn(2, n_pages, 2, *s, generator=g).to(BF) for s in ((16, 128), (128, 16))]
        held = [x.to(DEV) for x in pool]
        T.tidar_tree_commit(ctx, T.tidar_kv_cache(held[0].data_ptr(), held[1].data_ptr(), td.data_ptr(), pps, n_pages), B, new, n, at, path, st, rows,
                            k.to(DEV), v.to(DEV))
    torch.cuda.synchronize()
    for layer in range(2):
        for b in (0, 3):
            for j in range(3):
                p, row = lens[b] + j, start[b] + j
                page = int(table[b, p // 16])
                if four:
                    U.put_rows(pool[layer], 128, [page * 16 + p % 16], k[layer, row:row + 1], v[layer, row:row + 1])
                else:
                    pool[0][layer, page, :, p % 16], pool[1][layer, page, :, :, p % 16] = k[layer, row], v[layer, row]
    for got, want in zip(held, (pool,) if four else pool):
        assert torch.equal(got.cpu(), want)
    T.tidar_destroy(ctx)
