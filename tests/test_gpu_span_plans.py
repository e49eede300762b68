"""Attention over a span by the kernel and the cut that a call gets: every case names its plan, and the plan is checked on the host.

Of the workgroups of 128 rows the first ones walk all of their keys and the last ones, whose round would not fill the chip, are cut
into pieces (span_plan).  With more than 512 of them both kinds are in one launch; the sequences at the end are the ones that are cut,
so they are the long ones here.
"""
import math

import pytest
import torch

from span_plan import plan_of, workgroups
from test_gpu_cache_ops import BF, DEV, F32, STEP, Case, _ctx, _i32

NO_WINDOW = {True: 0, False: 10 ** 6}                       # by whether pages are in 4 bits


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    return T


def _planned(c, hint):
    """The case with room for a bound of `hint` on the prefixes."""
    pps = max(c.pps, (hint + c.rows[0] + 15) // 16)
    c.table = torch.cat((c.table, torch.full((c.B, pps - c.pps), -12345, dtype=torch.int32)), 1)
    c.pps, c.hint = pps, hint
    return c


def _lens(B, *last):
    """Short texts and, at the end, the given ones."""
    return [(23 * i + 5) % 71 for i in range(B - len(last))] + list(last)


# name: heads, prefixes, rows, window (None: none), sinks, bounds on the prefixes of two calls, walks whole and cut with the first
LARGE = {
    "both, groups in eights": ((8, 8, 128), _lens(33, 130, 700), STEP(11), None, 0, (1000, 4000), (512, 16)),
    "both, odd groups": ((5, 5, 128), _lens(53, 610, 700), STEP(11), None, 0, (1000, 2000), (512, 18)),
    "both, rows by head, groups in eights": ((16, 8, 128), _lens(17, 40, 700), (130, 1, 4, 130), None, 0, (1000, 4000), (512, 32)),
    "both, rows by head, odd groups": ((10, 5, 128), _lens(27, 333, 700), (130, 1, 4, 130), None, 0, (1000, 2000), (512, 28)),
    "both, window, sinks beyond a page": ((8, 8, 128), _lens(33, 130, 900), STEP(11), 400, 37, (1000, 300), (512, 16)),
    "both, window longer than most": ((5, 5, 128), _lens(53, 1100, 1300), STEP(11), 1000, 3, (1000, 500), (512, 18)),
    "both, window, rows by head": ((16, 8, 128), _lens(17, 40, 1003), (130, 1, 4, 130), 500, 16, (1000, 400), (512, 32)),
    "both, window, rows by head, odd groups": ((10, 5, 128), _lens(27, 800, 1111), (130, 1, 4, 130), 700, 33, (1000, 600), (512, 28)),
    "whole, window": ((32, 4, 128), [1200, 40, 633], STEP(16), 600, 20, (1200, 500), (204, 0)),
    "whole, window, sinks in a page": ((32, 4, 128), [1000, 1100, 0], STEP(16), 607, 5, (1100, 700), (204, 0)),
    "whole, prompts with a window": ((12, 2, 128), [800, 1000, 30, 0, 650], (300, 1, 16, 300), 600, 4, (1000, 600), (180, 0)),
    "cut, window": ((32, 4, 128), [2000, 700], STEP(16), 1500, 33, (2000, 1000), (0, 136)),
    "cut, no window": ((24, 2, 128), [1700, 500], STEP(16), None, 0, (2016, 1500), (0, 104)),
}


def _large(T, four, name):
    heads, Ls, rows, window, sinks, hints, counts = LARGE[name]
    return _planned(Case(T, four, heads, BF, Ls, *rows, NO_WINDOW[four] if window is None else window, sinks, seed=len(name)), hints[0])


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("name", LARGE)
def test_plans_of_the_large_calls(T, four, name):
    heads, Ls, rows, window, sinks, hints, counts = LARGE[name]
    c = _large(T, four, name)
    first = plan_of(c)
    assert first.rows and workgroups(c, first) == counts
    assert (first.splits > 1) == (counts[1] > 0)
    if counts[1]:                                           # the last sequence's walk is longer than a piece
        keys = max(Ls) if window is None else min(max(Ls), window)
        assert keys > 32 * first.per
    second = plan_of(_planned(c, hints[1]))
    assert second.rows                                      # another bound: the same kernel, cut elsewhere or not at all
    if counts[1]:
        assert (second.splits, second.per) != (first.splits, first.per)


@pytest.mark.gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("name", LARGE)
def test_large_calls(T, four, name):
    print(f"large four={four} {name}", flush=True)
    c = _large(T, four, name)
    _planned(c, max(LARGE[name][5]))                        # room for either bound
    c.build()
    for hint in LARGE[name][5]:
        c.hint = hint
        assert plan_of(c).rows
        c.ws.fill_(255)
        c.out.fill_(77.0)
        c.call()
        c.check()
    again = c.call(torch.full_like(c.out, 5.0))
    assert torch.equal(again, c.out)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("name", ["both, groups in eights", "both, rows by head, odd groups", "cut, no window"])
def test_invalid_lengths_and_pages_in_large_calls(T, four, name):
    """The first sequence is walked whole where there are such, the last one in pieces."""
    print(f"invalid four={four} {name}", flush=True)
    c = _large(T, four, name).build()
    n, nc = c.B, c.rows[0]
    pools = [c.pool] if four else [c.kp, c.vp]
    before = [p.clone() for p in pools]
    c.len[0], c.len[n - 1] = -1, c.pps * 16 - nc + 1
    c.call()
    c.check(skip=(0, n - 1))
    assert torch.isnan(c.out[0]).all() and torch.isnan(c.out[n - 1]).all()
    if not four:
        for b in (0, n - 1):
            used = c.ids[b].to(DEV)
            for p, q in zip(pools, before):
                assert torch.equal(torch.nan_to_num(p[used], 7.0), torch.nan_to_num(q[used], 7.0))
    c.len.copy_(_i32(c.Ls))
    c.table_d[0, 0], c.table_d[n - 1, 20] = c.n_pages, -1   # every row sees these pages
    c.call()
    c.check(skip=(0, n - 1))
    assert torch.isnan(c.out[0]).any(-1).all() and torch.isnan(c.out[n - 1]).any(-1).all()
    c.close()


def _few(T, four, seed):
    """One token each, the keys in splits."""
    c = _planned(Case(T, four, (12, 2, 128), BF, [2900, 1203], 1, 0, 1, 1, NO_WINDOW[four], 0, seed=seed), 3000)
    c.table = torch.cat((c.ids.to(torch.int32), c.table[:, c.ids.shape[1]:]), 1)
    return c


def _many(name):
    def make(T, four, seed):
        c = _large(T, four, name)
        c.table = torch.cat((c.ids.to(torch.int32), c.table[:, c.ids.shape[1]:]), 1)
        return c
    return make


PARTIAL = {"few rows": _few, "both": _many("both, groups in eights"), "cut": _many("cut, window")}


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("kind", PARTIAL)
def test_plans_with_partial_results(T, four, kind):
    p = plan_of(PARTIAL[kind](T, four, 1))
    assert p.splits > 1 and p.rows == (kind != "few rows")


@pytest.mark.gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("kind", PARTIAL)
def test_partial_results_on_streams_and_in_captured_calls(T, four, kind):
    """Two calls at once with a workspace each; two captured calls that share one, replayed in turn over changing lengths."""
    print(f"streams four={four} {kind}", flush=True)
    a, b = (PARTIAL[kind](T, four, i).build() for i in (1, 2))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            a.call()
        with torch.cuda.stream(s2):
            b.call()
    a.check()
    b.check()
    b.ws = a.ws
    graphs = []
    for c in (a, b):
        c.out.fill_(3.0)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.call()
    for i in range(4):
        for c, graph in zip((a, b), graphs):
            c.len.copy_(_i32([max(0, L - 37 * i) for L in c.Ls]))
            c.out.fill_(5.0)
            graph.replay()
        got = [c.out.clone() for c in (a, b)]
        torch.cuda.synchronize()
        for c, g in zip((a, b), got):
            eager = c.call(torch.empty_like(c.out))
            torch.cuda.synchronize()
            assert torch.isfinite(g).all() and torch.equal(g, eager)
    a.close()
    b.close()


# ---------------------------------------------------------------- layers, rows that are not aligned, head sizes
SMALL = {"one token": ((4, 2, 128), [40, 100], (1, 0, 1, 1)), "step": ((12, 2, 128), [40, 33], STEP(5)),
         "large": ((24, 2, 128), [1700, 500], STEP(16))}


@pytest.mark.gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", SMALL)
def test_another_layer(T, four, dtype, kind):
    """Layer 1 of three; the pages of the other two are as they were."""
    heads, Ls, rows = SMALL[kind]
    if dtype == F32 and kind == "large":
        Ls, rows = [170, 50], STEP(4)
    print(f"layer four={four} {dtype} {kind}", flush=True)
    c = Case(T, four, heads, dtype, Ls, *rows, 0 if four else 10 ** 6, 0, seed=11).build()
    one = [c.pool] if four else [c.kp, c.vp]
    pools = [torch.stack((torch.full_like(p, 3), p, torch.full_like(p, 5))) for p in one]
    at = [p.data_ptr() for p in pools] + [c.table_d.data_ptr()]
    kv = (T.tidar_kv4_cache if four else T.tidar_kv_cache)(*at, c.pps, c.n_pages)
    ctx = _ctx(T, heads, dtype, c.B, layers=3)
    fn = T.tidar_kv4_attention if four else T.tidar_window_attention
    c.out.fill_(77.0)
    fn(ctx, kv, 1, c.B, c.len, c.qd, c.kd, c.vd, *c.rows, c.window, c.sinks, c.out, c.hint, c.ws)
    c.check()
    for p in pools:
        assert bool((p[0] == 3).all()) and bool((p[2] == 5).all())
    T.tidar_destroy(ctx)
    c.close()


def _shifted(x):
    """The same values, one element behind a 16-byte border."""
    y = torch.empty(x.numel() + 1, dtype=x.dtype, device=x.device)[1:].view(x.shape)
    y.copy_(x)
    assert y.is_contiguous() and y.data_ptr() % 16 == x.element_size()
    return y


@pytest.mark.gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", SMALL)
def test_new_rows_anywhere_in_memory(T, four, dtype, kind):
    heads, Ls, rows = SMALL[kind]
    if dtype == F32 and kind == "large":
        Ls, rows = [170, 50], STEP(4)
    print(f"shifted four={four} {dtype} {kind}", flush=True)
    c = Case(T, four, heads, dtype, Ls, *rows, 0 if four else 10 ** 6, 0, seed=12).build()
    if c.kd.numel():
        c.kd, c.vd = _shifted(c.kd), _shifted(c.vd)
    c.call()
    c.check()
    if not four:                                            # the causal rows' K/V are in the cache
        kp, vp = c.kp.cpu(), c.vp.cpu()
        for b, L in enumerate(Ls):
            for i in range(rows[0]):
                page, slot = int(c.ids[b, (L + i) // 16]), (L + i) % 16
                assert torch.equal(kp[page, :, slot, :], c.kn[b, i]) and torch.equal(vp[page, :, :, slot], c.vn[b, i])
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads,dtype", [((4, 2, 128), BF), ((4, 2, 128), F32), ((2, 2, 96), F32)])
def test_rows_in_4_bits_from_anywhere_in_memory(T, heads, dtype):
    n_kv, hd = heads[1:]
    ctx = _ctx(T, heads, dtype, 1)
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn(37, n_kv, hd, generator=g).to(dtype).to(DEV) for _ in range(2))
    slots = _i32(torch.randperm(80, generator=g)[:37].tolist())
    pools, outs = [], []
    for shift in (False, True):
        pools.append(torch.zeros(5, n_kv, 544 * ((hd + 31) // 32), dtype=torch.uint8, device=DEV))
        kv = T.tidar_kv4_cache(pools[-1].data_ptr(), None, 0, 5)
        ks, vs = (_shifted(k), _shifted(v)) if shift else (k, v)
        T.tidar_kv4_store(ctx, kv, 0, 37, slots, ks, vs)
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        if shift:
            ko, vo = _shifted(ko.zero_()), _shifted(vo.zero_())
        T.tidar_kv4_load(ctx, kv, 0, 37, slots, ko, vo)
        outs.append((ko, vo))
    T.tidar_destroy(ctx)
    assert torch.equal(*pools) and int(pools[0].count_nonzero())
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("heads", [(2, 2, 96), (8, 2, 96), (4, 2, 64), (2, 2, 72), (4, 4, 36)])
def test_head_sizes_between_the_tiles(T, four, heads):
    for rows in ((1, 0, 1, 1), STEP(3), (37, 1, 8, 37)):
        for Ls, window, sinks in (([0], 1, 0), ([15, 47], 20, 3), ([200], 10 ** 6, 0)):
            print(f"heads four={four} {heads} rows={rows} L={Ls}", flush=True)
            c = Case(T, four, heads, F32, Ls, *rows, window, sinks, seed=13).build()
            c.call()
            c.check()
            c.close()
