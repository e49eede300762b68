"""Attention over trees by the kernel and the cut that a call gets: every case names its plan, and the plan is checked on the host (a bound on the
prefixes that is far above them makes a small call take the plan of a large one).  Tolerances: those of test_gpu_tree."""
import math

import pytest
import torch

import tree_util as V
from test_gpu_tree import BF, DEV, F32, HEADS, Case
from tree_plans import kind, tree_plan

pytestmark = pytest.mark.gpu
HEADS = {**HEADS, "shared": (32, 1, 128), "wide group": (40, 1, 128)}

# name: heads, prefixes, rows of the trees, bounds on the prefixes with exact and with 4-bit pages, plan
CALLS = {
    "whole": ("8b", [130, 40] * 16, [40, 64, 1, 33] * 8, (1500, 1600), "many"),
    "cut": ("gqa", [333, 90], [200, 256], (4000, 4000), "many, cut"),
    "some cut": ("8b", [40, 30] * 32 + [500, 400, 300, 200], [54, 7, 30, 21] * 17, (4000, 4000), "many, some cut"),
    "one head": ("shared", [700, 20, 300, 0, 1100], [256, 31, 256, 100, 255], (4000, 4000), "many, cut"),
    "one head of many": ("wide group", [400, 0, 90], [256, 256, 17], (4000, 4000), "many, cut"),
}


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    assert torch.cuda.is_available()
    return T


def _case(T, four, name, **more):
    heads, Ls, sizes, hints, plan = CALLS[name]
    print(f"{name} four={four}", flush=True)
    c = Case(T, four, HEADS[heads], BF, Ls, sizes, seed=len(name), **more)
    c.hint = hints[four]
    c.pps = -(-c.hint // 16) + 1
    c.n_pages = c.B * (-(-max(Ls) // 16) + 1) + 2                            # (pages for the prefixes that there are)
    used = -(-max(Ls) // 16) + 1
    ids = torch.randperm(c.n_pages, generator=torch.Generator().manual_seed(1))[:c.B * used].view(c.B, used)
    c.ids = torch.cat((ids, torch.full((c.B, c.pps - used), -99)), 1)
    assert kind(tree_plan(c)) == plan, kind(tree_plan(c))
    return c


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("name", list(CALLS))
def test_trees(T, four, name):
    c = _case(T, four, name).build()
    c.call()
    c.check()
    first = c.out.clone()
    c.ws.fill_(255)
    c.out.fill_(77)
    c.call()
    torch.cuda.synchronize()
    assert torch.equal(first, c.out)                                         # the same bits again
    c.close()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("name", ["whole", "cut", "some cut"])
def test_masks_that_are_no_trees(T, four, name):
    """Random bits, rows that see nothing of their tree, all of it, or (without a prefix) no key at all."""
    _, Ls, sizes, _, _ = CALLS[name]
    g = torch.Generator().manual_seed(3)
    see = [torch.rand(n, n, generator=g) < 0.4 for n in sizes]
    for s in see:
        s[0], s[-1] = False, False
        s[len(s) // 2] = True
    c = _case(T, four, name, see=see).build()
    b = c.B - 1
    c.Ls = list(Ls)
    c.Ls[b], c.len[b], c.k[b], c.v[b] = 0, 0, c.k[b][:0], c.v[b][:0]         # no prefix
    c.call()
    c.check()
    assert float(c.out[c.start[b]].abs().max()) == 0
    if max(sizes) < 250:
        c.anc |= torch.tensor([0] * 7 + [1 << 30], dtype=torch.int32, device=DEV)        # a row that is not there
        c.out.fill_(77)
        c.call()
        c.check()
    c.close()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("name", ["whole", "cut", "some cut"])
def test_what_a_row_does_not_see_has_no_influence(T, four, name):
    """Infinities and NaN in rows of the first and the last tree, and in exact pages: only rows that see them are touched."""
    c = _case(T, four, name, wide=6)
    for b in (0, c.B - 1):
        at = c.start[b] + c.sizes[b] - 5
        c.vn[at, 0, 3], c.vn[at - 1, -1, 0], c.kn[at - 2, 0, 1] = math.inf, math.nan, math.nan
        c.vn[at - 4, 0, 2] = -math.inf
    if not four:
        c.v[1][7, 0, 1] = math.inf
    c.build().call()
    c.check()
    c.close()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("name", ["whole", "cut", "some cut"])
@pytest.mark.parametrize("by", [1, 3])
def test_rows_at_any_element(T, four, name, by):
    """The tree's K/V from any element of the caller's memory on."""
    c = _case(T, four, name).build()
    c.call()
    c.check()
    first = c.out.clone()
    buf = torch.full((2, c.kd.numel() + 8), 77.0, dtype=BF, device=DEV)
    for i, x in enumerate((c.kd, c.vd)):
        buf[i, by:by + x.numel()] = x.flatten()
    c.kd, c.vd = (buf[i, by:by + c.kd.numel()].view(c.kd.shape) for i in range(2))
    c.out.fill_(77)
    c.call()
    torch.cuda.synchronize()
    assert torch.equal(c.out, first)
    c.close()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("name", ["whole", "cut", "some cut"])
def test_sequences_that_are_not_valid(T, four, name):
    """A length or a page id that is not valid makes NaN of its sequence, and of no other."""
    c = _case(T, four, name).build()
    good = c.call().clone()
    c.check()
    for b in (0, c.B - 1):
        for length, page in ((-4, None), (c.pps * 16 + 1, None), (c.Ls[b], c.n_pages), (c.Ls[b], -1)):
            keep = c.table_d.clone()
            c.len[b] = length
            if page is not None:
                c.table_d[b, 1] = page
            c.out.fill_(77)
            c.call()
            torch.cuda.synchronize()
            s, e = c.start[b], c.start[b + 1]
            assert bool(torch.isnan(c.out[s:e]).all()), (b, length, page)
            assert torch.equal(c.out[:s], good[:s]) and torch.equal(c.out[e:], good[e:]), (b, length, page)
            c.len[b] = c.Ls[b]
            c.table_d.copy_(keep)
    c.close()


# the largest bound of few rows' calls beside the least of many rows': both kernels give the same within rounding
@pytest.mark.parametrize("four", [False, True])
def test_both_kernels(T, four):
    outs = []
    for hint, plan in ((300, "few"), (8000, "many")):
        c = Case(T, four, HEADS["gqa"], BF, [300, 211], [256, 190], seed=9)
        c.hint, c.pps = hint, 501
        c.n_pages = 60
        c.ids = torch.cat((torch.randperm(60, generator=torch.Generator().manual_seed(1))[:40].view(2, 20), torch.full((2, 481), -99)), 1)
        assert kind(tree_plan(c)).startswith(plan)
        c.build().call()
        c.check()
        outs.append(c.out.clone())
        c.close()
    want = [c.want(b) for b in range(2)]
    for b, (w, size) in enumerate(want):
        s, e = c.start[b], c.start[b + 1]
        assert bool(((outs[0][s:e] - outs[1][s:e]).abs().cpu().double() <= 2 * c.tolerance(w, size)).all())
