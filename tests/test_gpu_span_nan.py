"""A key that is not a number and that a row sees makes the row one, also where a wave, a key split or a piece of a walk sees
nothing else for it: the parts of a row's softmax that are joined then include one without a largest score, whose sums are NaN."""
import math

import pytest
import torch

from span_plan import plan_of, workgroups
from test_gpu_cache_ops import BF, F32, STEP, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    assert torch.cuda.is_available()
    return T


def _check(c):
    c.build()
    c.call()
    c.check()
    c.close()


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("heads,dtype", [((4, 2, 128), BF), ((4, 2, 128), F32), ((4, 4, 32), F32), ((40, 1, 128), BF)])
@pytest.mark.parametrize("L", [0, 32, 64, 96, 128, 224, 256])
def test_the_new_row_alone_with_its_wave(T, four, heads, dtype, L):
    """Iterations of 32 keys, the waves take turns: the new row, at a multiple of 32, is the only key of its wave."""
    print(f"nan new row four={four} {heads} {dtype} L={L}", flush=True)
    c = Case(T, four, heads, dtype, [L, L + 1], 1, 0, 1, 1, 0 if four else 10 ** 6, 0, seed=L)
    c.kn[0, 0, 0, :] = math.nan                             # one kv head of the first sequence
    assert not plan_of(c).rows
    want, _ = c.want(0)
    group = heads[0] // heads[1]
    assert torch.isnan(want[:, :group]).all() and torch.isfinite(want[:, group:]).all()
    _check(c)


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_wave_with_a_sink_and_the_window_s_first_key(T, four, dtype):
    """Sink 0 and the one key of the window's first page are an iteration: both NaN, or one of them beside a finite one."""
    heads = (4, 2, 128) if dtype == BF else (4, 4, 32)
    L, window = 200, 58                                     # the row at 200 sees 143 .. 200; 143 is the last of page 8
    for bad in ((0, 143), (0,), (143,), (144,), tuple(range(144, 176))):
        print(f"nan four={four} {dtype} keys {bad[:2]}", flush=True)
        c = Case(T, four, heads, dtype, [L, 77], 1, 0, 1, 1, window, 1, seed=5)
        for p in bad:
            c.k[0][p] = math.nan
        assert torch.isnan(c.want(0)[0]).all()
        _check(c)


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_key_splits_of_nothing_else(T, four, dtype):
    """Every key but the new row's is NaN: whole key splits see nothing but them, the last one ends with a finite key."""
    heads, L = (8, 2, 128), 2016
    c = Case(T, four, heads, dtype, [L, 45], 1, 0, 1, 1, 0 if four else 10 ** 6, 0, seed=6)
    p = plan_of(c)
    assert p.splits > 2 and not p.rows
    print(f"nan splits four={four} {dtype} splits={p.splits}", flush=True)
    c.k[0][:, 0] = math.nan
    _check(c)
    c = Case(T, four, heads, dtype, [L, 45], 1, 0, 1, 1, 0 if four else 10 ** 6, 0, seed=7)
    per = -(-(L // 32 + 1) // plan_of(c).splits)            # and the iterations of one split alone
    c.k[0][32 * per:64 * per, 1] = math.nan
    assert torch.isnan(c.want(0)[0][:, 4:]).all() and torch.isfinite(c.want(0)[0][:, :4]).all()
    _check(c)


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("piece", [0, 1])
def test_pieces_of_a_cut_walk_of_nothing_else(T, four, piece):
    """128 rows to a workgroup: the NaN keys are the whole of one piece of the walk."""
    c = Case(T, four, (32, 4, 128), BF, [2016, 300], *STEP(16), 0 if four else 10 ** 6, 0, seed=8)
    p = plan_of(c)
    assert p.rows and p.splits > 2 and workgroups(c, p)[1] > 0 and 64 * p.per <= 2016
    print(f"nan pieces four={four} per={p.per} splits={p.splits}", flush=True)
    c.k[0][32 * p.per * piece:32 * p.per * (piece + 1), 2] = math.nan
    want = c.want(0)[0]
    assert torch.isnan(want[:, 16:24]).all() and torch.isfinite(want[:, :16]).all()
    _check(c)
