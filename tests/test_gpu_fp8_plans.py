"""8-bit products by the kernel, the tiles and the splits of K that a call gets: every case names its plan, and the plan is checked on the host.
Tolerances: those of test_gpu_fp8."""
import math

import pytest
import torch

from fp8_plan import fp8_plan, kind, needs
from test_gpu_fp8 import BF, DEV, F32, _check, _ctx, _held, _pack, _spread

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    assert torch.cuda.is_available()
    return T


def _call(T, ctx, a, w8, n, ws, out):
    m = a.shape[0]
    buf = torch.full((m * n + 512,), -77.0, dtype=out, device=DEV)
    T.tidar_fp8_gemm(ctx, a, w8, buf[256:256 + m * n].view(m, n), n, ws)
    torch.cuda.synchronize()
    assert bool((buf[:256] == -77).all()) and bool((buf[256 + m * n:] == -77).all())
    return buf[256:256 + m * n].view(m, n).cpu()


def test_fewer_rows_in_one_workspace(T):
    """Sized for a step's 272 rows, calls of fewer, of which some are split where the step is not; what lies behind it stays as it is."""
    n, k = 4096, 4096
    g = torch.Generator().manual_seed(5)
    a, w = torch.randn(272, k, generator=g).to(BF), torch.randn(n, k, generator=g).to(BF)
    w8, ctx, size = _pack(T, w), _ctx(T, BF), T.tidar_fp8_gemm_workspace_bytes(272, n, k)
    ws = torch.full((size + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
    ha, cols = _held(a), torch.randperm(n, generator=g)[:300]
    hw, splits = _held(w[cols]), set()
    for m in (272, 256, 200, 128, 100, 64, 17, 16, 5, 1, 272):
        print(f"fewer rows {m}", flush=True)
        got = _call(T, ctx, a[:m].to(DEV), w8, n, ws[:size], BF)
        _check(got[:, cols], ha[:m], hw, BF)
        assert bool((ws[size:] == 0xa5).all())
        splits.add(fp8_plan(T, m, n, k).splits)
    assert len(splits) > 1
    T.tidar_destroy(ctx)


# Every wave tile (row tiles, column tiles) of the many-row kernel, with and without passes of one row tile less, K whole and split: row counts that end
# inside a tile of 64, columns inside one of 128, a last block of K that is not whole
PLANS = {
    (728, 1200, 960): (1, 2, False, 1), (563, 1120, 3040): (1, 2, False, 3), (1587, 2528, 928): (1, 4, False, 1), (391, 2960, 7616): (1, 4, False, 3),
    (1370, 1472, 928): (2, 2, False, 1), (1093, 560, 5984): (2, 2, False, 4), (1667, 1200, 928): (2, 2, True, 1), (781, 1168, 4896): (2, 2, True, 3),
    (2136, 3648, 960): (2, 4, False, 1), (2125, 1264, 5728): (2, 4, False, 3), (2320, 3312, 928): (2, 4, True, 1), (794, 2800, 5472): (2, 4, True, 3),
    (2447, 1568, 960): (3, 2, False, 1), (1146, 528, 6880): (3, 2, False, 8), (2506, 1632, 928): (3, 2, True, 1), (1358, 416, 7232): (3, 2, True, 8),
    (3010, 2768, 928): (3, 4, False, 1), (2243, 1312, 8736): (3, 4, False, 3), (2920, 2848, 928): (3, 4, True, 1), (1808, 1296, 10080): (3, 4, True, 4),
    (2531, 2352, 928): (4, 2, False, 1), (1515, 1360, 4960): (4, 2, False, 3), (2181, 2736, 928): (4, 2, True, 1), (1557, 1328, 4896): (4, 2, True, 3),
    (3807, 3248, 928): (4, 4, False, 1), (3266, 1168, 8800): (4, 4, False, 3), (2313, 4928, 928): (4, 4, True, 1), (2357, 1680, 9024): (4, 4, True, 3),
    # a step's rows and a prompt's through the projections of the larger model
    (272, 4096, 12288): (3, 2, True, 4), (272, 24576, 4096): (3, 4, True, 1), (2064, 24576, 4096): (4, 4, True, 1), (2064, 4096, 12288): (3, 4, False, 1),
}
SMALL = [(563, 1120, 3040), (1146, 528, 6880), (1587, 2528, 928), (2313, 4928, 928)]           # split into 3 and 8, and not


def _inputs(m, n, k, dtype):
    g = torch.Generator().manual_seed(m + n + k)
    return _spread(g, m, k, dtype, 3).to(DEV), _spread(g, n, k, dtype, 3).to(DEV)


def _need(T, m, n, k):
    """A workspace of what the call itself needs, and a guard behind it."""
    size = needs(T, m, n, k)
    ws = torch.full((size + 4096,), 0xff, dtype=torch.uint8, device=DEV)
    return ws[:size], ws[size:]


@pytest.mark.parametrize("shape", list(PLANS))
@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
def test_products(T, shape, dtype, out):
    m, n, k = shape
    assert kind(T, m, n, k) == PLANS[shape]
    print(f"plan {PLANS[shape]}: {m} x {n} x {k} {dtype} {out}", flush=True)
    (a, w), (ws, guard), ctx = _inputs(m, n, k, dtype), _need(T, m, n, k), _ctx(T, dtype)
    got = _call(T, ctx, a, _pack(T, w), n, ws, out)
    T.tidar_destroy(ctx)
    assert bool((guard == 0xff).all())
    _check(got.to(DEV), _held(a), _held(w), out)


@pytest.mark.parametrize("m,k,n,plan", [(1120, 1120, 1040, (1, 2, False, 1)), (2080, 2080, 1552, (2, 2, True, 1)), (3104, 3104, 2576, (3, 4, True, 1))])
@pytest.mark.parametrize("out", [BF, F32])
def test_held_values_exactly(T, m, k, n, plan, out):
    """Against the unit matrix every held value comes out alone, as weights and as activations."""
    assert kind(T, m, n, k) == plan
    g = torch.Generator().manual_seed(n)
    w = _spread(g, n, k, BF).to(DEV)
    ws, _ = _need(T, m, n, k)
    ctx = _ctx(T, BF)
    got = _call(T, ctx, torch.eye(k, dtype=BF, device=DEV), _pack(T, w), n, ws, out)
    T.tidar_destroy(ctx)
    assert torch.equal(got.to(DEV).double(), _held(w).T)


@pytest.mark.parametrize("shape", SMALL)
@pytest.mark.parametrize("out", [BF, F32])
def test_blocks_that_are_not_finite(T, shape, out):
    """Infinities and NaN, in the first and the last row and column among others, make NaN of their rows and columns and of nothing else."""
    m, n, k = shape
    a, w = _inputs(m, n, k, BF)
    rows, cols = [0, m // 2, m - 1], [0, n // 2 + 1, n - 1]
    for r, v in zip(rows, (math.inf, math.nan, -math.inf)):
        a[r, (r * 37) % k] = v
    for c, v in zip(cols, (math.nan, math.inf, -math.inf)):
        w[c, k - 1 - (c * 13) % k] = v
    ws, _ = _need(T, m, n, k)
    ctx = _ctx(T, BF)
    got = _call(T, ctx, a, _pack(T, w), n, ws, out).to(DEV)
    T.tidar_destroy(ctx)
    odd = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    odd[rows], odd[:, cols] = True, True
    assert torch.equal(torch.isnan(got), odd)
    r, c = [x for x in range(m) if x not in rows], [x for x in range(n) if x not in cols]
    _check(got[r][:, c], _held(a[r]), _held(w[c]), out)


@pytest.mark.parametrize("shape", SMALL)
@pytest.mark.parametrize("out", [BF, F32])
def test_streams_captured_calls_and_the_same_bits(T, shape, out):
    """Two calls at once with a workspace each, one call captured and replayed over changing inputs, every result bit for bit the eager one's."""
    m, n, k = shape
    print(f"streams {shape} {out}", flush=True)
    g = torch.Generator().manual_seed(m)
    w8, ctx = _pack(T, torch.randn(n, k, generator=g).to(BF)), _ctx(T, BF)
    a = [torch.randn(m, k, generator=g).to(BF).to(DEV) for _ in range(4)]
    wss = [_need(T, m, n, k) for _ in range(3)]
    want = [_call(T, ctx, x, w8, n, wss[0][0], out).to(DEV) for x in a]
    outs, streams = [torch.zeros(m, n, dtype=out, device=DEV) for _ in range(2)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            for j in (2, 3, i):
                T.tidar_fp8_gemm(ctx, a[j], w8, outs[i], n, wss[i][0])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i])
    inp, got, graph = a[0].clone(), torch.zeros(m, n, dtype=out, device=DEV), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.tidar_fp8_gemm(ctx, inp, w8, got, n, wss[2][0])
    for i in (1, 2, 3, 0):
        inp.copy_(a[i])
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want[i])
        T.tidar_fp8_gemm(ctx, a[3], w8, outs[0], n, wss[0][0])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[3])
    T.tidar_destroy(ctx)


def test_graphs_that_share_a_workspace(T):
    """Captured products, K split and not, of many rows and few, one after another in one workspace, with an eager one in between."""
    g = torch.Generator().manual_seed(6)
    shapes = SMALL + [(40, 272, 640), (1, 528, 1056)]
    assert [kind(T, *s) if s not in PLANS else PLANS[s][3] for s in shapes] == [3, 8, 1, 1, "few", "own"]
    ctx = _ctx(T, BF)
    ws = torch.full((max(needs(T, *s) for s in shapes),), 0xff, dtype=torch.uint8, device=DEV)
    calls = []
    for m, n, k in shapes:
        a, w8 = torch.randn(m, k, generator=g).to(BF).to(DEV), _pack(T, torch.randn(n, k, generator=g).to(BF))
        out, graph = torch.zeros(m, n, dtype=BF, device=DEV), torch.cuda.CUDAGraph()
        T.tidar_fp8_gemm(ctx, a, w8, out, n, torch.empty_like(ws))
        torch.cuda.synchronize()
        calls.append((a, w8, out, n, out.clone(), graph))
        with torch.cuda.graph(graph):
            T.tidar_fp8_gemm(ctx, a, w8, out, n, ws)
    for order in ((0, 1, 2, 3, 4, 5), (5, 3, 4, 2, 1, 0), (2, 0, 5, 3, 1, 4)):
        for c in calls:
            c[2].zero_()
        for i in order[:5]:
            calls[i][5].replay()
        a, w8, out, n, _, _ = calls[order[5]]
        T.tidar_fp8_gemm(ctx, a, w8, out, n, ws)
        torch.cuda.synchronize()
        for c in calls:
            assert torch.equal(c[2], c[4])
    T.tidar_destroy(ctx)


@pytest.mark.parametrize("shape", SMALL)
def test_rows_do_not_depend_on_their_neighbours(T, shape):
    """Rows beside such that are NaN, and with others: the same bits."""
    m, n, k = shape
    a, w = _inputs(m, n, k, BF)
    b = torch.flip(a, (1,)) * 3
    keep = [1, 2, m // 2, m - 2]
    b[keep], b[0], b[m - 1] = a[keep], math.nan, math.nan
    w8, ctx, (ws, _) = _pack(T, w), _ctx(T, BF), _need(T, m, n, k)
    x, y = (_call(T, ctx, v, w8, n, ws, BF) for v in (a, b))
    T.tidar_destroy(ctx)
    assert torch.equal(x[keep], y[keep])
