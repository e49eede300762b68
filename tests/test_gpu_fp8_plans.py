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
