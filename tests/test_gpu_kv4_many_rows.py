"""Rows into 4-bit pages and back where a call has more than 2^32 lanes' work: a launch has fewer."""
import pytest
import torch

import cache_util as U
from test_gpu_cache_ops import DEV, F32, _ctx, _rows

pytestmark = pytest.mark.gpu


def test_rows_beyond_one_launch():
    """2^27 + 37 rows of 8 heads of 2 values (32 lanes a row), nearly all of them padding: the first, the last and those around powers
    of two are stored and read back, every other row reads 0."""
    import paper_2511_08923_amd as T
    heads, n = (8, 8, 2), (1 << 27) + 37
    n_kv, hd = heads[1:]
    print(f"kv4 rows n={n}", flush=True)
    ctx = _ctx(T, heads, F32, 1)
    real = [0, 15, 16, (1 << 26) - 17, (1 << 26) - 1, 1 << 26, (1 << 26) + 1, (1 << 27) - 33, (1 << 27) - 1, 1 << 27, n - 1]
    real_d = torch.tensor(real, device=DEV)
    slots = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    slots[real_d] = torch.arange(len(real), dtype=torch.int32, device=DEV) * 5 + 2
    k, v = torch.zeros(n, n_kv, hd, device=DEV), torch.zeros(n, n_kv, hd, device=DEV)
    kr, vr = _rows(len(real), n_kv, hd, 3, F32), _rows(len(real), n_kv, hd, 4, F32)
    k[real_d], v[real_d] = kr.to(DEV), vr.to(DEV)
    pool = torch.zeros(4, n_kv, 544, dtype=torch.uint8, device=DEV)
    kv = T.tidar_kv4_cache(pool.data_ptr(), None, 0, 4)
    T.tidar_kv4_store(ctx, kv, 0, n, slots, k, v)
    want = torch.zeros(4, n_kv, 544, dtype=torch.uint8)
    U.put_rows(want, hd, [5 * i + 2 for i in range(len(real))], kr, vr)
    assert torch.equal(pool.cpu(), want)
    k.fill_(9.0)
    v.fill_(9.0)
    T.tidar_kv4_load(ctx, kv, 0, n, slots, k, v)
    T.tidar_destroy(ctx)
    for got, x in ((k, kr), (v, vr)):
        held = U.fake4(x)
        assert torch.equal(got[real_d].cpu().double(), held)
        assert int(torch.count_nonzero(got)) == int(torch.count_nonzero(held))
