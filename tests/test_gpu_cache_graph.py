"""A serving step around the 4-bit cache as one captured call: pages from the free list, new rows into them, attention over them."""
import pytest
import torch

import cache_util as U
from test_gpu_cache_ops import BF, DEV, _ctx, _i32

pytestmark = pytest.mark.gpu


def test_tables_rows_and_attention_in_one_captured_step():
    """Replayed over changing lengths, pages and rows, with eager work in between; each replay against the same calls made eagerly from
    the same state and, the last one, against the definition."""
    import paper_2511_08923_amd as T
    heads, B, pps, n_pages = (12, 2, 128), 3, 12, 40
    n_q, n_kv, hd = heads
    n, g = 4, torch.Generator().manual_seed(3)
    ctx = _ctx(T, heads, BF, B)
    rnd = lambda *s: torch.randn(*s, generator=g).to(BF)
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device=DEV)
    pool, table = torch.zeros(n_pages, n_kv, 2176, dtype=torch.uint8, device=DEV), i32(B, pps)
    kv = T.tidar_kv4_cache(pool.data_ptr(), table.data_ptr(), pps, n_pages)
    P, new, held, free = _i32([0] * B), _i32([n] * B), _i32([0] * B), i32(6)
    start, slots, now, granted, taken = i32(B + 1), i32(B * n + 3), i32(B), i32(B), i32(1)
    k, v = torch.zeros(B * n + 3, n_kv, hd, dtype=BF, device=DEV), torch.zeros(B * n + 3, n_kv, hd, dtype=BF, device=DEV)
    k_held, v_held = torch.zeros_like(k), torch.zeros_like(v)
    q, out = torch.zeros(B, n, n_q, hd, dtype=BF, device=DEV), torch.zeros(B, n, n_q, hd, dtype=BF, device=DEV)
    ws = torch.empty(T.tidar_attention_workspace_bytes(ctx, B, n, 0, 1, 100), dtype=torch.uint8, device=DEV)

    def step():
        T.tidar_table_extend(ctx, B, P, new, held, free, 6, table, n_pages, start, slots, now, granted, taken)
        T.tidar_kv4_store(ctx, kv, 0, B * n + 3, slots, k, v)
        T.tidar_kv4_load(ctx, kv, 0, B * n + 3, slots, k_held, v_held)
        T.tidar_kv4_attention(ctx, kv, 0, B, P, q, None, None, n, 0, 1, 1, 0, 0, out, 100, ws)

    state = (pool, table, start, slots, now, granted, taken, k_held, v_held, out)
    step()                                                  # (lengths and table as they are: nothing here is read later)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    pool.zero_()
    table.fill_(-7)
    lens, used, order = [0] * B, 0, torch.randperm(n_pages, generator=g).tolist()
    text = [(torch.empty(0, n_kv, hd, dtype=BF), torch.empty(0, n_kv, hd, dtype=BF)) for _ in range(B)]
    for i in range(7):
        counts = [n, n, n] if i % 3 else [n, 0, n]          # a sequence without new rows now and then: its attention reads what it has
        P.copy_(_i32(lens))
        new.copy_(_i32(counts))
        held.copy_(_i32([-(-L // 16) for L in lens]))
        free.copy_(_i32(order[used:used + 6]))
        rows_k, rows_v, rows_q = rnd(B * n + 3, n_kv, hd), rnd(B * n + 3, n_kv, hd), rnd(B, n, n_q, hd)
        for d, h in ((k, rows_k), (v, rows_v), (q, rows_q)):
            d.copy_(h)
        before = [t.clone() for t in state]
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in state]
        for t, b in zip(state, before):
            t.copy_(b)
        step()
        torch.cuda.synchronize()
        for t, x in zip(state[:-1], got):
            assert torch.equal(t, x)
        assert granted.tolist() == [1] * B
        used += int(taken)
        s = start.tolist()
        for b in range(B):
            if counts[b]:
                assert torch.equal(out[b], got[-1][b])
                text[b] = tuple(torch.cat((t, r[s[b]:s[b + 1]])) for t, r in zip(text[b], (rows_k, rows_v)))
                kk, vv = U.fake4(text[b][0]), U.fake4(text[b][1])
                want, size = U.attention(rows_q[b].double(), kk, vv, U.mask(lens[b], n, 0, 1, 1, 0, 0))
                off = (out[b].cpu().double() - want).abs() - 2.0 ** -8 * (1.25 * (size + want.abs()) + want.abs())
                assert float(off.max()) <= 0, (i, b, float(off.max()))
            lens[b] += counts[b]
    T.tidar_destroy(ctx)
