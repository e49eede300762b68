"""The operators around the paged cache on the GPU, against their definitions in 64 bits (cache_util).

Tolerances of the attention.  bf16: a weight is rounded to bf16 (2^-8 of itself) in numerator and denominator alike, which moves an
output by at most 2^-8 (sum w|v| + |out|); the output's own rounding adds 2^-8 |out|; a quarter of the first covers what fp32 does in
between (scores of 128 products, the exponential: below 2^-10 of a weight for scores up to 100).  fp32: a score is a sum of hd
products, off by at most hd 2^-24 of sum |q k| / sqrt(hd) (below 8 sqrt(hd) here), which a weight takes over; the sums over the
keys add 2^-24 each per key, the exponential and the division a few more.
"""
import math

import pytest
import torch

import cache_util as U
import tidar_inputs as TI

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F64 = torch.float64


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    assert torch.cuda.is_available()
    return T


def _ctx(T, heads, dtype, batch, layers=1):
    n_q, n_kv, hd = heads
    code = T.TIDAR_BF16 if dtype == torch.bfloat16 else T.TIDAR_F32
    return T.tidar_create(T.tidar_config(layers, 128, n_q, n_kv, hd, 512, 512, 0, code, 16, 16, batch, 511, 1e4, 1e-6))


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------- page tables
def _extend(T, prefix, new, held, free, table, n_pages, slot_cap):
    B = len(prefix)
    ctx = _ctx(T, (4, 4, 32), torch.float32, B)
    t = _i32(table)
    out = [torch.full((n,), -7, dtype=torch.int32, device=DEV) for n in (B + 1, slot_cap, B, B, 1)]
    P, n, h, fr = _i32(prefix), _i32(new), _i32(held), _i32(free) if free else None
    T.tidar_table_extend(ctx, B, P, n, h, fr, len(free), t, n_pages, *out)
    torch.cuda.synchronize()
    T.tidar_destroy(ctx)
    return [t.tolist()] + [o.tolist() for o in out]


def _check_extend(T, prefix, new, free, table, n_pages, slot_cap, held=None):
    held = [max(0, -(-p // 16)) for p in prefix] if held is None else held
    got = _extend(T, prefix, new, held, free, table, n_pages, slot_cap)
    want = U.extend(prefix, new, held, free, table, n_pages, slot_cap)
    assert got[0] == want[0]
    assert got[1] == want[1]
    assert got[2] == want[2]
    assert got[3] == want[3]
    assert got[4] == want[4]
    assert got[5] == [want[5]]
    return want


@pytest.mark.parametrize("B,prefix,new,pps", [(1, 0, 0, 1), (1, 0, 1, 1), (1, 15, 1, 1), (1, 16, 1, 2), (3, 40, 33, 6), (6, 100, 1, 7),
                                              (255, 60, 20, 6), (257, 60, 20, 6), (2048, 90, 40, 9), (2051, 90, 40, 9), (5000, 20, 5, 2)])
@pytest.mark.parametrize("short", [1.0, 0.6])
def test_table_extend(T, B, prefix, new, pps, short):
    print(f"extend B={B} prefix={prefix} new={new} short={short}", flush=True)
    g = torch.Generator().manual_seed(B + prefix)
    P = torch.randint(0, prefix + 1, (B,), generator=g).tolist() if B > 1 else [prefix]
    n = torch.randint(0, new + 1, (B,), generator=g).tolist() if B > 1 else [new]
    held = [min(pps, -(-p // 16) + (i % 3 == 2)) for i, p in enumerate(P)]              # every third has a page to spare
    need = sum(max(0, -(-(p + m) // 16) - h) for p, m, h in zip(P, n, held))
    n_pages = sum(held) + need + 3
    ids = torch.randperm(n_pages, generator=g).tolist()
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-5] * (pps - h))
        at += h
    free = ids[at:at + int(need * short)]
    want = _check_extend(T, P, n, free, table, n_pages, sum(n) + 5, held)
    if short == 1.0:
        assert want[4] == [1] * B and want[5] == need


def test_table_extend_refuses_single_sequences(T):
    """Lengths and ids that only the device sees: the sequence is refused, its table and slots stay, the others are served."""
    full = [3, 4, 5, -9]
    P = [10, -1, 33, 5, 70, 10, 2 ** 31 - 1, 20, 16, 0, 40]
    n = [20, 4, 40, -3, 1, 2 ** 31 - 1, 2, 3, 2, 16, 0]
    table = [[0, -9, -9, -9], full, full, full, full, full, full, [1, 99, -9, -9], [6, -9, -9, -9], [-9] * 4, [0, 1, 2, -9]]
    want = _check_extend(T, P, n, [7, 8, 9, 10], table, 12, 60)
    assert want[4] == [1, -1, -1, -1, -1, -1, -1, 0, 0, 0, 1]       # the slot map ends in the third sequence's rows
    want = _check_extend(T, P, n, [7, 8, 9, 10], table, 12, 100)
    assert want[4] == [1, -1, -1, -1, -1, -1, -1, -1, 1, 1, 1]
    # pages that do not hold the positions, more pages than the table has, a page to spare that is not valid
    want = _check_extend(T, [17, 3, 3, 3], [2, 2, 2, 20], [7, 8], [[0, 1, 2, 3], [4, 5, 6, 9], full, [10, 77, -9, -9]], 12, 60, [1, 5, -1, 2])
    assert want[4] == [-1, -1, -1, -1] and want[5] == 0
    # ids of the list outside the pool: that sequence alone, its part is used up
    want = _check_extend(T, [0, 0, 0], [16, 20, 16], [7, 12, 8, -1, 9], [[-9] * 4] * 3, 12, 60)
    assert want[4] == [1, -1, -1] and want[5] == 4
    want = _check_extend(T, [0, 0, 0], [16, 16, 16], [7, 12, 8], [[-9] * 4] * 3, 12, 60)
    assert want[4] == [1, -1, 1] and want[5] == 3
    # no list at all; rows that the slot map has no room for
    assert _check_extend(T, [3, 16], [5, 1], [], [[2, -9], [1, -9]], 12, 60)[4] == [1, 0]
    assert _check_extend(T, [0, 0, 0], [16, 20, 0], [7, 1, 8, 9], [[-9] * 4] * 3, 12, 20)[4] == [1, 0, 1]
    assert _check_extend(T, [0], [16], [7], [[-9]], 12, 0)[4] == [0]


def test_table_extend_counts_beyond_31_bits(T):
    """Rows of many sequences add up to more than an int32: the numbering saturates, sequences behind slot_cap get nothing."""
    pps = 1 << 15
    B = 5000
    table = torch.full((B, pps), -1, dtype=torch.int32, device=DEV)
    ctx = _ctx(T, (4, 4, 32), torch.float32, B)
    start, slots, held, now, granted, taken = (torch.zeros(k, dtype=torch.int32, device=DEV) for k in (B + 1, 1000, B, B, B, 1))
    P, n = _i32([0] * B), _i32([pps * 16] * B)
    n[0] = 1000
    free = torch.arange(100, dtype=torch.int32, device=DEV)
    T.tidar_table_extend(ctx, B, P, n, held, free, 100, table, 1 << 20, start, slots, now, granted, taken)
    T.tidar_destroy(ctx)
    rows = (1000 + torch.arange(B, dtype=torch.int64) * pps * 16).clamp(max=2 ** 31 - 1)
    assert start[0] == 0 and torch.equal(start[1:].cpu().long(), rows)
    assert granted.tolist() == [1] + [0] * (B - 1) and taken.tolist() == [63]
    assert slots.tolist() == list(range(1000)) and now.tolist() == [63] + [0] * (B - 1)


# ---------------------------------------------------------------- 4-bit rows
HEADS = {"8b": (32, 8, 128), "gqa": (4, 2, 128), "tiny": (4, 4, 32), "odd": (8, 8, 40), "narrow": (8, 8, 6), "wide": (2, 2, 96)}


def _rows(n, n_kv, hd, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, n_kv, hd, generator=g) * torch.randn(n, n_kv, 1, generator=g).exp()
    # values on and beside the borders of the levels, in every third row
    edge = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0])
    tie = edge[torch.randint(0, 10, (n, n_kv, hd), generator=g)] * torch.sign(torch.randn(n, n_kv, hd, generator=g))
    tie = tie * 2.0 ** torch.randint(-9, 9, (n, n_kv, 1), generator=g)
    x[::3] = tie[::3]
    return x.to(dtype)


@pytest.mark.parametrize("heads,dtype", [("8b", torch.bfloat16), ("gqa", torch.bfloat16), ("gqa", torch.float32), ("tiny", torch.float32),
                                         ("odd", torch.float32), ("narrow", torch.float32), ("wide", torch.float32)])
@pytest.mark.parametrize("n", [1, 3, 4, 37])
def test_kv4_rows_bytes_and_values(T, heads, dtype, n):
    print(f"kv4 rows {heads} {dtype} n={n}", flush=True)
    n_q, n_kv, hd = HEADS[heads]
    ctx = _ctx(T, HEADS[heads], dtype, 1, layers=2)
    n_pages, nb = 5, (hd + 31) // 32
    assert T.tidar_kv4_page_bytes(ctx) == n_kv * 544 * nb
    g = torch.Generator().manual_seed(n)
    slots = torch.randperm(n_pages * 16, generator=g)[:n].tolist()
    if n > 3:
        slots[1], slots[2] = -1, n_pages * 16                                  # neither is stored, both read 0
    k, v = _rows(n, n_kv, hd, 5 + n, dtype), _rows(n, n_kv, hd, 6 + n, dtype)
    before = torch.randint(0, 256, (2, n_pages, n_kv, 544 * nb), generator=g, dtype=torch.uint8)
    pool = before.to(DEV)
    kv = T.tidar_kv4_cache(pool.data_ptr(), None, 0, n_pages)
    sd = _i32(slots)
    T.tidar_kv4_store(ctx, kv, 1, n, sd, k.to(DEV), v.to(DEV))
    want = before.clone()
    U.put_rows(want[1], hd, slots, k, v)
    assert torch.equal(pool.cpu(), want)                                       # the other layer and every other token as they were
    ko, vo = (torch.full((n, n_kv, hd), 9.0, dtype=dtype, device=DEV) for _ in range(2))
    T.tidar_kv4_load(ctx, kv, 1, n, sd, ko, vo)
    T.tidar_destroy(ctx)
    keep = torch.tensor([0 <= s < n_pages * 16 for s in slots]).view(-1, 1, 1)
    for got, x in ((ko, k), (vo, v)):
        assert torch.equal(got.cpu().double(), torch.where(keep, U.fake4(x), torch.tensor(0.0, dtype=F64)))


def test_kv4_rows_extremes(T):
    """Zeros, subnormals, the largest numbers, infinities and NaN; a block that holds one of the last two reads back as NaN."""
    big = torch.finfo(torch.float32).max
    for dtype in (torch.float32, torch.bfloat16):
        heads = (4, 2, 128)
        ctx = _ctx(T, heads, dtype, 1)
        x = torch.zeros(10, 2, 128)
        x[1] = 1e-45
        x[2] = 2.0 ** -126
        x[3] = big if dtype == torch.float32 else 3.3895e38
        x[4, :, ::2] = 2.0 ** 125 * 6.5
        x[5, 0, 3], x[5, 1, 100] = math.nan, math.inf
        x[6, 0, 64:] = -math.inf
        x[7] = torch.randn(2, 128, generator=torch.Generator().manual_seed(1)) * 1e-38
        x[8] = 7 * 2.0 ** -127
        x[9, :, 5] = -0.0
        x = x.to(dtype)
        pool = torch.zeros(1, 2, 2176, dtype=torch.uint8, device=DEV)
        kv = T.tidar_kv4_cache(pool.data_ptr(), None, 0, 1)
        s = _i32(range(10))
        T.tidar_kv4_store(ctx, kv, 0, 10, s, x.to(DEV), x.to(DEV))
        ko, vo = (torch.empty(10, 2, 128, dtype=dtype, device=DEV) for _ in range(2))
        T.tidar_kv4_load(ctx, kv, 0, 10, s, ko, vo)
        want = U.fake4(x)
        assert torch.isnan(want[5, 0, :32]).all() and not torch.isnan(want[5, 0, 32:]).any()
        for got in (ko, vo):
            assert torch.equal(torch.nan_to_num(got.cpu().double(), 77.0), torch.nan_to_num(want, 77.0))
        T.tidar_destroy(ctx)


# ---------------------------------------------------------------- attention
class Case:
    """A pool with stale NaN everywhere that nothing is held, its table with ids that are not valid where nothing may be read, and the
    dense K/V of every sequence as the operator has to see them."""

    def __init__(self, T, four, heads, dtype, Ls, nc, nb, bl, cond0, window, sinks, seed=0, scale=1.0, stale=math.nan):
        self.T, self.four, self.dtype, self.heads = T, four, dtype, heads
        self.rows, self.window, self.sinks, self.Ls = (nc, nb, bl, cond0), window, sinks, Ls
        n_q, n_kv, hd = heads
        B, R, nm = len(Ls), nc + nb * bl, nb * bl
        self.B, self.R = B, R
        g = torch.Generator().manual_seed(seed + 1)
        rnd = lambda *s: torch.randn(*s, generator=g).to(dtype)
        self.pps = (max(Ls) + nc + 15) // 16 + 1
        self.n_pages = B * self.pps + 3
        ids = torch.randperm(self.n_pages, generator=g)[:B * self.pps].view(B, self.pps)
        self.table = torch.full((B, self.pps), -12345, dtype=torch.int32)
        for b, L in enumerate(Ls):
            lo = max(0, L + 1 - window) if window else 0                # the first row's window; rows behind it see no more
            low_mask = L + cond0 + 1 - window if window and nb else lo  # a mask row at its block's first slot, block 0
            lo = max(0, min(lo, low_mask))
            for u in range((L + nc + 15) // 16):
                if 16 * u + 16 > lo or (window and 16 * u < sinks):
                    self.table[b, u] = ids[b, u]
        self.ids = ids
        self.q = rnd(B, R, n_q, hd) * scale
        self.k = [rnd(L, n_kv, hd) for L in Ls]                          # the cached prefix
        self.v = [rnd(L, n_kv, hd) for L in Ls]
        self.kn, self.vn = rnd(B, R, n_kv, hd), rnd(B, R, n_kv, hd)
        self.stale = stale
        self.hint = max(Ls)

    def build(self):
        n_q, n_kv, hd = self.heads
        nc, _, bl, _ = self.rows
        if self.four:
            nb = (hd + 31) // 32
            self.pool = torch.full((self.n_pages, n_kv, 544 * nb), 255, dtype=torch.uint8, device=DEV)       # scales of NaN blocks
            self.ctx = _ctx(self.T, self.heads, self.dtype, self.B)
            self.kv = self.T.tidar_kv4_cache(self.pool.data_ptr(), None, 0, self.n_pages)
            for b, L in enumerate(self.Ls):
                n = L + nc
                at = torch.arange(n)
                slots = (self.ids[b, at // 16] * 16 + at % 16).to(torch.int32).to(DEV)
                k, v = torch.cat((self.k[b], self.kn[b, :nc])).to(DEV), torch.cat((self.v[b], self.vn[b, :nc])).to(DEV)
                self.T.tidar_kv4_store(self.ctx, self.kv, 0, n, slots, k, v)
            torch.cuda.synchronize()
            self.table_d = self.table.to(DEV)
            self.kv = self.T.tidar_kv4_cache(self.pool.data_ptr(), self.table_d.data_ptr(), self.pps, self.n_pages)
            self.kd, self.vd = self.kn[:, nc:].contiguous().to(DEV), self.vn[:, nc:].contiguous().to(DEV)
        else:
            self.ctx = _ctx(self.T, self.heads, self.dtype, self.B)
            kp = torch.full((self.n_pages, n_kv, 16, hd), self.stale, dtype=self.dtype)
            vp = torch.full((self.n_pages, n_kv, hd, 16), self.stale, dtype=self.dtype)
            for b, L in enumerate(self.Ls):
                at = torch.arange(L)
                kp[self.ids[b, at // 16], :, at % 16, :] = self.k[b]
                vp[self.ids[b, at // 16], :, :, at % 16] = self.v[b]
            self.kp, self.vp, self.table_d = kp.to(DEV), vp.to(DEV), self.table.to(DEV)
            self.kv = self.T.tidar_kv_cache(self.kp.data_ptr(), self.vp.data_ptr(), self.table_d.data_ptr(), self.pps, self.n_pages)
            self.kd, self.vd = self.kn.to(DEV), self.vn.to(DEV)
        self.len = _i32(self.Ls)
        self.qd = self.q.to(DEV)
        n = self.T.tidar_attention_workspace_bytes(self.ctx, self.B, *self.rows[:3], self.hint)
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)
        self.out = torch.full(self.q.shape, 77.0, dtype=self.dtype, device=DEV)
        return self

    def call(self, out=None):
        fn = self.T.tidar_kv4_attention if self.four else self.T.tidar_window_attention
        out = self.out if out is None else out
        fn(self.ctx, self.kv, 0, self.B, self.len, self.qd, self.kd, self.vd, *self.rows, self.window, self.sinks, out, self.hint, self.ws)
        return out

    def want(self, b):
        nc, nb, bl, cond0 = self.rows
        L = self.Ls[b]
        k, v = torch.cat((self.k[b], self.kn[b, :nc])).double(), torch.cat((self.v[b], self.vn[b, :nc])).double()
        if self.four:
            k, v = U.fake4(k), U.fake4(v)
        k, v = torch.cat((k, self.kn[b, nc:].double())), torch.cat((v, self.vn[b, nc:].double()))
        see = U.mask(L, nc, nb, bl, cond0, self.window, self.sinks)
        return U.attention(self.q[b].double(), k, v, see)

    def tolerance(self, want, size):
        want = torch.nan_to_num(want, 0.0, 0.0, 0.0)
        if self.dtype == torch.bfloat16:
            return 2.0 ** -8 * (1.25 * (size + want.abs()) + want.abs()) + 1e-30
        hd, keys = self.heads[2], max(self.Ls) + self.R
        return 2.0 ** -24 * (8 * hd * math.sqrt(hd) + keys + 32) * (size + want.abs()) + 1e-30

    def check(self, skip=()):
        torch.cuda.synchronize()
        got = self.out.cpu().double()
        for b in range(self.B):
            if b in skip:
                continue
            want, size = self.want(b)
            fin = torch.isfinite(want)
            assert torch.equal(torch.isnan(got[b]), torch.isnan(want)), (b, int(torch.isnan(got[b]).sum()), int(torch.isnan(want).sum()))
            assert torch.equal(got[b][~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)])
            off = (got[b] - want).abs()[fin] - self.tolerance(want, size)[fin]
            assert off.numel() == 0 or float(off.max()) <= 0, (b, float(off.max()))

    def close(self):
        self.T.tidar_destroy(self.ctx)


def _run(T, *a, **kw):
    c = Case(T, *a, **kw).build()
    c.call()
    c.check()
    return c


BF, F32 = torch.bfloat16, torch.float32
STEP = lambda k: (k, k, k, 1)
GEOM = [("gqa", BF), ("gqa", F32), ("tiny", F32), ("odd", F32), ("narrow", F32)]


@pytest.mark.parametrize("heads,dtype", GEOM)
@pytest.mark.parametrize("rows", [(1, 0, 1, 1), STEP(1), STEP(2), STEP(4), STEP(5), STEP(16), (37, 1, 8, 37), (3, 2, 5, 0)])
def test_kv4_attention(T, heads, dtype, rows):
    for Ls in ([0], [1], [15, 16, 17], [129, 40]):
        for window, sinks in ((0, 0), (1, 0), (16, 0), (17, 3), (40, 20), (1000, 4)):
            print(f"kv4 {heads} {dtype} rows={rows} L={Ls} w={window} t={sinks}", flush=True)
            _run(T, True, HEADS[heads], dtype, Ls, *rows, window, sinks, seed=len(Ls) + window).close()


@pytest.mark.parametrize("heads,dtype", GEOM)
@pytest.mark.parametrize("rows", [(1, 0, 1, 1), STEP(1), STEP(2), STEP(4), STEP(5), STEP(16), (37, 1, 8, 37), (3, 2, 5, 0)])
def test_window_attention(T, heads, dtype, rows):
    nc = rows[0]
    for Ls in ([0], [1], [15, 16, 17], [129, 40]):
        for window, sinks in ((1, 0), (3, 1), (16, 0), (17, 3), (40, 20), (1000, 4), (2 ** 31 - 1, 2 ** 31 - 1)):
            print(f"window {heads} {dtype} rows={rows} L={Ls} w={window} t={sinks}", flush=True)
            c = _run(T, False, HEADS[heads], dtype, Ls, *rows, window, sinks, seed=len(Ls) + window)
            # the causal rows' K/V are in the cache, every other slot as it was
            kp, vp = c.kp.cpu(), c.vp.cpu()
            for b, L in enumerate(Ls):
                at = torch.arange(L + nc)
                pg, sl = c.ids[b, at // 16], at % 16
                assert torch.equal(kp[pg, :, sl, :], torch.cat((c.k[b], c.kn[b, :nc])))
                assert torch.equal(vp[pg, :, :, sl], torch.cat((c.v[b], c.vn[b, :nc])))
                kp[pg, :, sl, :] = math.nan
                vp[pg, :, :, sl] = math.nan
            assert torch.isnan(kp).all() and torch.isnan(vp).all()
            c.close()


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("heads,Ls,rows,window,sinks", [
    ((32, 8, 128), [3000], (1, 0, 1, 1), 700, 4), ((32, 8, 128), [2000, 77, 1301], (1, 0, 1, 1), 0, 0),
    ((12, 2, 128), [1500, 900], STEP(16), 333, 5), ((12, 2, 128), [800], (300, 1, 16, 300), 256, 16),
    ((12, 2, 128), [800], (300, 1, 16, 300), 0, 0), ((20, 1, 128), [500], STEP(3), 64, 1), ((24, 24, 128), [260], STEP(8), 100, 0),
    ((6, 3, 128), [700, 650], STEP(11), 0, 0)])
def test_attention_of_longer_texts(T, four, heads, Ls, rows, window, sinks):
    print(f"long four={four} {heads} {Ls} {rows} {window} {sinks}", flush=True)
    if not four and window == 0:
        window, sinks = 10 ** 6, 0
    _run(T, four, heads, BF, Ls, *rows, window, sinks, seed=3).close()


def _room(c, pps):
    """A longer page table, and with it a bound on the prefixes under which the call is planned as a large one."""
    c.table = torch.cat((c.table, torch.full((c.B, pps - c.pps), -12345, dtype=torch.int32)), 1)
    c.pps, c.hint = pps, pps * 16 - c.rows[0]
    return c


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("rows", [STEP(5), STEP(7), STEP(16), (37, 1, 8, 37), (40, 2, 5, 0), (128, 0, 1, 0), (150, 1, 3, 150), (1, 1, 16, 1)])
def test_small_calls_planned_as_large_ones(T, four, rows):
    """128 rows to a workgroup and pieces of the walks, most of them empty: planned for 65536 positions, filled to a few hundred."""
    heads = (32, 4, 128) if rows[0] < 30 else (12, 4, 128)
    for Ls in ([0], [1, 16, 250], [300, 0, 17, 511, 40]):
        for window, sinks in ((10 ** 6, 0), (10 ** 6, 3)) if not four else ((0, 0),):
            print(f"large four={four} rows={rows} L={Ls}", flush=True)
            c = _room(Case(T, four, heads, BF, Ls, *rows, window, sinks, seed=len(Ls)), 4096).build()
            c.call()
            c.check()
            again = c.call(torch.full_like(c.out, 5.0))
            assert torch.equal(again, c.out)
            c.close()


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("heads,Ls,rows,window,sinks", [
    ((32, 8, 128), [500, 0, 33, 410, 20, 290, 505], STEP(12), 70, 4),       # 700 workgroups of 128 rows: 512 whole, the others cut
    ((16, 4, 128), [100] * 8, (200, 1, 16, 200), 0, 0), ((8, 8, 128), [300, 290], (520, 0, 1, 0), 250, 2),
    ((40, 1, 128), [700, 100, 690], STEP(9), 333, 0), ((12, 2, 128), [1500, 20], STEP(15), 900, 7)])
def test_many_workgroups_and_windows_of_large_calls(T, four, heads, Ls, rows, window, sinks):
    print(f"many four={four} {heads} {Ls} {rows} {window} {sinks}", flush=True)
    if not four and window == 0:
        window = 10 ** 6
    c = Case(T, four, heads, BF, Ls, *rows, window, sinks, seed=21)
    if window == 0 or window >= 10 ** 6:
        _room(c, 4096)
    c.build().call()
    c.check()
    c.hint = 0                                              # too small a bound: other pieces, the same values within rounding
    c.ws.fill_(255)
    c.call()
    c.check()
    c.close()


@pytest.mark.parametrize("heads,dtype", [((6, 2, 24), F32), ((20, 1, 64), F32), ((40, 1, 128), BF), ((8, 8, 2), F32), ((5, 1, 128), F32)])
def test_one_token_window(T, heads, dtype):
    """The step that stores its own row, or, with more than 16 query heads to a kv head, does not."""
    for Ls in ([0], [15], [16, 31, 900], [64, 0]):
        for window, sinks in ((1, 0), (16, 1), (300, 20)):
            print(f"one {heads} {dtype} {Ls} {window}", flush=True)
            c = _run(T, False, heads, dtype, Ls, 1, 0, 1, 1, window, sinks, seed=31)
            kp, vp = c.kp.cpu(), c.vp.cpu()
            for b, L in enumerate(Ls):
                assert torch.equal(kp[c.ids[b, L // 16], :, L % 16, :], c.kn[b, 0])
                assert torch.equal(vp[c.ids[b, L // 16], :, :, L % 16], c.vn[b, 0])
            c.close()


@pytest.mark.parametrize("four", [True, False])
def test_infinities_in_large_calls(T, four):
    """The same as below, 128 rows to a workgroup."""
    for what in range(5):
        c = _room(Case(T, four, (32, 4, 128), BF, [50, 33, 200], 6, 6, 6, 1, 0 if four else 10 ** 6, 0, seed=4), 4096)
        if what == 0:
            c.vn[0, 3, :, 1] = math.nan
        elif what == 1:
            c.kn[0, 4] = math.nan
        elif what == 2:
            c.vn[0, 6 + 6 * 2 + 3, 0, 5] = math.inf
            c.vn[1, 6 + 6 * 2 + 1, 1, 7] = -math.inf
        elif what == 3:
            c.vn[2, 1, :, 2] = math.inf
            c.vn[2, 4, :, 2] = -math.inf
        else:
            c.v[0][1, :, 0] = math.inf
        c.build()
        c.call()
        c.check()
        c.close()


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_that_outgrow_the_reference(T, four, dtype):
    """Scores of several hundred: the softmax reference moves along the text, and most weights underflow."""
    if dtype == BF:
        c = Case(T, four, (4, 2, 128), dtype, [300], *STEP(4), 200, 3, seed=9, scale=20.0)
    else:
        c = Case(T, four, (4, 4, 32), dtype, [300], *STEP(4), 200, 3, seed=9, scale=20.0)
    c.q = c.q * torch.linspace(0.1, 4.0, c.R).view(1, -1, 1, 1).to(dtype)
    c.build()
    c.call()
    torch.cuda.synchronize()
    want, size = c.want(0)
    got = c.out[0].cpu().double()
    # a score off by d moves a weight by d of itself: |s| up to 1000 here, 128 products in fp32 (2^-17 |s|)
    slack = 2.0 ** -6 * (size + want.abs()) if dtype == BF else 2.0 ** -24 * 32 * 1000 * (size + want.abs())
    assert bool(((got - want).abs() <= c.tolerance(want, size) + slack).all())
    c.close()


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_masked_places_and_visible_infinities(T, four, dtype):
    """Infinities and NaN in K and V: rows that do not see the key are as if it were not there, rows that see it get what the sum
    gives (an infinity of V as such from exact pages; 4-bit blocks hold NaN)."""
    heads = (4, 2, 128) if dtype == BF else (4, 4, 32)
    for what in range(6):
        c = Case(T, four, heads, dtype, [50, 33], 6, 6, 6, 1, 20, 2, seed=4)
        if what == 0:
            c.vn[0, 3, :, 1] = math.nan                    # a causal row's V: rows before it do not see it
        elif what == 1:
            c.kn[0, 4] = math.nan
        elif what == 2:
            c.vn[0, 6 + 6 * 2 + 3, 0, 5] = math.inf        # a mask row of block 2
            c.vn[1, 6 + 6 * 2 + 1, 1, 7] = -math.inf
        elif what == 3:
            c.k[0][10], c.v[0][11] = math.nan, math.nan    # behind every window, in front of no sink
        elif what == 4:
            c.v[0][33, :, 2] = math.inf                    # at the window's edge: some rows see it
            c.v[0][35, :, 2] = -math.inf
        else:
            c.v[0][1, :, 0] = math.inf                     # a sink: everybody sees it
        c.build()
        c.call()
        c.check()
        c.close()


@pytest.mark.parametrize("four", [True, False])
def test_invalid_lengths_and_pages_are_reported_and_touch_nothing(T, four):
    c = Case(T, four, (4, 2, 128), BF, [40, 41, 42, 43], *STEP(4), 30, 2, seed=6).build()
    pools = [c.pool] if four else [c.kp, c.vp]
    before = [p.clone() for p in pools]
    c.len[0], c.len[2] = -1, c.pps * 16 - 3                 # negative; no room for the four rows
    c.call()
    c.check(skip=(0, 2))
    assert torch.isnan(c.out[0]).all() and torch.isnan(c.out[2]).all()
    if not four:                                            # nothing of the two is stored
        for b in (0, 2):
            used = c.ids[b].to(DEV)
            for p, q in zip(pools, before):
                assert torch.equal(torch.nan_to_num(p[used], 7.0), torch.nan_to_num(q[used], 7.0))
    c.len[0], c.len[2] = 40, 42
    c.table_d[1, 1], c.table_d[3, 2] = c.n_pages, -1        # pages inside the window
    c.call()
    c.check(skip=(1, 3))
    assert torch.isnan(c.out[1]).any(-1).all() and torch.isnan(c.out[3]).any(-1).all()
    c.close()


@pytest.mark.parametrize("four", [True, False])
def test_any_hint_and_any_workspace_of_the_size(T, four):
    """The bound only plans: too small or too large a hint gives the same values within rounding; two calls the same bits."""
    c = Case(T, four, (32, 8, 128), BF, [1200, 300], 1, 0, 1, 1, 900, 4, seed=8).build()
    c.call()
    c.check()
    again = c.call(torch.empty_like(c.out))
    assert torch.equal(again, c.out)
    for hint in (0, 1200, c.pps * 16 - 1):
        c.hint = hint
        c.ws.fill_(255)
        c.call()
        c.check()
    c.close()


@pytest.mark.parametrize("four", [True, False])
def test_streams_and_captured_calls(T, four):
    """Two calls at once on two streams with a workspace each, and a captured call replayed over changing inputs."""
    a = Case(T, four, (12, 2, 128), BF, [700], *STEP(8), 300, 4, seed=1)
    a.table = a.ids.to(torch.int32)                         # the lengths below reach pages in front of the first window
    a.build()
    b = Case(T, four, (12, 2, 128), BF, [650], *STEP(8), 200, 4, seed=2).build()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            a.call()
        with torch.cuda.stream(s2):
            b.call()
    a.check()
    b.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call()
    eager = torch.empty_like(a.out)
    for i in range(4):
        a.qd.copy_(torch.randn(a.q.shape, generator=torch.Generator().manual_seed(i)).to(BF))
        a.len.fill_(700 - 9 * i)
        a.out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got = a.out.clone()
        a.call(eager)
        torch.cuda.synchronize()
        assert torch.isfinite(got).all() and torch.equal(got, eager)
    a.close()
    b.close()


def test_kv4_pool_beyond_4_gib(T):
    """Page offsets of 64 bits: the pages of one sequence are the last ones of a pool of more than 4 GiB."""
    heads, n_pages = (32, 8, 128), 260000
    ctx = _ctx(T, heads, BF, 1)
    assert n_pages * T.tidar_kv4_page_bytes(ctx) > 1 << 32
    pool = torch.empty(n_pages * T.tidar_kv4_page_bytes(ctx), dtype=torch.uint8, device=DEV)
    L, g = 100, torch.Generator().manual_seed(0)
    table = torch.arange(n_pages - 7, n_pages, dtype=torch.int32, device=DEV).flip(0).contiguous()
    kv = T.tidar_kv4_cache(pool.data_ptr(), table.data_ptr(), 7, n_pages)
    k, v = torch.randn(L + 1, 8, 128, generator=g).to(BF), torch.randn(L + 1, 8, 128, generator=g).to(BF)
    q = torch.randn(1, 1, 32, 128, generator=g).to(BF)
    at = torch.arange(L + 1)
    slots = (table.cpu()[at // 16] * 16 + at % 16).to(torch.int32).to(DEV)
    T.tidar_kv4_store(ctx, kv, 0, L + 1, slots, k.to(DEV), v.to(DEV))
    out = torch.empty(1, 1, 32, 128, dtype=BF, device=DEV)
    ws = torch.empty(T.tidar_attention_workspace_bytes(ctx, 1, 1, 0, 1, L), dtype=torch.uint8, device=DEV)
    T.tidar_kv4_attention(ctx, kv, 0, 1, _i32([L]), q.to(DEV), None, None, 1, 0, 1, 1, 0, 0, out, L, ws)
    torch.cuda.synchronize()
    T.tidar_destroy(ctx)
    want, size = U.attention(q[0].double(), U.fake4(k), U.fake4(v), torch.ones(1, L + 1, dtype=torch.bool))
    assert bool(((out[0].cpu().double() - want).abs() <= 2.0 ** -8 * (1.25 * (size + want.abs()) + want.abs())).all())


def test_binding_refuses_views_and_short_tensors(T):
    c = Case(T, True, (4, 2, 128), BF, [20], *STEP(2), 0, 0).build()
    q = c.qd
    for bad in (torch.empty(1, 6, 4, 256, dtype=BF, device=DEV)[..., ::2], q[:, :5].contiguous(), q.float(), q.transpose(1, 2)):
        c.qd = bad
        with pytest.raises(ValueError, match="q"):
            c.call()
    c.qd = q
    c.call()
    c.check()
    with pytest.raises(ValueError, match="k: "):
        T.tidar_kv4_store(c.ctx, c.kv, 0, 3, _i32([0, 1, 2]), c.kd[:, :2].contiguous(), c.vd)
    c.close()


# ---------------------------------------------------------------- together, as a serving loop uses them
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_tables_rows_and_attention_together(T, window, sinks):
    """Three sequences of different length: prompts into pages from the free list, then steps that append what was accepted, every
    step's attention against the definition over everything that was ever stored."""
    heads = (12, 2, 128)
    n_q, n_kv, hd = heads
    B, pps, n_pages, k_len = 3, 12, 30, 4
    ctx = _ctx(T, heads, BF, B)
    pool = torch.zeros(n_pages, n_kv, 2176, dtype=torch.uint8, device=DEV)
    table = torch.full((B, pps), -1, dtype=torch.int32, device=DEV)
    kv = T.tidar_kv4_cache(pool.data_ptr(), table.data_ptr(), pps, n_pages)
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(2)).to(torch.int32).to(DEV)
    used = 0
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).to(BF)
    lens, text = [0] * B, [(torch.empty(0, n_kv, hd, dtype=BF), torch.empty(0, n_kv, hd, dtype=BF)) for _ in range(B)]
    start, granted, taken = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, 1))
    held, now = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
    for new, accept in (([50, 7, 33], [50, 7, 33]), ([k_len] * B, [1, 4, 2]), ([k_len] * B, [4, 4, 1]), ([1, 1, 1], [1, 1, 1]), ([k_len] * B, [2, 1, 3])):
        slots = torch.empty(sum(new) + 2, dtype=torch.int32, device=DEV)
        P = _i32(lens)
        rest = free[used:].contiguous()
        T.tidar_table_extend(ctx, B, P, _i32(new), held, rest, rest.numel(), table, n_pages, start, slots, now, granted, taken)
        held, now = now, held
        assert granted.tolist() == [1] * B
        used += int(taken)
        rows_k, rows_v = rnd(sum(new) + 2, n_kv, hd), rnd(sum(new) + 2, n_kv, hd)
        T.tidar_kv4_store(ctx, kv, 0, sum(new) + 2, slots, rows_k.to(DEV), rows_v.to(DEV))
        s = start.tolist()
        if len(set(new)) == 1:                              # one attention call for the batch
            nc, nb = new[0], (new[0] if new[0] > 1 else 0)
            rows = (nc, nb, nc if nb else 1, 1)
            R, nm = nc + nb * rows[2], nb * rows[2]
            q, km, vm = rnd(B, R, n_q, hd), rnd(B, nm, n_kv, hd), rnd(B, nm, n_kv, hd)
            out = torch.empty(B, R, n_q, hd, dtype=BF, device=DEV)
            ws = torch.empty(T.tidar_attention_workspace_bytes(ctx, B, *rows[:3], max(lens)), dtype=torch.uint8, device=DEV)
            T.tidar_kv4_attention(ctx, kv, 0, B, P, q.to(DEV), km.to(DEV) if nm else None, vm.to(DEV) if nm else None, *rows, window,
                                  sinks, out, max(lens), ws)
            torch.cuda.synchronize()
            for b in range(B):
                kk = torch.cat((U.fake4(torch.cat((text[b][0], rows_k[s[b]:s[b + 1]]))), km[b].double()))
                vv = torch.cat((U.fake4(torch.cat((text[b][1], rows_v[s[b]:s[b + 1]]))), vm[b].double()))
                want, size = U.attention(q[b].double(), kk, vv, U.mask(lens[b], *rows, window, sinks))
                off = (out[b].cpu().double() - want).abs() - 2.0 ** -8 * (1.25 * (size + want.abs()) + want.abs())
                assert float(off.max()) <= 0, (b, float(off.max()))
        for b in range(B):
            text[b] = tuple(torch.cat((t, r[s[b]:s[b] + accept[b]])) for t, r in zip(text[b], (rows_k, rows_v)))
            lens[b] += accept[b]                            # rejected rows stay behind, and their pages in the table
    T.tidar_destroy(ctx)
