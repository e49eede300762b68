"""The operators around the paged cache, what needs no GPU: argument checks, sizes, and the test side's own definitions."""
import ctypes as C
import math

import pytest
import torch

import cache_util as U
import tidar_inputs as TI


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    return T


@pytest.fixture()
def ctx(T):
    h = T.tidar_create(T.make_config(TI.SHAPE_8B.with_layers(2), T.TIDAR_BF16, max_k=16, max_batch=8))
    yield h
    T.tidar_destroy(h)


P = 1 << 20                       # non-null, 16-byte aligned; never dereferenced on the host


def test_page_bytes(T, ctx):
    assert T.tidar_kv4_page_bytes(ctx) == 8 * 2176
    tiny = T.tidar_create(T.make_config(TI.TINY, T.TIDAR_F32, max_k=4))
    assert T.tidar_kv4_page_bytes(tiny) == 4 * 544
    T.tidar_destroy(tiny)
    assert T._lib.tidar_kv4_page_bytes(None) == 0


def test_table_extend_refusals(T, ctx):
    good = dict(batch=2, P=P, n=2 * P, held=3 * P, held_out=4 * P, free=5 * P, n_free=3, table=6 * P, pps=4, n_pages=9, start=7 * P,
                slots=8 * P, cap=8, granted=9 * P, taken=10 * P)

    def rc(**kw):
        a = {**good, **kw}
        return T._lib.tidar_table_extend(a.get("ctx", ctx), a["batch"], a["P"], a["n"], a["held"], a["free"], a["n_free"], a["table"],
                                         a["pps"], a["n_pages"], a["start"], a["slots"], a["cap"], a["held_out"], a["granted"],
                                         a["taken"], None)

    for bad in (dict(ctx=None), dict(batch=0), dict(batch=9), dict(P=None), dict(n=None), dict(held=None), dict(held_out=None), dict(held_out=P), dict(held_out=3 * P + 4), dict(held_out=3 * P - 4),
                dict(granted=2 * P), dict(start=P - 8), dict(slots=3 * P - 28), dict(table=5 * P - 28), dict(taken=5 * P + 8), dict(held_out=4 * P, free=4 * P - 8),
                dict(free=None), dict(n_free=-1),
                dict(table=None), dict(pps=0), dict(pps=(1 << 26) + 1), dict(n_pages=0), dict(n_pages=(1 << 27) + 1),
                dict(start=None), dict(slots=None), dict(cap=-1), dict(granted=None), dict(taken=None)):
        assert rc(**bad) == 1, bad


def test_row_refusals(T, ctx):
    for fn in (T._lib.tidar_kv4_store, T._lib.tidar_kv4_load):
        kv = T.tidar_kv4_cache(P, None, 0, 5)
        assert fn(ctx, C.byref(kv), 1, 0, None, None, None, None) == 0            # no rows, nothing to do
        assert fn(None, C.byref(kv), 0, 0, None, None, None, None) == 1
        assert fn(ctx, None, 0, 0, None, None, None, None) == 1
        for layer, n, s, k, v in ((-1, 1, P, P, P), (2, 1, P, P, P), (0, -1, P, P, P), (0, 1, None, P, P), (0, 1, P, None, P),
                                  (0, 1, P, P, None)):
            assert fn(ctx, C.byref(kv), layer, n, s, k, v, None) == 1
        for bad in (T.tidar_kv4_cache(None, None, 0, 5), T.tidar_kv4_cache(P + 8, None, 0, 5), T.tidar_kv4_cache(P, None, 0, 0),
                    T.tidar_kv4_cache(P, None, 0, (1 << 27) + 1)):
            assert fn(ctx, C.byref(bad), 0, 1, P, P, P, None) == 1


@pytest.mark.parametrize("four", [False, True])
def test_attention_refusals(T, ctx, four):
    fn = T._lib.tidar_kv4_attention if four else T._lib.tidar_window_attention
    cache = T.tidar_kv4_cache(P, P, 4, 9) if four else T.tidar_kv_cache(P, P, P, 4, 9)
    good = dict(kv=cache, layer=0, batch=1, pl=P, q=P, k=P, v=P, nc=4, nb=4, bl=4, cond0=1, window=8, sinks=2, out=P, hint=20, ws=P,
                size=1 << 40)

    def rc(**kw):
        a = {**good, **kw}
        kv = a["kv"]
        return fn(a.get("ctx", ctx), None if kv is None else C.byref(kv), a["layer"], a["batch"], a["pl"], a["q"], a["k"], a["v"],
                  a["nc"], a["nb"], a["bl"], a["cond0"], a["window"], a["sinks"], a["out"], a["hint"], a["ws"], a["size"], None)

    bad_caches = [T.tidar_kv4_cache(None, P, 4, 9), T.tidar_kv4_cache(P + 4, P, 4, 9), T.tidar_kv4_cache(P, None, 4, 9),
                  T.tidar_kv4_cache(P, P, 0, 9), T.tidar_kv4_cache(P, P, 4, 0), T.tidar_kv4_cache(P, P, (1 << 26) + 1, 9)] if four else \
                 [T.tidar_kv_cache(None, P, P, 4, 9), T.tidar_kv_cache(P + 4, P, P, 4, 9), T.tidar_kv_cache(P, P + 8, P, 4, 9),
                  T.tidar_kv_cache(P, P, None, 4, 9), T.tidar_kv_cache(P, P, P, (1 << 26) + 1, 9), T.tidar_kv_cache(P, P, P, 4, 1 << 20)]
    for kv in bad_caches + [None]:
        assert rc(kv=kv) == 1
    for bad in (dict(ctx=None), dict(layer=-1), dict(layer=2), dict(batch=0), dict(batch=9), dict(pl=None), dict(q=None),
                dict(q=P + 2), dict(k=None), dict(v=None), dict(nc=0), dict(nb=-1), dict(bl=0), dict(bl=17), dict(cond0=-1),
                dict(cond0=2), dict(cond0=2 ** 31 - 1), dict(window=-1), dict(sinks=-1), dict(out=None), dict(out=P + 4),
                dict(hint=-1), dict(ws=None), dict(ws=P + 8), dict(nc=2 ** 30, hint=0), dict(nb=2 ** 30, nc=2 ** 30),
                dict(nc=(1 << 18) - 15, hint=0), dict(nc=(1 << 23) // 4, hint=0, batch=8)):
        assert rc(**bad) == 1, bad
    assert rc(window=0, sinks=0 if not four else 3) == 1        # no window: exact pages have a call for that; sinks say nothing then
    assert rc(hint=61) == 3                                     # 61 + 4 > 64
    assert rc(size=64) == 2
    if four:
        assert rc(nb=0, k=None, v=None, size=64) == 2           # without mask rows their K/V may be NULL


def test_workspace_covers_fewer_sequences_and_any_window(T, ctx):
    need = [T.tidar_attention_workspace_bytes(ctx, b, 16, 16, 16, 8192) for b in range(1, 9)]
    assert need == sorted(need)
    for args in ((0, 1, 0, 1, 5), (9, 1, 0, 1, 5), (1, 0, 0, 1, 5), (1, 1, 0, 0, 5), (1, 1, 0, 17, 5), (1, 1, -1, 1, 5), (1, 1, 0, 1, -1)):
        with pytest.raises(T.TidarError) as e:
            T.tidar_attention_workspace_bytes(ctx, *args)
        assert e.value.status == 1


def test_binding_refuses_other_tensors(T, ctx):
    """Host tensors, other types: refused before the library is called."""
    kv = T.tidar_kv4_cache(P, P, 4, 9)
    i32, bf = (lambda n: torch.zeros(n, dtype=torch.int32)), (lambda n: torch.zeros(n, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="slots"):
        T.tidar_kv4_store(ctx, kv, 0, 2, i32(2), bf(2 * 1024), bf(2 * 1024))
    with pytest.raises(ValueError, match="int64"):
        T.tidar_kv4_load(ctx, kv, 0, 2, torch.zeros(2, dtype=torch.int64), bf(2 * 1024), bf(2 * 1024))
    with pytest.raises(ValueError, match="prefix_len"):
        T.tidar_kv4_attention(ctx, kv, 0, 1, i32(1), bf(4096), None, None, 1, 0, 1, 1, 0, 0, bf(4096), 8, bf(4096))
    with pytest.raises(ValueError, match="prefix_len"):
        T.tidar_table_extend(ctx, 1, i32(1), i32(1), i32(1), i32(4), 4, i32(8).view(1, 8), 9, i32(2), i32(8), i32(1), i32(1), i32(1))


# ---------------------------------------------------------------- the test side's definitions
def test_levels_and_ties_of_the_reference():
    edge = [0, 0.25, 0.2500001, 0.75, 0.7499999, 1.25, 1.2500001, 1.75, 1.7499999, 2.5, 2.5000001, 3.5, 3.4999999, 5, 5.0000001, 6, 6.9, 7]
    want = [0, 0, 0.5, 1, 0.5, 1, 1.5, 2, 1.5, 2, 3, 4, 3, 4, 6, 6, 6, 6]
    x = torch.tensor(edge + [7.0] * 14, dtype=torch.float64)
    assert U.fake4(x)[:len(edge)].tolist() == want
    assert U.fake4(-x)[:len(edge)].tolist() == [-w for w in want]
    assert U.fake4(torch.full((32,), 7.0001, dtype=torch.float64)).tolist() == [8.0] * 32      # the next exponent
    for e in (-140, -125, 0, 3, 120):                                                          # scales: powers of two, held in range
        y = U.fake4(x * 2.0 ** e)[:len(edge)]
        if -125 <= e <= 125:
            assert y.tolist() == [w * 2.0 ** e for w in want]
        else:
            assert y.tolist() == [0.0] * len(edge)
    assert torch.isnan(U.fake4(torch.tensor([math.inf] + [1.0] * 31))).all()


def test_no_element_is_off_by_more_than_half_a_step():
    x = torch.randn(400, 64, dtype=torch.float64, generator=torch.Generator().manual_seed(1)) * 3
    code, byte = U.quantise(x)
    step = torch.exp2(byte.double() - 127).unsqueeze(-1)
    mag = torch.tensor(U.LEVELS, dtype=torch.float64)[code % 8].unflatten(-1, (2, 32))
    gap = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0)) * step
    assert bool(((U.values(code, byte, 64) - x).unflatten(-1, (2, 32)).abs() <= gap / 2 * (1 + 1e-12)).all())


def test_mask_without_window_is_the_hybrid_mask_of_the_oracle():
    from oracle import tidar_oracle as O
    for k, L in ((1, 0), (3, 5), (4, 17)):
        assert torch.equal(U.mask(L, k, k, k, 1, 0, 0), O.decode_mask(k, L))
        assert torch.equal(U.mask(L, k, k, k, 1, L + 3 * k, 0), O.decode_mask(k, L))           # a window that holds everything
    assert torch.equal(U.mask(7, 5, 0, 1, 5, 0, 0), O.causal_mask(5, 7))
    see = U.mask(40, 1, 0, 1, 1, 8, 3)[0]
    assert see.nonzero().flatten().tolist() == [0, 1, 2] + list(range(33, 41))
