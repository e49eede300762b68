"""The attention over a span, what the host decides: which calls it refuses for their size, and which kernel the others get."""
import ctypes as C
import random

import pytest

import tidar_inputs as TI
from span_plan import span_plan

P = 1 << 20                       # non-null, 16-byte aligned; never dereferenced on the host


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    return T


@pytest.mark.parametrize("four", [False, True])
def test_more_heads_of_sequences_than_a_launch_has_workgroups_for(T, four):
    """8 kv heads: 2^19 sequences are planned (and need more workspace than is given), one more is refused."""
    most = 1 << 19
    ctx = T.tidar_create(T.make_config(TI.SHAPE_8B.with_layers(1), T.TIDAR_BF16, max_k=16, max_batch=2 * most))
    fn = T._lib.tidar_kv4_attention if four else T._lib.tidar_window_attention
    kv = T.tidar_kv4_cache(P, P, 4, 9) if four else T.tidar_kv_cache(P, P, P, 4, 9)
    for batch, status in ((most, 2), (most + 1, 1), (2 * most, 1)):
        assert fn(ctx, C.byref(kv), 0, batch, P, P, P, P, 1, 0, 1, 1, 8, 0, P, 20, P, 64, None) == status
        n = C.c_size_t()
        assert T._lib.tidar_attention_workspace_bytes(ctx, batch, 1, 0, 1, 20, C.byref(n)) == (0 if status == 2 else 1)
    T.tidar_destroy(ctx)


BIG, SMALL = (32, 8, 128), (12, 2, 128)                    # 4 and 6 query heads to a kv head
STEP = lambda k: (k, k, k, 1)
ONE = (1, 0, 1, 1)


@pytest.mark.parametrize("four,B,heads,rows,window,prefix,many", [
    # 4-bit pages, both sides of the rule: its work, and the rows that a workgroup of 128 needs
    (True, 8, BIG, STEP(6), 0, 1000, False), (True, 8, SMALL, STEP(4), 0, 8000, False), (True, 32, SMALL, STEP(6), 0, 1000, True),
    (True, 8, BIG, STEP(8), 0, 1000, True), (True, 8, BIG, STEP(3), 0, 8000, False),
    # exact pages: one round of workgroups by their number, several in whole rounds
    (False, 1, SMALL, STEP(16), 1000, 4096, False), (False, 1, SMALL, STEP(16), 3000, 4096, True), (False, 8, BIG, STEP(4), 1000, 8192, True),
    (False, 8, BIG, STEP(8), 1000, 8192, True),
    # a decode step of 16 drafts, prompts, single tokens
    (True, 8, BIG, STEP(16), 0, 8192, True), (True, 1, SMALL, (1999, 1, 16, 1999), 0, 1000, True),
    (False, 1, BIG, (2048, 1, 16, 2048), 1024, 2048, True), (True, 32, BIG, ONE, 0, 8192, False), (False, 16, BIG, ONE, 1024, 8192, False),
    (True, 1 << 15, BIG, ONE, 0, 8192, False)])
def test_which_kernel(T, four, B, heads, rows, window, prefix, many):
    assert span_plan(T, True, four, B, heads, rows, window, 4 if window else 0, prefix).rows == many
    assert not span_plan(T, False, four, B, heads, rows, window, 4 if window else 0, prefix).rows        # fp32: one kernel


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_workspace_holds_the_partial_results_of_any_plan(T, dtype):
    """For every smaller batch, either kind of pages, any window, sinks, first conditioning row and bound on the prefixes."""
    rng, bf16 = random.Random(5), dtype == "bf16"
    for _ in range(400):
        group, n_kv, hd = rng.choice([1, 2, 4, 6, 7, 20]), rng.choice([1, 2, 3, 4, 8]), 128 if bf16 else rng.choice([16, 32, 48, 128])
        nc = rng.choice([1, 2, 5, 16, 100, 128, 300, 2048])
        nb, bl = rng.choice([0, 1, min(nc, 16)]), rng.choice([1, 3, 5, 16])
        most = rng.choice([1, 3, 8, 40])
        heads = (group * n_kv * (2 if bf16 else 1), n_kv, hd)
        ctx = T.tidar_create(T.tidar_config(1, 128, *heads, 512, 512, 0, T.TIDAR_BF16 if bf16 else T.TIDAR_F32, 16, 16, most, 511, 1e4, 1e-6))
        size = T.tidar_attention_workspace_bytes(ctx, most, nc, nb, bl, rng.choice([0, 100, 8000]))
        T.tidar_destroy(ctx)
        for _ in range(20):
            B, window = rng.randint(1, most), rng.choice([0, 1, 300, 5000])
            cond0 = rng.randint(0, nc + 1 - nb) if nb else 0
            p = span_plan(T, bf16, rng.random() < 0.5, B, heads, (nc, nb, bl, cond0), window, 4 if window else 0, rng.choice([0, 50, 900, 70000]))
            tiles = 2 * B * n_kv * ((nb * bl + 15) // 16) * 16 * hd * (2 if bf16 else 4)
            assert p.part_floats * 4 + tiles <= size
            if not p.rows:                                  # a result and two statistics for every row and split
                assert p.splits == 1 or p.part_floats >= B * heads[0] * (nc + nb * bl) * p.splits * (hd + 2)
            elif p.splits > 1:                              # of every piece of the walks that are cut, and two numbers for each walk
                cut = B * n_kv * p.tiles - p.whole
                assert 0 < cut < 512 and cut * p.splits <= 1024 and p.part_floats >= cut * (p.splits * 128 * 130 + 2)
