"""The attention over a span, what the host decides: which calls it refuses for their size, and which kernel the others get."""
import ctypes as C

import pytest

import tidar_inputs as TI

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
