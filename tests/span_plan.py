"""Which kernel an attention call over a span gets and how its walks are cut: pure host arithmetic, read from the library through
the C++ symbol of the planner (no GPU)."""
import ctypes as C

from test_attention_order import RowDesc


class SpanPlan(C.Structure):
    """Mirrors SpanPlan of csrc/tidar_internal.h."""
    _fields_ = [("rows", C.c_bool)] + [(n, C.c_int) for n in ("span_rows", "whole", "per", "tiles", "splits")] + [
        ("part_floats", C.c_size_t)]


def span_plan(T, bf16, four, B, heads, rows, window, sinks, hint):
    """heads: (query heads, kv heads, head_dim); rows: (n_causal, n_blocks, block_len, cond0)."""
    f = C.CDLL(T.LIB_PATH)._Z9plan_spanibiiiiRK7RowDesciii
    f.argtypes = [C.c_int, C.c_bool, C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(RowDesc), C.c_int, C.c_int, C.c_int]
    f.restype = SpanPlan
    nc, nb, bl, cond0 = rows
    d = RowDesc(nc, nb, bl, cond0, 1, nb * bl, nc + nb * bl, 0)
    return f(T.TIDAR_BF16 if bf16 else T.TIDAR_F32, four, B, heads[0], heads[1], heads[2], C.byref(d), window, sinks, hint)


def plan_of(case):
    """The plan of a call of test_gpu_cache_ops.Case."""
    import torch
    most = 1 << 30
    return span_plan(case.T, case.dtype == torch.bfloat16, case.four, case.B, case.heads, case.rows, min(case.window, most),
                     min(case.sinks, most), case.hint)


def workgroups(case, p):
    """Of 128 rows: (whole ones, walks that are cut)."""
    assert p.rows
    return p.whole, case.B * case.heads[1] * p.tiles - p.whole
