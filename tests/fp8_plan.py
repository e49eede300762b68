"""What an 8-bit product gets: pure host arithmetic, read from the library through the C++ symbols of the planner (no GPU)."""
import ctypes as C


class Gemm8Plan(C.Structure):
    """Mirrors Gemm8Plan of csrc/tidar_internal.h."""
    _fields_ = [(n, C.c_int) for n in ("ra", "ca", "tall", "shorts", "splits", "per")]


def fp8_plan(T, m, n, k):
    f = C.CDLL(T.LIB_PATH)._Z13plan_gemm_fp8iii
    f.argtypes, f.restype = [C.c_int] * 3, Gemm8Plan
    return f(m, n, k)


def own_rows(T, m, n, k):
    f = C.CDLL(T.LIB_PATH)._Z17gemm_fp8_own_rowsiii
    f.argtypes, f.restype = [C.c_int] * 3, C.c_bool
    return f(m, n, k)


def kind(T, m, n, k):
    """"own": few rows that the product brings into 8 bits itself; "few": few rows; else (row tiles of a wave, column tiles, whether passes of one
    row tile less follow, splits of K)."""
    p = fp8_plan(T, m, n, k)
    return ("own" if own_rows(T, m, n, k) else "few") if p.ra == 0 else (p.ra, p.ca, p.shorts > 0, p.splits)


def needs(T, m, n, k):
    """Bytes of the workspace that the call itself asks for: the rows in 8 bits, and partial sums."""
    up = lambda x: (x + 255) // 256 * 256
    blocks, tiles, p = (k + 127) // 128, (m + 15) // 16, fp8_plan(T, m, n, k)
    return up(tiles * blocks * 2048 + (blocks + 3) // 4 * tiles * 64) + up(p.splits * m * n * 4 if p.splits > 1 else 0)
