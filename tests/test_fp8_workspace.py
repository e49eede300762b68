"""The workspace of an 8-bit product holds every call of fewer rows, whose K can be split further (no GPU)."""
import pytest

from fp8_plan import fp8_plan, needs


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    return T


@pytest.mark.parametrize("n,k", [(4096, 4096), (4096, 12288), (6144, 4096), (24576, 4096), (1536, 8960), (17920, 1536), (528, 1056), (16, 32),
                                 (16, 12288), (64, 1 << 17), (16, 1 << 20), (48, 1 << 22)])
def test_fewer_rows_fit(T, n, k):
    most, said = 0, 0
    for m in range(1, min(1500, (1 << 31) // k // 16 * 16 - 16) + 1):
        most = max(most, needs(T, m, n, k))
        now = T.tidar_fp8_gemm_workspace_bytes(m, n, k)
        assert now >= most and now >= said, m
        said = now


def test_rows_in_the_millions(T):
    """Larger counts than are split: the rows in 8 bits, and what the split counts below them need."""
    for m, n, k in (((1 << 20) - 16, 16, 2000 // 32 * 32), ((1 << 24) - 16, 16, 32), (1 << 16, 4096, 16384)):
        assert fp8_plan(T, m, n, k).splits == 1
        rest = T.tidar_fp8_gemm_workspace_bytes(m, n, k) - needs(T, m, n, k)
        assert rest >= max(needs(T, x, n, k) for x in range(1, 3000, 7)) - needs(T, 3000, n, k)


def test_the_step_before_a_smaller_one(T):
    """272 rows take no split at 4096 x 4096, 128 and 256 take two: a workspace of the 272 holds them."""
    size = T.tidar_fp8_gemm_workspace_bytes(272, 4096, 4096)
    assert [fp8_plan(T, m, 4096, 4096).splits > 1 for m in (128, 256, 272)] == [True, True, False]
    assert size >= max(needs(T, m, 4096, 4096) for m in (1, 16, 64, 128, 256, 272))
