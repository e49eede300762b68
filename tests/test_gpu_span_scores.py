"""Scores so large that neighbouring floats are whole units apart: the softmax is one for the largest score of a row and zero for the
others, unless the two largest are as close as a sum of products in fp32 is off (by at most hd 2^-24 of the sum of their magnitudes
each): such a row may take either, and only has to be finite.

bf16 takes numerators as 2^(s * scale - m) with one rounding, whose error reaches 2^7 from s * scale = 2^31 on: magnitudes up to 2^30.
fp32 scales the scores first, and the distance from m is exact then at any size.
"""
import math

import pytest
import torch

import cache_util as U
from span_plan import plan_of
from test_gpu_cache_ops import BF, F32, STEP, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import paper_2511_08923_amd as T
    assert torch.cuda.is_available()
    return T


def _clear(c, b):
    """[row][head]: whether the largest score stands out, by what both may be off and by 24, so that other weights are below e^-24 < 2^-34."""
    nc, nb, bl, cond0 = c.rows
    hd, group = c.heads[2], c.heads[0] // c.heads[1]
    k = torch.cat((c.k[b], c.kn[b, :nc])).double()
    k = torch.cat((U.fake4(k) if c.four else k, c.kn[b, nc:].double()))
    see = U.mask(c.Ls[b], nc, nb, bl, cond0, c.window, c.sinks)
    q, out = c.q[b].double(), torch.empty(c.R, c.heads[0], dtype=torch.bool)
    for h in range(c.heads[0]):
        kk, low = k[:, h // group], torch.tensor(-math.inf, dtype=torch.float64)
        top = torch.where(see, q[:, h] @ kk.T, low).topk(2, -1).values if see.shape[1] > 1 else None
        off = hd * 2.0 ** -24 * (q[:, h].abs() @ kk.T.abs()).amax(-1)
        out[:, h] = True if top is None else top[:, 0] - top[:, 1] > 2 * off + 24 * math.sqrt(hd)
    return out


def _check(T, four, heads, dtype, Ls, rows, e, many=False):
    c = Case(T, four, heads, dtype, Ls, *rows, 0 if four else 10 ** 6, 0, seed=3, scale=2.0 ** e)
    assert plan_of(c).rows == many
    print(f"scores four={four} {heads} {dtype} rows={rows} 2^{e}", flush=True)
    c.build()
    c.call()
    for b in range(c.B):
        want, size = c.want(b)
        got, clear = c.out[b].cpu().double(), _clear(c, b)
        assert torch.isfinite(got).all() and float(clear.double().mean()) > 0.9
        # the one value that is left, rounded to bf16 (fp32 holds it), and up to 2048 values below 8 with weights below 2^-34
        off = (got - want).abs() - (2.0 ** -8 if dtype == BF else 2.0 ** -22) * (size + want.abs()) - 2.0 ** -20
        assert bool((off[clear] <= 0).all())
    c.close()


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("heads", [(4, 2, 128), (4, 4, 32), (2, 2, 72)])
@pytest.mark.parametrize("rows", [(1, 0, 1, 1), STEP(4)])
@pytest.mark.parametrize("e", [24, 28, 32, 60, 100])
def test_fp32_scores_of_any_size(T, four, heads, rows, e):
    _check(T, four, heads, F32, [300], rows, e)


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("e", [24, 27])
def test_bf16_scores_up_to_2_to_the_30(T, four, e):
    for rows in ((1, 0, 1, 1), STEP(4)):
        _check(T, four, (4, 2, 128), BF, [300], rows, e)
    _check(T, four, (24, 2, 128), BF, [1700, 500], STEP(16), e, many=True)
