"""Rows that hold NaN or an infinity, or whose squares pass fp32, in both kinds of norm: the whole row is
NaN, the others keep their values, whichever kernel has them."""
import pytest
import torch

import paper_2606_11660_gb300 as bg
from tests.test_gpu_norm import DEV, DTYPES, LAYER, RMS, forward, inputs, matrix, ok

pytestmark = pytest.mark.gpu
KEEP = [0, 1, 3, 5, 8, 9]


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1), (2, 2)])
@pytest.mark.parametrize("d", [1, 24, 100, 300, 520, 1000, 3000, 9000, 17_000])
def test_spoiled_rows(d, pad, offset, dtype, kind):
    R = 10
    x, dy, w, b = inputs(R, d, dtype, torch.float32, pad, offset, seed=d)
    good, _, _ = forward(x, w, b, kind)
    x[2, d // 2], x[4, 0], x[6, d - 1], x[7] = float("inf"), float("nan"), float("-inf"), float("inf")
    flat, y = matrix(R, d, dtype, pad, offset)
    _, mean, rstd = forward(x, w, b, kind, y=y)
    ok()
    spoiled = [2, 4, 6, 7]
    assert bool(y[spoiled].isnan().all()) and bool(rstd[spoiled].isnan().all())
    assert torch.equal(y[KEEP], good[KEEP])
    dx = torch.empty_like(x)
    ws = bg.workspace_tensor(bg.bergson_norm_backward_workspace(R, d), DEV)
    bg.bergson_norm_backward(x, w, kind, mean, rstd, dy, dx, None, None, ws)
    ok()
    assert bool(dx[spoiled].isnan().all()) and not bool(dx[KEEP].isnan().any())
    y.fill_(7.0)
    assert bool((flat == 7.0).all())


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("d", [24, 300, 1000, 3000, 9000, 17_000])
def test_squares_that_overflow(d, kind):
    """1e25 and its negative in turn: the mean is 0, the squares are not numbers that fp32 holds."""
    for pad in (0, 1):
        x, _, w, b = inputs(10, d, torch.float32, torch.float32, pad, seed=d)
        good, _, _ = forward(x, w, b, kind)
        x[4, ::2], x[4, 1::2] = 1e25, -1e25
        y, _, rstd = forward(x, w, b, kind)
        ok()
        assert bool(y[4].isnan().all()) and bool(rstd[4].isnan())
        assert torch.equal(y[KEEP], good[KEEP])
