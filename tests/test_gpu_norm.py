"""GPU parity of layer norm and its form without a mean, and their backward pass, with the fp64 oracle.

Tolerances, from the roundings in the path: a row's sums run 16 values deep in a
thread and at most 10 levels of a tree above, so that a mean is off by at most 26 *
2^-24 = 1.6e-6 of the mean magnitude and a mean square by as much relatively (a
half of that in rstd); what follows are at most six roundings of 2^-24.  Sums over
rows are as deep as a CTA's turns, its warps and the 1/8 of the CTAs that one thread
adds.  An output in 16 bits adds its half unit.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import model_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
LAYER, RMS = bg.BERGSON_NORM_LAYER, bg.BERGSON_NORM_RMS
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 1e-42, torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}
EPS = 1e-5


def np64(x):
    return x.detach().cpu().double().numpy()


def matrix(R, d, dtype, pad=0, offset=0, fill=7.0):
    flat = torch.full((offset + R * (d + pad) + 16,), fill, dtype=dtype, device=DEV)
    return flat, flat[offset:offset + R * (d + pad)].view(R, d + pad)[:, :d]


def inputs(R, d, dtype, wt, pad=0, offset=0, seed=0, shift=0.3):
    g = torch.Generator().manual_seed(seed)
    _, x = matrix(R, d, dtype, pad, offset)
    _, dy = matrix(R, d, dtype, pad, offset)
    scale = torch.exp(torch.randn((R, 1), generator=g))
    x.copy_(scale * (torch.randn((R, d), generator=g) + shift))
    dy.copy_(torch.randn((R, d), generator=g))
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(wt).to(DEV)
    b = (0.2 * torch.randn(d, generator=g)).to(wt).to(DEV)
    return x, dy, w, b


def forward(x, w, b, kind, eps=EPS, y=None, stats=True):
    R, _ = x.shape
    y = torch.empty_like(x) if y is None else y
    mean = torch.full((R,), 7.0, device=DEV) if stats and kind == LAYER else None
    rstd = torch.full((R,), 7.0, device=DEV) if stats else None
    bg.bergson_norm(x, w, b, kind, eps, y, mean, rstd)
    return y, mean, rstd


def ok():
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()


def near(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4],
                           np.broadcast_to(tol, got.shape)[bad][:4])


def check_forward(x, w, b, kind, eps=EPS, y=None):
    x64 = np64(x)
    y, mean, rstd = forward(x, w, b, kind, eps, y)
    ok()
    w64, b64 = (None if t is None else np64(t) for t in (w, b))
    want, mu, rs = orc.norm(x64, w64, b64, kind == LAYER, eps)
    size = np.abs(x64).mean(1)
    if mean is not None:
        near(np64(mean), mu, 28 * U * size, "mean")
    near(np64(rstd), rs, 20 * U * rs + rs ** 2 * 60 * U * size, "rstd")
    n = np.abs((x64 - mu[:, None]) * rs[:, None])
    ws = 1.0 if w64 is None else np.abs(w64)
    tol = ws * (rs[:, None] * 30 * U * size[:, None] + n * (26 + rs[:, None] * 60 * size[:, None]) * U)
    near(np64(y), want, tol + (HALF_UNIT[x.dtype] + U) * np.abs(want) * 1.01 + SMALLEST[x.dtype], "y")
    return y, mean, rstd


def check_backward(x, dy, w, kind, mean, rstd, dx=None, sums=(True, True)):
    R, d = x.shape
    x64, dy64 = np64(x), np64(dy)
    dx = torch.empty_like(x) if dx is None else dx
    dw, db = (torch.full((d,), 7.0, device=DEV) if k else None for k in sums)
    ws = bg.workspace_tensor(bg.bergson_norm_backward_workspace(R, d), DEV)
    ws.fill_(255)
    bg.bergson_norm_backward(x, w, kind, mean, rstd, dy, dx, dw, db, ws)
    ok()
    w64 = np.ones(d) if w is None else np64(w)
    mu = np64(mean) if kind == LAYER else np.zeros(R)
    rs = np64(rstd)
    want, wdw, wdb = orc.norm_backward(x64, w64, kind == LAYER, mu, rs, dy64)
    n, h = np.abs((x64 - mu[:, None]) * rs[:, None]), np.abs(dy64 * w64)
    tol = rs[:, None] * U * (4 * h + n * 34 * (h * n).mean(1, keepdims=True) +
                             32 * h.mean(1, keepdims=True))
    near(np64(dx), want, tol + (HALF_UNIT[x.dtype] + U) * np.abs(want) * 1.01 + SMALLEST[x.dtype], "dx")
    depth = R + 30 if R < 64 else R / 152 + 160 + 30
    if dw is not None:
        near(np64(dw), wdw, (depth + 4) * U * (np.abs(dy64) * n).sum(0) + 1e-42, "dw")
    if db is not None:
        near(np64(db), wdb, depth * U * np.abs(dy64).sum(0) + 1e-42, "db")
    return dx, dw, db


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,d", [(1, 1), (7, 3), (5, 24), (130, 33), (64, 128), (9, 256), (33, 257),
                                 (5, 512), (6, 513), (5, 768), (31, 1029), (17, 2048), (3, 5000),
                                 (4, 8192), (3, 8200), (2, 16384), (3, 16385), (2, 40_001)])
def test_norm(R, d, dtype, kind):
    x, dy, w, b = inputs(R, d, dtype, dtype if d % 2 else torch.float32, seed=R + d)
    _, mean, rstd = check_forward(x, w, b if kind == LAYER else None, kind)
    check_backward(x, dy, w, kind, mean, rstd)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(3, 0), (8, 0), (8, 8), (0, 1), (5, 3)])
@pytest.mark.parametrize("d", [40, 264, 1032, 2051, 9000])
def test_rows_apart(d, pad, offset, dtype):
    """Any leading dimension and start; what lies between the rows keeps its value."""
    R = 6
    x, dy, w, b = inputs(R, d, dtype, torch.float32, pad, offset, seed=d)
    flat, y = matrix(R, d, dtype, pad, offset)
    _, mean, rstd = check_forward(x, w, b, LAYER, y=y)
    flat2, dx = matrix(R, d, dtype, pad, offset)
    check_backward(x, dy, w, LAYER, mean, rstd, dx)
    for f, m in ((flat, y), (flat2, dx)):
        m.fill_(7.0)
        assert bool((f == 7.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,pad,offset", [(41, 1, 0), (40, 2, 2), (250, 4, 6), (257, 5, 4), (777, 1, 10),
                                          (1030, 4, 0), (8191, 1, 2), (9001, 1, 4), (16383, 3, 2)])
def test_rows_of_whole_words(d, pad, offset, dtype):
    """Rows at even elements, no multiple of 16 bytes apart or not on one, odd and even lengths."""
    R = 7
    x, dy, w, b = inputs(R, d, dtype, dtype, pad, offset, seed=d)
    flat, y = matrix(R, d, dtype, pad, offset)
    _, mean, rstd = check_forward(x, w, b, LAYER, y=y)
    flat2, dx = matrix(R, d, dtype, pad, offset)
    check_backward(x, dy, w, LAYER, mean, rstd, dx)
    for f, m in ((flat, y), (flat2, dx)):
        m.fill_(7.0)
        assert bool((f == 7.0).all())


@pytest.mark.parametrize("R,d", [(4000, 24), (5000, 300), (3000, 1100), (700, 8192), (400, 10_000),
                                 (700, 17_000)])
def test_many_rows(R, d):
    """Several turns of a CTA, and the sums over them."""
    x, dy, w, b = inputs(R, d, torch.bfloat16, torch.bfloat16, seed=R)
    _, mean, rstd = check_forward(x, w, b, LAYER)
    check_backward(x, dy, w, LAYER, mean, rstd)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,d,pad", [(1, 520, 0), (7, 520, 8), (4001, 776, 0), (6003, 1001, 7), (9, 1017, 7),
                                     (2500, 1024, 8)])
def test_medium_rows(R, d, pad, dtype):
    """Rows that end inside a vector, of a warp's last turn alone or of many turns."""
    x, dy, w, b = inputs(R, d, dtype, dtype, pad, 8, seed=R)
    flat, y = matrix(R, d, dtype, pad, 8)
    _, mean, rstd = check_forward(x, w, b, LAYER, y=y)
    check_backward(x, dy, w, LAYER, mean, rstd)
    y.fill_(7.0)
    assert bool((flat == 7.0).all())


@pytest.mark.parametrize("d", [100, 1000, 9000, 17_000])
def test_in_place_and_optional(d):
    x, dy, w, b = inputs(40, d, torch.bfloat16, torch.float32, seed=d)
    y, mean, rstd = forward(x, w, b, LAYER)
    x2 = x.clone()
    y2, _, _ = forward(x2, w, b, LAYER, y=x2, stats=False)
    assert torch.equal(y2, y)
    dx, dw, db = check_backward(x, dy, w, LAYER, mean, rstd)
    for into in ("x", "dy"):
        a, g = x.clone(), dy.clone()
        got = check_backward(a, g, w, LAYER, mean, rstd, a if into == "x" else g)
        assert all(torch.equal(u, v) for u, v in zip(got, (dx, dw, db)))
    assert torch.equal(check_backward(x, dy, w, LAYER, mean, rstd, sums=(False, False))[0], dx)
    assert torch.equal(check_backward(x, dy, w, LAYER, mean, rstd, sums=(False, True))[2], db)
    assert torch.equal(check_backward(x, dy, w, LAYER, mean, rstd, sums=(True, False))[1], dw)
    check_forward(x, None, None, RMS)
    check_forward(x, None, b, LAYER)
    _, _, r2 = forward(x, None, None, RMS)
    check_backward(x, dy, None, RMS, None, r2)


@pytest.mark.parametrize("d", [64, 700, 3000, 17_000])
def test_values_at_the_borders(d):
    """A far offset, a constant row, zeros, and rows that hold infinities or NaN."""
    x, dy, w, b = inputs(8, d, torch.float32, torch.float32, seed=d)
    x[1] += 1000.0
    x[2] = 5.0
    x[3] = 0.0
    check_forward(x, w, b, LAYER)
    good, mean, rstd = forward(x, w, b, LAYER)
    x[5, d // 2], x[6, 0] = float("inf"), float("nan")
    y, mean, rstd = forward(x, w, b, LAYER)
    ok()
    assert bool(y[5:7].isnan().all())
    keep = [0, 1, 2, 3, 4, 7]
    assert torch.equal(y[keep], good[keep])
    dx = torch.empty_like(x)
    ws = bg.workspace_tensor(bg.bergson_norm_backward_workspace(8, d), DEV)
    bg.bergson_norm_backward(x, w, LAYER, mean, rstd, dy, dx, None, None, ws)
    assert bool(dx[5:7].isnan().all()) and not bool(dx[keep].isnan().any())


def test_no_rows():
    x = torch.empty((0, 64), device=DEV)
    dw, db = torch.full((64,), 7.0, device=DEV), torch.full((64,), 7.0, device=DEV)
    bg.bergson_norm(x, None, None, LAYER, EPS, x, torch.empty(0, device=DEV), torch.empty(0, device=DEV))
    ws = bg.workspace_tensor(bg.bergson_norm_backward_workspace(0, 64), DEV)
    e = torch.empty(0, device=DEV)
    bg.bergson_norm_backward(x, None, LAYER, e, e, x, x, dw, db, ws)
    ok()
    assert not bool(dw.any()) and not bool(db.any())


def test_same_bits_every_time():
    x, dy, w, b = inputs(3000, 1000, torch.bfloat16, torch.float32)
    _, mean, rstd = forward(x, w, b, LAYER)
    first = check_backward(x, dy, w, LAYER, mean, rstd)
    for _ in range(3):
        assert all(torch.equal(u, v) for u, v in
                   zip(first, check_backward(x, dy, w, LAYER, mean, rstd)))


def test_gradients_against_differences():
    """The kernels' own gradients along a direction, and the change of the kernels' forward pass."""
    g = torch.Generator().manual_seed(3)
    R, d, e = 6, 96, 2.0 ** -9
    x, u, dy = (torch.randn((R, d), generator=g).to(DEV) for _ in range(3))
    w, b, uw, ub = (torch.randn(d, generator=g).to(DEV) for _ in range(4))
    for kind in (LAYER, RMS):
        _, mean, rstd = forward(x, w, b, kind)
        dx, dw, db = check_backward(x, dy, w, kind, mean, rstd)

        def f(s):
            y, _, _ = forward(x + s * u, w + s * uw, b + s * ub, kind)
            return float((y.double() * dy.double()).sum())
        slope = (f(e) - f(-e)) / (2 * e)
        want = float(((dx * u).sum() + (dw * uw).sum() + (db * ub).sum()).double())
        # rounding: 576 values of a few units, 1e-6 each, over 2e; curvature: e^2 / 6 times third
        # derivatives of some 10 a value along a direction of length 1 a row's element
        size = float((dx.abs() * u.abs()).sum() + (dw.abs() * uw.abs()).sum())
        assert abs(slope - want) <= 576 ** 0.5 * 4e-6 / (2 * e) + 10 * e * e * size, (slope, want)


def test_refused_tensors():
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    y32, e = torch.zeros((4, 64), device=DEV), torch.zeros(4, device=DEV)
    ws = bg.workspace_tensor(256, DEV)
    with pytest.raises(ValueError):
        bg.bergson_norm(x, None, None, LAYER, EPS, y32)
    with pytest.raises(ValueError):
        bg.bergson_norm(x, torch.ones(63, device=DEV), None, LAYER, EPS, x)
    with pytest.raises(ValueError):
        bg.bergson_norm(x, torch.ones(64, device=DEV), torch.ones(64, device=DEV).bfloat16(), LAYER, EPS, x)
    with pytest.raises(ValueError):
        bg.bergson_norm(x, torch.ones(64), None, LAYER, EPS, x)
    with pytest.raises(ValueError):
        bg.bergson_norm(x.t(), None, None, LAYER, EPS, x.t())
    with pytest.raises(TypeError):
        bg.bergson_norm(x.long(), None, None, LAYER, EPS, x.long())
    with pytest.raises(bg.BergsonError) as err:
        bg.bergson_norm_backward(x, None, LAYER, e, e, x, torch.empty_like(x), y32[0], None, ws)
    assert err.value.status == bg.BERGSON_EWORKSPACE
