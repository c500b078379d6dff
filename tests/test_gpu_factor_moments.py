"""GPU parity of the factored second moments against the fp64 oracle.

Sums of positive fp32 values in short chains and trees: 3e-6 relative covers
rows and columns of 2^17 elements (chains of at most some tens of additions
at 2^-24 each, and as many tree levels).
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
RTOL = 3e-6


def make(o, i, eight=False, seed=0, offset=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    v = torch.randn(o * i, generator=g, device=DEV).square_() * 1e-6
    r, c = torch.full((o,), -1.0, device=DEV), torch.full((i,), -1.0, device=DEV)
    if not eight:
        flat = torch.empty(o * i + offset, device=DEV)[offset:]
        return bg.MomentMatrix(flat.copy_(v).view(o, i), r, c)
    codes = torch.randint(0, 256, (o * i + offset,), generator=g, device=DEV).to(torch.uint8)[offset:]
    scale = torch.rand(-(-o * i // 256), generator=g, device=DEV) * 1e-6
    return bg.MomentMatrix(codes.view(o, i), r, c, scale)


def values(m):
    if m.v_scale is None:
        return m.v.cpu().double().numpy()
    return orc.dequantise(m.v.cpu().numpy().reshape(-1), m.v_scale.cpu().numpy(), True).reshape(m.v.shape)


def run(mats, correction=3.0, floor=1e-12):
    ws = bg.workspace_tensor(bg.bergson_factor_moments_workspace(mats), DEV)
    ws.fill_(0xFF)
    bg.bergson_factor_moments(mats, correction, floor, ws)
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()


def check(m, correction=3.0, floor=1e-12):
    r, c = orc.factor_moments(values(m), correction, floor)
    np.testing.assert_allclose(m.r.cpu().double().numpy(), r, rtol=RTOL)
    np.testing.assert_allclose(m.c.cpu().double().numpy(), c, rtol=RTOL)


SHAPES = [(1, 1), (1, 300), (300, 1), (3, 5), (64, 64), (63, 257), (65, 255), (130, 1000), (7, 4099),
          (1031, 129), (2, 131_072), (70_001, 3), (513, 2048)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("o,i", SHAPES)
def test_shapes(o, i, eight):
    m = make(o, i, eight, seed=o + i)
    run([m])
    check(m)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_starts_off_vector_boundaries(offset, eight):
    for shape in ((129, 512), (70, 333)):
        m = make(*shape, eight, seed=offset, offset=offset)
        run([m])
        check(m)


def test_many_matrices_in_one_call():
    r = np.random.default_rng(1)
    mats = [make(int(r.integers(1, 200)), int(r.integers(1, 200)), bool(k % 3 == 0), seed=k)
            for k in range(650)]
    run(mats)
    for k in list(range(0, 650, 17)) + [298, 299, 300, 301, 600, 649]:
        check(mats[k])


def test_no_gradient_yet():
    """v = 0: r is the floor and c is 1, so a layer may take them."""
    m = make(50, 70)
    m.v.zero_()
    run([m], floor=1e-10)
    np.testing.assert_allclose(m.r.cpu().numpy(), 1e-10, rtol=1e-6)
    np.testing.assert_allclose(m.c.cpu().numpy(), 1.0, rtol=1e-6)


def test_nan_shows():
    m = make(100, 300)
    m.v[40, 50] = float("nan")
    run([m])
    r, c = m.r.cpu().numpy(), m.c.cpu().numpy()
    assert np.isnan(r[40]) and np.isfinite(np.delete(r, 40)).all() and np.isnan(c).all()


def test_same_bits_every_time():
    a, b = make(1000, 3001, seed=5), make(1000, 3001, seed=5)
    run([a])
    run([make(10, 10), b])
    assert torch.equal(a.r, b.r) and torch.equal(a.c, b.c)


def test_none():
    run([])


def test_projection_takes_them():
    """r and c of a weight's v as a layer's second moments: the projected
    gradients are those of the oracle's r and c."""
    from paper_2606_11660_gb300 import workloads as wl
    spec = wl.TINY.modules[0]
    A, G = wl.layer_inputs(spec, 4, 32, seed=0)
    m = make(spec.d_out, spec.d_in, seed=3)
    run([m])
    r, c = (torch.tensor(x, dtype=torch.float32, device=DEV)
            for x in orc.factor_moments(values(m), 3.0, 1e-12))
    outs = []
    for rr, cc in ((m.r, m.c), (r, c)):
        layer = bg.Layer(A.to(DEV), G.to(DEV), 16, 16, 1, 2, rr, cc, 0)
        ws = bg.workspace_tensor(bg.bergson_project_grads_workspace([layer], 4, 32), DEV)
        out = torch.empty((4, 256), device=DEV)
        bg.bergson_project_grads([layer], 4, 32, None, out, ws)
        assert bg.bergson_sync_status() == bg.BERGSON_OK
        outs.append(out)
    assert float((outs[0] - outs[1]).norm() / outs[1].norm()) < 1e-4


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("o,i", [(4096, 2048), (4100, 2064), (4099, 2001), (16_411, 513), (1031, 8192)])
def test_rows_of_several_turns(o, i, eight):
    """Matrices whose warps take up to 32 rows each, in several turns of their loops."""
    m = make(o, i, eight, seed=o)
    run([m])
    check(m)
