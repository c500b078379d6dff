"""Muon steps on updates of any size that fp32 holds, and over more tiles than one count of all takes.

Tolerances are test_gpu_muon's: an update's size drops out of X = u / |u|_F, so that they hold at
every size.  u is read back from m (beta 0, or no new gradient), so that the roundings of small
numbers on the way to it are the oracle's too.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import model_oracle as orc
from tests.test_gpu_muon import DEV, FIVE, check_x, np64, ok, step

pytestmark = pytest.mark.gpu


def update(o, i, scale, rank=0, seed=0):
    """Gaussian entries, or of `rank`, in fp32: the smaller ones in what subnormals leave of them."""
    g = torch.Generator().manual_seed(seed + 1000 * o + i + rank)
    x = torch.randn((o, i), generator=g, dtype=torch.float64)
    if rank:
        x = torch.randn((o, rank), generator=g, dtype=torch.float64) @ torch.randn(
            (rank, i), generator=g, dtype=torch.float64) / rank ** 0.5
    return (scale * x).float().to(DEV)


SCALES = [1e-44, 1e-42, 5e-39, 1.5e-38, 1e-37, 1e-36, 1e-34, 1e-32, 1e-20, 1e18, 1e32, 1e34, 1e36, 2e37]


@pytest.mark.parametrize("products", [3, 1])
@pytest.mark.parametrize("o,i,rank", [(64, 64, 0), (100, 140, 0), (264, 264, 3)])
@pytest.mark.parametrize("scale", SCALES)
def test_any_size(scale, o, i, rank, products):
    g = update(o, i, scale, rank)
    assert bool(g.isfinite().all()) and bool(g.any())
    w, m = torch.zeros_like(g), torch.zeros_like(g)
    step([bg.MuonTensor(w, g, m)], -1.0, 0.0, False, FIVE, products)
    assert torch.equal(m, g)
    check_x(np64(w), np64(g), FIVE, products)


@pytest.mark.parametrize("products", [3, 1])
def test_scaled_gradients(products):
    """16-bit gradients whose scale takes them to the ends of the range."""
    for scale in (1e-37, 3e-39, 5e36):
        g = update(72, 96, 1.0).bfloat16()
        w, m = torch.zeros((72, 96), device=DEV), torch.zeros((72, 96), device=DEV)
        step([bg.MuonTensor(w, g, m)], -1.0, 0.0, False, FIVE, products, torch.full((1,), scale, device=DEV))
        check_x(np64(w), np64(m), FIVE, products)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("products", [3, 1])
@pytest.mark.parametrize("o,i,rank", [(48, 64, 0), (70, 33, 2)])
def test_momentum_that_fades(o, i, rank, products, nesterov):
    """No gradient any more: m halves step by step through the subnormals to 0, and every step is the
    oracle's; a step of zeros changes nothing."""
    m, g = update(o, i, 1e-34, rank), torch.zeros((o, i), device=DEV)
    w = torch.zeros_like(m)
    t = [bg.MuonTensor(w, g, m)]
    for turn in range(60):
        w.zero_()
        step(t, -1.0, 0.5, nesterov, FIVE, products)
        if not bool(m.any()):
            break
        u = np64(m)
        if nesterov:                               # beta m, rounded to what fp32 holds of it
            u = (0.5 * u).astype(np.float32).astype(np.float64)
        if not u.any():
            assert not bool(w.any())
            continue
        check_x(np64(w), u, FIVE, products)
    assert 20 < turn < 59 and not bool(w.any())


def test_many_thin_matrices():
    """264 rows of 2^20, 64 iterations: 34 million tiles, counted matrix by matrix.

    Rows are their own singular direction.  The iteration has its fixed point at 1, but for what A's sum
    loses: 65,536 products are added one after the other and lose up to 2^-23 each, 0.8%, which raises the
    fixed point by half of that; X's entries and B round to 11 bits."""
    n, length = 264, 1 << 20
    gen = torch.Generator(device=DEV).manual_seed(1)
    g = torch.randn((n, length), generator=gen, device=DEV).bfloat16()
    w, m = torch.zeros((n, length), device=DEV), torch.zeros((n, length), device=DEV)
    step([bg.MuonTensor(w[k:k + 1], g[k:k + 1], m[k:k + 1]) for k in range(n)], -1.0, 0.0, False,
         [(1.5, -0.5, 0.0)] * 64, 1)
    for k in range(0, n, 8):
        x = g[k:k + 8].double()
        x = x / x.norm(dim=1, keepdim=True)
        off = (w[k:k + 8].double() - x).abs() - (2.0 ** -8 + 3 * 2.0 ** -11) * x.abs()
        assert float(off.max()) <= 2.0 ** -34


@pytest.mark.parametrize("products", [3, 1])
def test_columns_in_several_batches(products):
    """Rows of one element take 64 in the planes: eight such matrices are a batch."""
    grads = [update(1 << 20, 1, 1e-3, seed=k) for k in range(10)] + [update(40, 50, 1e-3)]
    w = [torch.zeros_like(g) for g in grads]
    step([bg.MuonTensor(a, g, torch.zeros_like(g)) for a, g in zip(w, grads)], -1.0, 0.0, False, FIVE, products)
    for k in (0, 7, 8, 9, 10):
        check_x(np64(w[k]), np64(grads[k]), FIVE, products)


def test_coefficients_without_a_square():
    """c = 0: A itself is held nowhere, so that |X| may be 10 on the way."""
    for k in ([(10.0, 0.0, 0.0), (0.1, 0.0, 0.0)], [(9.0, -2.0, 0.0), (0.25, 0.0, 0.0)]):
        for products in (3, 1):
            g = update(130, 200, 1e-3)
            w, m = torch.zeros_like(g), torch.zeros_like(g)
            step([bg.MuonTensor(w, g, m)], -1.0, 0.0, False, k, products)
            check_x(np64(w), np64(g), k, products)


def test_oracle_at_the_ends():
    """The oracle's own X does not depend on the update's size."""
    u = np64(update(30, 40, 1.0))
    x = orc.newton_schulz(u, FIVE)
    for f in (2.0 ** -120, 2.0 ** 100):
        assert np.abs(orc.newton_schulz(u * f, FIVE) - x).max() <= 1e-12
    ok()
