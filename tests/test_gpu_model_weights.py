"""The weights after steps of the small model, against Muon and AdamW in 64 bits.

Every step is taken again in 64 bits from the state before it and the step's own gradients (which
test_gpu_model_step holds against autograd).  Muon's tolerance is test_gpu_muon's; AdamW's step is off
by some 2e-6 of itself, or what a v below fp32's normal numbers leaves of it (|g| < 1e-18: a step of
1e-10 of the rate), and a weight takes two roundings more.
"""
import numpy as np
import pytest

import paper_2606_11660_gb300 as bg
from oracle import model_oracle, train_oracle
from tests.test_gpu_model_step import QUINTIC, Model
from tests.test_gpu_muon import U, np64, x_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,V,d", [(60, 97, 48), (400, 200, 128), (4400, 150, 100)])
def test_weights_of_steps(R, V, d):
    m = Model(R, V, d)
    for turn in range(4):
        W, E, mW, mE, vE = (np64(t).copy() for t in (m.W, m.E, m.mW, m.mE, m.vE))
        m.step()
        assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()
        g, size = np64(m.dW), 0.2 * d ** 0.5
        want, wm, x = model_oracle.muon_step(W, g, mW, 0.02, 0.95, True, QUINTIC, size, 0.1)
        assert np.all(np.abs(np64(m.mW) - wm) <= 6 * U * (np.abs(mW) + np.abs(g))), turn
        _, tol = x_error(0.95 * np64(m.mW) + 0.05 * g, QUINTIC, 3)
        entry = 8 * tol * max(1 / np.sqrt(x.size), np.abs(x).max() / np.linalg.norm(x))
        off = np.abs(np64(m.W) - want)
        assert np.all(off <= 0.02 * size * (entry + 4 * U * np.abs(x)) + 6 * U * np.abs(W)), (turn, off.max())
        # the step itself is far larger than what is allowed
        assert np.abs(want - W).max() > 1e3 * off.max()
        g = np64(m.dE).reshape(-1)
        want, wm, wv = train_oracle.adamw(E.reshape(-1), g, mE, vE, 1e-3, 0.9, 0.99, 1e-8, 1, 0.0)
        assert np.all(np.abs(np64(m.mE) - wm) <= 6 * U * (np.abs(mE) + np.abs(g)) + 1e-44), turn
        assert np.all(np.abs(np64(m.vE) - wv) <= 8 * U * (np.abs(vE) + g * g) + 1e-44), turn
        up = np.abs(want - E.reshape(-1))
        off = np.abs(np64(m.E).reshape(-1) - want)
        assert np.all(off <= 2e-6 * up + 1e-13 + 2 * U * np.abs(want)), (turn, off.max())
