"""The fp64 definitions of the training-side operators against differences and closed forms (CPU)."""
import numpy as np
import pytest

from oracle import train_oracle as orc


def along(f, eps=1e-6):
    return (f(eps) - f(-eps)) / (2 * eps)


@pytest.mark.parametrize("tau", [1.0, 0.6])
def test_logprob_gradients(tau):
    r = np.random.default_rng(0)
    x, u = r.normal(size=(4, 30)) * 2, r.normal(size=(4, 30))
    x[1, 5:9] = -np.inf
    t, w, h = [3, 1, -1, 29], r.normal(size=4), r.normal(size=4)
    d = orc.token_logprobs_backward(x, t, tau, w, h)

    def f(e):
        lp, _, ent = orc.token_logprobs(x + e * u, t, tau)
        return (w * lp + h * ent).sum()
    assert abs(along(f) - (d * u).sum()) < 1e-7
    assert np.all(d[2] == 0) and np.all(d[1, 5:9] == 0)


def test_logprobs_closed_forms():
    lp, lse, ent = orc.token_logprobs(np.zeros((1, 8)), [2], 1.0)
    assert np.allclose([lp[0], lse[0], ent[0]], [-np.log(8), np.log(8), np.log(8)])
    lp, lse, ent = orc.token_logprobs(np.full((1, 3), -np.inf), [0], 1.0)
    assert lp[0] == -np.inf and lse[0] == -np.inf and ent[0] == 0


@pytest.mark.parametrize("reduction", ["token_mean", "seq_mean", "sum_norm"])
def test_policy_gradients(reduction):
    r = np.random.default_rng(1)
    old = -r.exponential(size=(3, 20))
    logp, ref, ent = old + 0.3 * r.normal(size=(3, 20)), old + 0.1, r.random((3, 20))
    adv, mask = r.normal(size=3), r.random((3, 20)) < 0.6
    u, u2 = r.normal(size=(3, 20)), r.normal(size=(3, 20))

    def f(e):
        return orc.policy_loss(logp + e * u, old, ref, ent + e * u2, adv, mask, 0.2, 0.3, 0.1, 0.02,
                               reduction, 7.0)["loss"]
    o = orc.policy_loss(logp, old, ref, ent, adv, mask, 0.2, 0.3, 0.1, 0.02, reduction, 7.0)
    assert abs(along(f) - (o["d"] * u).sum() - (o["dh"] * u2).sum()) < 1e-8
    assert np.isclose(o["seq"].sum(), o["loss"])


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("mean", [False, True])
def test_preference_gradients(kind, mean):
    r = np.random.default_rng(2)
    logp, ref = -r.exponential(size=(6, 15)), -r.exponential(size=(6, 15))
    mask, u = r.random((6, 15)) < 0.7, r.normal(size=(6, 15))

    def f(e):
        return orc.preference_loss(logp + e * u, ref, mask, kind, 0.3, 0.1, 0.2, mean)["loss"]
    o = orc.preference_loss(logp, ref, mask, kind, 0.3, 0.1, 0.2, mean)
    assert abs(along(f) - (o["d"] * u).sum()) < 1e-7


def test_codes_round_trip_and_are_unbiased():
    r = np.random.default_rng(3)
    for second in (False, True):
        levels = orc.code_values(second)
        assert np.all(np.diff(levels[:128]) > 0) and levels[255 if second else 127] == 1.875
        x = np.float32(levels[r.permutation(256)] * 0.25)
        x = x if second else np.concatenate([x])
        codes, scales = orc.quantise(x, second, np.zeros(256))
        assert np.allclose(orc.dequantise(codes, scales, second), x)
        y = np.full(256, 0.3, np.float32)
        y[0] = 1.875
        got = [orc.dequantise(*orc.quantise(y, second, r.integers(0, 65536, 256)), second)[1:].mean()
               for _ in range(200)]
        assert abs(np.mean(got) - 0.3) < 4 * 0.03125 / 2 / np.sqrt(200 * 255) + 1e-6


def test_chance_is_spread_evenly():
    c = orc.chance(4096, 1, 2, 3)
    assert c.min() >= 0 and c.max() < 65536 and abs(c.mean() - 32767.5) < 4 * 18919 / 64
    assert not np.array_equal(c, orc.chance(4096, 1, 3, 3))


def test_adamw_first_step_is_lr_sign():
    p, m, v = orc.adamw(np.zeros(3), np.array([2.0, -0.5, 0.0]), np.zeros(3), np.zeros(3), 0.1, 0.9,
                        0.99, 1e-12, 1, 0.0)
    assert np.allclose(p, [-0.1, 0.1, 0.0])


def test_factors_have_the_row_and_column_sums():
    v = np.random.default_rng(4).random((7, 5))
    r, c = orc.factor_moments(v, 2.0, 1e-3)
    want = 2 * v + 1e-3
    approx = r[:, None] * c[None]
    assert np.allclose(approx.sum(1), want.sum(1)) and np.allclose(approx.sum(0), want.sum(0))


def lowest_step(y):
    """The mean that a first moment of y (over the scale) keeps: code 0 is zero, but has the place of 2^-15."""
    low, first = 2.0 ** -15, 1.125 * 2.0 ** -15
    return y if y >= first else first * max(0.0, (y - low) / (first - low))


@pytest.mark.parametrize("y", [2.0 ** -17, 2.0 ** -15, 1.06 * 2.0 ** -15, 1.2 * 2.0 ** -15, 3.3 * 2.0 ** -15])
def test_small_first_moments(y):
    """The mean over all 2^16 chances: unbiased from the smallest code (1.125 * 2^-15) on; below it at most
    2^-15 is lost."""
    x = np.full(256, y, np.float32)
    x[0] = 1.875
    mean = 0.0
    for first in range(0, 65536, 255):
        rnd = np.minimum(first + np.arange(-1, 255), 65535)
        codes, scales = orc.quantise(x, False, rnd)
        live = (rnd >= first) & (first + np.arange(-1, 255) < 65536)
        mean += orc.dequantise(codes, scales, False)[live].sum() / 65536
    # 2^-16 of a code's step, and the scale's rounding (of y, times 9 where the step is steep)
    assert abs(mean - lowest_step(y)) <= 1.125 * 2.0 ** -31 + 9 * 2.0 ** -22 * y
    assert 0 <= y - mean + 2.0 ** -22 * y <= 2.0 ** -15 * (1 + 2.0 ** -20)
