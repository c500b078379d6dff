"""GPU parity of the policy and preference losses against the fp64 oracle.

Tolerances: a token's loss and gradient take a handful of fp32 operations
(exp and expm1 at 2 units, a difference of log-probabilities at half a unit
of their size), so they are held to 2e-6 of the sizes that enter; sums over
tokens are fp32 within 1024 and twice its bits above, held to 2e-6 of the sum of
magnitudes.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN, INF = float("nan"), float("inf")
REDUCTIONS = {"token_mean": bg.BERGSON_POLICY_TOKEN_MEAN, "seq_mean": bg.BERGSON_POLICY_SEQ_MEAN,
              "sum_norm": bg.BERGSON_POLICY_SUM_NORM}
KINDS = {"sigmoid": bg.BERGSON_PREFERENCE_SIGMOID, "hinge": bg.BERGSON_PREFERENCE_HINGE,
         "squared": bg.BERGSON_PREFERENCE_SQUARED}


def padded(x, pad, offset=0):
    """x on the device with rows `pad` elements apart, from element `offset` of its buffer."""
    x = torch.as_tensor(x)
    R, T = x.shape
    flat = torch.empty(R * (T + pad) + offset, dtype=x.dtype, device=DEV)
    flat.fill_(99)
    out = flat[offset:].view(R, T + pad)[:, :T]
    out.copy_(x)
    return out


def f32(x):
    return np.asarray(x, np.float32)


def policy_inputs(B, T, seed=0, token_adv=False, fill=0.7):
    g = np.random.default_rng(seed)
    old = f32(-g.exponential(size=(B, T)))
    logp = f32(old + 0.2 * g.normal(size=(B, T)))
    ref = f32(logp + 0.3 * g.normal(size=(B, T)))
    ent = f32(2 * g.random((B, T)))
    adv = f32(g.normal(size=(B, T) if token_adv else B))
    mask = g.random((B, T)) < fill
    return logp, old, ref, ent, adv, mask


def run_policy(logp, old, ref, ent, adv, mask, low=0.2, high=0.28, kl=0.05, ec=0.01,
               reduction="token_mean", norm=100.0, pad=0, offset=0, parts=True, stream=None):
    B, T = logp.shape
    dev = [None if x is None else padded(x, pad, offset) for x in (logp, old, ref, ent)]
    advd = torch.tensor(adv, device=DEV) if adv.ndim == 1 else padded(adv, pad, offset)
    md = None if mask is None else padded(mask.astype(np.uint8) * 3, pad, offset)
    loss, stats = torch.full((1,), NAN, device=DEV), torch.full((3,), NAN, device=DEV)
    seq = torch.full((B,), NAN, device=DEV)
    d, dh = padded(np.full((B, T), NAN, np.float32), pad), padded(np.full((B, T), NAN, np.float32), pad)
    ws = bg.workspace_tensor(bg.bergson_policy_loss_workspace(B, T), DEV)
    ws.fill_(0xFF)
    bg.bergson_policy_loss(dev[0], dev[1], dev[2], dev[3], advd, md, low, high, kl, ec,
                           REDUCTIONS[reduction], norm, loss, seq if parts else None,
                           stats if parts else None, d, dh if parts else None, ws, stream=stream)
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()
    out = dict(loss=loss, seq=seq, stats=stats, d=d, dh=dh)
    return {k: v.cpu().double().numpy() for k, v in out.items()}


def check_policy(inputs, low=0.2, high=0.28, kl=0.05, ec=0.01, reduction="token_mean", norm=100.0,
                 **kw):
    logp, old, ref, ent, adv, mask = inputs
    got = run_policy(*inputs, low=low, high=high, kl=kl, ec=ec, reduction=reduction, norm=norm, **kw)
    on = np.ones(logp.shape, bool) if mask is None else mask
    d64 = [None if x is None else np.asarray(x, np.float64) for x in (logp, old, ref, ent, adv)]
    want = orc.policy_loss(*d64, on, low, high, kl, ec, reduction, norm)
    B, T = logp.shape
    a = np.abs(np.where(on, np.broadcast_to(adv[:, None] if adv.ndim == 1 else adv, (B, T)), 0))
    size = np.where(on, (1 + np.abs(d64[0])) * (2 * a + 1), 0) * want["w"][:, None]
    # where the ratio is at a clip's edge within rounding either branch is right
    ratio = np.exp(np.where(on, d64[0] - d64[1], 0.0))
    edge = np.minimum(np.abs(ratio - 1 + low), np.abs(ratio - 1 - high)) < 1e-6
    assert np.all(np.abs(got["d"] - want["d"])[~edge] <= (2e-6 * size + 1e-45)[~edge])
    np.testing.assert_allclose(got["dh"], want["dh"], rtol=3e-7, atol=1e-45)
    assert np.all(np.abs(got["seq"] - want["seq"]) <= 2e-6 * size.sum(1) + 1e-45)
    assert abs(got["loss"][0] - want["loss"]) <= 2e-6 * size.sum() + 1e-45
    n = max(on.sum(), 1)
    assert got["stats"][2] == np.float32(on.sum())
    assert abs(got["stats"][1] - want["stats"][1]) <= (edge.sum() + 0.01) / n
    assert abs(got["stats"][0] - want["stats"][0]) <= 1e-6 * (1 + want["stats"][0]) + 1e-9
    return got, want


POLICY_SHAPES = [(1, 1), (1, 2), (2, 31), (3, 33), (8, 97), (17, 128), (5, 511), (4, 513), (2, 1025),
                 (300, 7), (64, 300), (1, 40_000), (3, 9001), (1000, 130), (2100, 33), (40, 4096)]


@pytest.mark.parametrize("reduction", REDUCTIONS)
@pytest.mark.parametrize("B,T", POLICY_SHAPES)
def test_policy_shapes(B, T, reduction):
    check_policy(policy_inputs(B, T, seed=B + T), reduction=reduction)


@pytest.mark.parametrize("reduction", REDUCTIONS)
@pytest.mark.parametrize("token_adv", [False, True])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 2), (4, 0)])
def test_policy_strides(pad, offset, token_adv, reduction):
    for B, T in ((7, 250), (3, 2000)):
        check_policy(policy_inputs(B, T, seed=pad, token_adv=token_adv), reduction=reduction,
                     pad=pad, offset=offset)


@pytest.mark.parametrize("reduction", REDUCTIONS)
@pytest.mark.parametrize("B,T", [(9, 60), (40, 3000)])
def test_policy_terms_left_out(B, T, reduction):
    logp, old, ref, ent, adv, mask = policy_inputs(B, T, seed=3)
    check_policy((logp, old, None, None, adv, None), kl=0.0, ec=0.0, reduction=reduction)
    check_policy((logp, old, ref, None, adv, mask), ec=0.0, reduction=reduction)
    check_policy((logp, old, None, ent, adv, mask), kl=0.0, reduction=reduction)
    full, _ = check_policy((logp, old, ref, ent, adv, mask), reduction=reduction)
    part = run_policy(logp, old, ref, ent, adv, mask, reduction=reduction, parts=False)
    assert part["loss"] == full["loss"] and np.array_equal(part["d"], full["d"])


@pytest.mark.parametrize("reduction", REDUCTIONS)
@pytest.mark.parametrize("B,T", [(6, 90), (9, 1500), (200, 700)])
def test_policy_masks(B, T, reduction):
    logp, old, ref, ent, adv, mask = policy_inputs(B, T, seed=5)
    mask[1] = False                               # an empty sequence
    mask[2] = True
    mask[3, 1:] = False
    got, _ = check_policy((logp, old, ref, ent, adv, mask), reduction=reduction)
    assert got["seq"][1] == 0 and np.all(got["d"][1] == 0)
    # whatever masked places hold
    junk = np.array([NAN, INF, -INF, -3.4e38], np.float32)
    for x in (logp, old, ref, ent):
        x[~mask] = junk[np.arange((~mask).sum()) % 4]
    again, _ = check_policy((logp, old, ref, ent, adv, mask), reduction=reduction)
    for k in got:
        assert np.array_equal(got[k], again[k])
    none, _ = check_policy((logp, old, ref, ent, adv, np.zeros_like(mask)), reduction=reduction)
    assert none["loss"] == 0 and np.all(none["d"] == 0) and np.all(none["stats"] == 0)


def test_policy_clipping_sides():
    """Ratios far outside the clip on either side, with advantages of either sign and zero."""
    logp = f32(np.tile([-1.0, -3.0, -2.0], (3, 1)))
    old = f32(np.full((3, 3), -2.0))
    adv = f32([2.0, -2.0, 0.0])
    none = np.ones((3, 3), bool)
    got, want = check_policy((logp, old, None, None, adv, none), kl=0.0, ec=0.0)
    assert got["d"][0, 0] == 0 and got["d"][1, 1] == 0
    assert got["d"][0, 1] < 0 < got["d"][1, 0] and got["stats"][1] == np.float32(2 / 9)


def test_policy_gradient_against_differences():
    logp, old, ref, ent, adv, mask = policy_inputs(5, 40, seed=9)
    for reduction in REDUCTIONS:
        got, _ = check_policy((logp, old, ref, ent, adv, mask), reduction=reduction)
        u = np.random.default_rng(1).normal(size=logp.shape) * mask
        u2 = np.random.default_rng(2).normal(size=logp.shape) * mask

        def loss(step):
            l64 = [np.asarray(x, np.float64) for x in (logp, old, ref, ent, adv)]
            return orc.policy_loss(l64[0] + step * u, l64[1], l64[2], l64[3] + step * u2, l64[4],
                                   mask, 0.2, 0.28, 0.05, 0.01, reduction, 100.0)["loss"]
        diff = (loss(1e-6) - loss(-1e-6)) / 2e-6
        along = (got["d"] * u).sum() + (got["dh"] * u2).sum()
        assert abs(diff - along) <= 5e-6 * (np.abs(got["d"] * u).sum() + 1e-2)


def test_policy_bits_repeat_and_streams():
    inputs = policy_inputs(37, 1501, seed=4)
    a = run_policy(*inputs)
    side = torch.cuda.Stream()
    b = run_policy(*inputs)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c = run_policy(*inputs)
    for k in a:
        assert np.array_equal(a[k], b[k]) and np.array_equal(a[k], c[k])


@pytest.mark.parametrize("B,T", [(0, 5), (4, 0)])
def test_policy_nothing(B, T):
    for reduction in REDUCTIONS:
        z = np.zeros((B, T), np.float32)
        got = run_policy(z, z, z, z, np.zeros(B, np.float32), np.ones((B, T), bool),
                         reduction=reduction)
        assert got["loss"] == 0 and np.all(got["seq"] == 0) and np.all(got["stats"] == 0)


def test_policy_rows_past_32_bit_offsets():
    """Row strides that put the last row beyond 2^31 elements."""
    T, ld = 600, 1 << 30
    logp, old, ref, ent, adv, mask = policy_inputs(3, T, seed=2)
    buf = torch.empty(2 * ld + T, device=DEV)
    wide = torch.as_strided(buf, (3, T), (ld, 1))
    wide.copy_(torch.tensor(logp))
    d = torch.empty((3, T), device=DEV)
    loss = torch.empty(1, device=DEV)
    ws = bg.workspace_tensor(bg.bergson_policy_loss_workspace(3, T), DEV)
    bg.bergson_policy_loss(wide, torch.tensor(old, device=DEV), None, None,
                           torch.tensor(adv, device=DEV), padded(mask.astype(np.uint8), 0), 0.2, 0.28,
                           0.0, 0.0, bg.BERGSON_POLICY_TOKEN_MEAN, 1.0, loss, None, None, d, None, ws)
    want = run_policy(logp, old, None, None, adv, mask, kl=0.0, ec=0.0)
    assert np.array_equal(d.cpu().double().numpy(), want["d"])


# ------------------------------------------------------------------ preference

def preference_inputs(P, T, seed=0, fill=0.7):
    g = np.random.default_rng(seed)
    logp = f32(-g.exponential(size=(2 * P, T)))
    ref = f32(logp + 0.1 * g.normal(size=(2 * P, T)))
    return logp, ref, g.random((2 * P, T)) < fill


def run_preference(logp, ref, mask, kind="sigmoid", beta=0.1, margin=0.0, eps=0.0, mean=False,
                   pad=0, offset=0):
    rows, T = logp.shape
    x = padded(logp, pad, offset)
    r = None if ref is None else padded(ref, pad, offset)
    m = None if mask is None else padded(mask.astype(np.uint8) * 255, pad, offset)
    loss = torch.full((1,), NAN, device=DEV)
    pair, rewards = torch.full((rows // 2,), NAN, device=DEV), torch.full((rows,), NAN, device=DEV)
    d = padded(np.full((rows, T), NAN, np.float32), pad)
    bg.bergson_preference_loss(x, r, m, KINDS[kind], beta, margin, eps, mean, loss, pair, rewards, d)
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()
    return {k: v.cpu().double().numpy()
            for k, v in dict(loss=loss, pair=pair, rewards=rewards, d=d).items()}


def check_preference(logp, ref, mask, kind="sigmoid", beta=0.1, margin=0.0, eps=0.0, mean=False,
                     **kw):
    got = run_preference(logp, ref, mask, kind, beta, margin, eps, mean, **kw)
    on = np.ones(logp.shape, bool) if mask is None else mask
    r64 = None if ref is None else ref.astype(np.float64)
    want = orc.preference_loss(logp.astype(np.float64), r64, on, kind, beta, margin, eps, mean)
    P = logp.shape[0] // 2
    n = np.maximum(on.sum(1), 1) if mean else np.ones(2 * P)
    gap = np.abs(np.where(on, logp, 0)) + (0 if ref is None else np.abs(np.where(on, ref, 0)))
    off = 2e-6 * gap.sum(1) / n * beta            # of a reward
    assert np.all(np.abs(got["rewards"] - want["rewards"]) <= off + 1e-7 * np.abs(want["rewards"]))
    dx = off[:P] + off[P:] + 2e-7 * (1 + abs(margin) + np.abs(want["rewards"][:P] - want["rewards"][P:]))
    # the loss moves with x by its slope, the gradient by its second derivative
    steep = {"sigmoid": 1.0, "hinge": 1.0, "squared": 2 / beta ** 2}[kind]
    x = want["rewards"][:P] - want["rewards"][P:] - margin
    slope = steep * (np.abs(x) + 1) if kind == "squared" else steep
    assert np.all(np.abs(got["pair"] - want["pair"]) <= dx * slope + 1e-6 * want["pair"] + 1e-30)
    assert abs(got["loss"][0] - want["loss"]) <= (dx * slope).mean() + 1e-6 * np.abs(want["pair"]).mean()
    second = steep if kind == "squared" else 0.25 if kind == "sigmoid" else 0.0
    kink = (np.abs(np.abs(x) - 1) < 1e-4) if kind == "hinge" else np.zeros(P, bool)
    ok = ~np.concatenate([kink, kink])
    bound = (np.concatenate([dx, dx]) * second * beta / P / n)[:, None] + 1e-6 * np.abs(want["d"]) + 1e-45
    assert np.all((np.abs(got["d"] - want["d"]) <= bound)[ok])
    assert np.all(got["d"][~on] == 0)
    return got, want


PAIR_SHAPES = [(1, 1), (1, 40), (2, 33), (3, 383), (8, 1000), (9, 513), (1, 30_001), (5, 9000),
               (200, 65), (700, 129), (160, 2100), (40, 5001)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("P,T", PAIR_SHAPES)
def test_preference_shapes(P, T, kind):
    logp, ref, mask = preference_inputs(P, T, seed=P + T)
    mean = kind == "squared"
    check_preference(logp, ref, mask, kind, 2.0 if mean else 0.05, 0.0, 0.0, mean)
    check_preference(logp, None, mask, kind, 2.0, 0.3, 0.1, True)
    check_preference(logp, ref, None, kind, 2.0 if mean else 0.05, 0.0, 0.2, mean)


@pytest.mark.parametrize("P,T", [(6, 200), (3, 5000), (400, 70)])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (4, 0), (7, 3)])
def test_preference_strides(P, T, pad, offset):
    logp, ref, mask = preference_inputs(P, T, seed=pad)
    check_preference(logp, ref, mask, pad=pad, offset=offset)


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("P,T", [(4, 100), (4, 20_000), (300, 90)])
def test_preference_masks(P, T, mean):
    logp, ref, mask = preference_inputs(P, T, seed=8)
    mask[0] = False
    mask[P + 1] = False
    mask[2] = mask[P + 2] = False                 # a pair without tokens: x = 0
    got, _ = check_preference(logp, ref, mask, mean=mean)
    assert abs(got["pair"][2] - np.log(2)) < 1e-6
    junk = np.array([NAN, INF, -INF, -3.4e38], np.float32)
    for x in (logp, ref):
        x[~mask] = junk[np.arange((~mask).sum()) % 4]
    again, _ = check_preference(logp, ref, mask, mean=mean)
    for k in got:
        assert np.array_equal(got[k], again[k])


@pytest.mark.parametrize("kind", KINDS)
def test_preference_extremes(kind):
    """Margins of hundreds either way: no overflow, saturated slopes."""
    logp = f32([[0.0], [-900.0], [-900.0], [0.0]])
    got, _ = check_preference(logp, None, None, kind, 1.0)
    assert np.all(np.isfinite(got["pair"])) and np.all(np.isfinite(got["d"]))
    check_preference(logp, None, None, kind, 1.0, eps=0.3)
    if kind == "sigmoid":
        assert got["pair"][0] == 0 and got["pair"][1] == 900


def test_preference_gradient_against_differences():
    logp, ref, mask = preference_inputs(5, 30, seed=2)
    for kind in KINDS:
        for mean in (False, True):
            got, _ = check_preference(logp, ref, mask, kind, 0.7, 0.2, 0.1, mean)
            u = np.random.default_rng(0).normal(size=logp.shape)

            def loss(step):
                return orc.preference_loss(logp + step * u, ref.astype(np.float64), mask, kind, 0.7,
                                           0.2, 0.1, mean)["loss"]
            diff = (loss(1e-6) - loss(-1e-6)) / 2e-6
            # both sides' roundings: fp32 gradients, and 1e-16 loss / step
            assert abs(diff - (got["d"] * u).sum()) <= 1e-5 * np.abs(got["d"] * u).sum() + 1e-8


def test_preference_bits_repeat():
    logp, ref, mask = preference_inputs(90, 3001, seed=1)
    a, b = run_preference(logp, ref, mask), run_preference(logp, ref, mask)
    for k in a:
        assert np.array_equal(a[k], b[k])


def test_preference_nothing():
    z = np.zeros((0, 5), np.float32)
    assert run_preference(z, None, None)["loss"] == 0
    got = run_preference(np.zeros((4, 0), np.float32), None, None)
    np.testing.assert_allclose(got["pair"], np.log(2), rtol=1e-6)


@pytest.mark.parametrize("reduction", REDUCTIONS)
@pytest.mark.parametrize("B,T", [(512, 256), (513, 256), (512, 257), (2, 65_536), (1, 131_073),
                                 (256, 300), (9800, 40), (20, 7000)])
def test_policy_at_the_launches_limits(B, T, reduction):
    """One launch of a cluster up to 512 segments of 256 tokens; longer segments from 9728 on."""
    check_policy(policy_inputs(B, T, seed=B), reduction=reduction)


@pytest.mark.parametrize("ref", [True, False])
@pytest.mark.parametrize("P,T", [(607, 512), (608, 512), (608, 513), (700, 511), (1500, 1), (8, 4096),
                                 (8, 4097), (9, 64), (2, 16_400), (608, 1024), (608, 1025), (650, 1001),
                                 (3, 30_003), (20, 12_349)])
def test_preference_at_the_launches_limits(P, T, ref):
    """A warp a pair, a cluster of pairs, a CTA and a cluster a pair."""
    logp, r, mask = preference_inputs(P, T, seed=P)
    check_preference(logp, r if ref else None, mask)


@pytest.mark.parametrize("T,pad", [(1001, 0), (997, 2), (4099, 4), (30, 1), (3, 0), (5, 2), (9, 7)])
def test_rows_off_vector_boundaries(T, pad):
    """Leading dimensions alike modulo 4 or 8: every row's vectors start elsewhere."""
    for B in (6, 700):
        check_policy(policy_inputs(B, T, seed=T), pad=pad)
        logp, ref, mask = preference_inputs(B, T, seed=T)
        check_preference(logp, ref, mask, pad=pad)
        check_preference(logp, None, None, pad=pad)


@pytest.mark.parametrize("reduction", REDUCTIONS)
@pytest.mark.parametrize("B,T", [(6, 90), (300, 700)])
def test_policy_watches_the_reference_without_the_term(B, T, reduction):
    """kl_coef = 0 with a reference: the mean of k is reported, the loss and gradients are those without."""
    logp, old, ref, ent, adv, mask = policy_inputs(B, T, seed=12)
    got, want = check_policy((logp, old, ref, ent, adv, mask), kl=0.0, reduction=reduction)
    assert want["stats"][0] > 0.01
    none = run_policy(logp, old, None, ent, adv, mask, kl=0.0, reduction=reduction)
    for k in ("loss", "seq", "d", "dh"):
        assert np.array_equal(got[k], none[k])
    ref[mask.nonzero()[0][0], mask.nonzero()[1][0]] = INF
    spoilt = run_policy(logp, old, ref, ent, adv, mask, kl=0.0, reduction=reduction)
    assert np.isnan(spoilt["stats"][0])           # exp(inf) - inf
    for k in ("loss", "seq", "d", "dh"):
        assert np.array_equal(spoilt[k], none[k])


@pytest.mark.parametrize("pad", [0, 1])
def test_policy_large_gaps_to_the_reference(pad):
    """Gaps of a quarter to 60, exact in fp32, weights and coefficient powers of two: the gradient is
    kl_coef (exp(gap) - 1) / n within exp's 2 units and three roundings."""
    gap = np.concatenate([np.linspace(-60, 60, 3841), np.linspace(-4, 4, 255)])
    gap = f32(np.round(gap * 1024) / 1024).reshape(4, 1024)
    logp = f32(-np.round(np.random.default_rng(0).exponential(size=gap.shape) * 1024) / 1024)
    ref = logp + gap
    assert np.array_equal(ref - logp, gap)
    got = run_policy(logp, logp, ref, None, f32(np.zeros(4)), None, kl=0.0625, ec=0.0, pad=pad)
    up = np.expm1(gap.astype(np.float64))
    big = np.abs(gap) >= 0.25
    off = np.abs(got["d"] + 0.0625 * up / 4096)
    assert np.all((off <= 7 * 2.0 ** -24 * (np.abs(up) + 1) * 0.0625 / 4096)[big])
    k = up - gap
    assert abs(got["stats"][0] - k.mean()) <= 2e-6 * k.mean()
    assert abs(got["loss"][0] - 0.0625 * k.mean()) <= 2e-6 * 0.0625 * k.mean()


@pytest.mark.parametrize("reduction", REDUCTIONS)
@pytest.mark.parametrize("B,T,pad", [(256, 256, 0), (257, 256, 0), (256, 1, 0), (257, 1, 0), (1, 65_536, 0),
                                     (1, 65_537, 0), (85, 700, 2), (86, 700, 2), (2431, 1025, 0),
                                     (2432, 1025, 0), (1650, 2500, 0), (2500, 1030, 1), (1621, 2049, 3),
                                     (4864, 1000, 4)])
def test_policy_forms_at_their_limits(B, T, pad, reduction):
    """One launch up to 256 segments of 256 tokens; segments of 1024 tokens from 4864 of them on, several
    a row, rows off 16-byte boundaries among them."""
    check_policy(policy_inputs(B, T, seed=B + 1, token_adv=pad == 1), reduction=reduction, pad=pad)
