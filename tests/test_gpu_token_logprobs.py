"""GPU parity of the token log-probabilities and their backward pass against the fp64 oracle.

Tolerances, from the roundings in the path: z = x / tau is rounded twice and
z - lse once, each 2^-24 of |z| or |lse|, and the sums' relative error stays
below 1e-6 with trees of fp32 sums, so a log-probability is off by at most
some 1e-6 (2 max|z| + 8); a probability is off by that much relatively.  A
16-bit output adds its half unit (2^-8 bf16, 2^-11 f16 of the value, 2^-25
for f16 below its normal range).
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN, INF = float("nan"), float("inf")
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 1e-42, torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}


def tol_of(x, tau):
    z = np.abs(x[np.isfinite(x) & (np.abs(x) < 1e30)]) / tau
    return 1e-6 * (2 * (z.max() if z.size else 0.0) + 8)


def logits(R, V, dtype, pad=0, seed=0, scale=3.0, offset=0):
    g = torch.Generator().manual_seed(seed)
    flat = torch.empty(R * (V + pad) + offset, dtype=dtype, device=DEV)
    x = flat[offset:].view(R, V + pad)[:, :V]
    x.copy_((scale * torch.randn((R, V), generator=g)).to(dtype))
    t = torch.randint(0, V, (R,), generator=g)
    return x, t.to(DEV)


def forward(x, t, tau, entropy=True):
    R = x.shape[0]
    out = [torch.full((R,), 7.0, device=DEV) for _ in range(3 if entropy else 2)]
    bg.bergson_token_logprobs(x, t, tau, *out)
    return [o.cpu().double().numpy() for o in out]


def np64(x):
    return x.detach().cpu().double().numpy()


def check_forward(x, t, tau):
    logp, lse, ent = forward(x, t, tau)
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()
    want = orc.token_logprobs(np64(x), t.tolist(), tau)
    tol = tol_of(np64(x), tau)
    for got, w in zip((logp, lse, ent), want):
        np.testing.assert_allclose(got, w, rtol=1e-6, atol=tol)
    return logp, lse, ent


def check_backward(x, t, tau, w, h, in_place=False, pad=0, offset=0):
    R, V = x.shape
    ref = np64(x)
    lse, ent = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    bg.bergson_token_logprobs(x, t, tau, torch.empty(R, device=DEV), lse, ent)
    if in_place:
        dx = x
    else:
        flat = torch.full((R * (V + pad) + offset + 16,), 7.0, dtype=x.dtype, device=DEV)
        dx = flat[offset:offset + R * (V + pad)].view(R, V + pad)[:, :V]
    wd = None if w is None else torch.tensor(w, dtype=torch.float32, device=DEV)
    hd = None if h is None else torch.tensor(h, dtype=torch.float32, device=DEV)
    bg.bergson_token_logprobs_backward(x, t, tau, lse, ent, wd, hd, dx)
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()
    w64 = np.zeros(R) if w is None else np64(wd)
    h64 = np.zeros(R) if h is None else np64(hd)
    want = orc.token_logprobs_backward(ref, t.tolist(), tau, w64, h64)
    got = np64(dx)
    # the terms' sizes before they cancel
    tol = tol_of(ref, tau)
    p = np.zeros_like(ref)
    lse64 = orc.token_logprobs(ref, t.tolist(), tau)[1]
    for r in range(R):
        if t[r] >= 0 and np.isfinite(lse64[r]):
            p[r] = np.exp(ref[r] / tau - lse64[r])
            p[r, t[r]] += 1
    logq = np.where(p > 0, np.abs(np.log(np.maximum(p, 1e-300))), 0.0)
    size = (np.abs(w64)[:, None] * p + np.abs(h64)[:, None] * p * (logq + 12)) / tau
    bound = (tol + 4e-7) * size + HALF_UNIT[x.dtype] * np.abs(want) + SMALLEST[x.dtype]
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)
    if not in_place and pad:
        assert torch.all(flat[offset:offset + R * (V + pad)].view(R, V + pad)[:, V:] == 7.0)
    if not in_place:
        assert torch.all(flat[:offset] == 7.0) and torch.all(flat[offset + R * (V + pad):] == 7.0)
    return got


SHAPES = [(1, 1), (3, 2), (2, 7), (5, 31), (4, 33), (70, 96), (9, 257), (3, 1000), (2, 2049),
          (33, 4099), (3, 8191), (2, 16_391), (2, 50_257), (1, 131_072), (1, 262_147), (160, 5000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", SHAPES)
def test_forward_shapes(R, V, dtype):
    x, t = logits(R, V, dtype, seed=R * 7 + V)
    check_forward(x, t, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", SHAPES)
def test_backward_shapes(R, V, dtype):
    x, t = logits(R, V, dtype, seed=R * 5 + V)
    g = np.random.default_rng(V)
    w, h = g.normal(size=R), 0.1 * g.normal(size=R)
    check_backward(x, t, 1.0, w, None)
    check_backward(x, t, 0.7, w, h)
    check_backward(x, t, 1.0, None, h)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (5, 3), (8, 0), (0, 1), (13, 7)])
@pytest.mark.parametrize("V", [200, 4097, 40_001])
def test_strides_and_starts(V, pad, offset, dtype):
    x, t = logits(3, V, dtype, pad=pad, offset=offset, seed=V + pad)
    check_forward(x, t, 1.3)
    w = np.array([1.0, -0.5, 2.0])
    check_backward(x, t, 1.3, w, w * 0.1, pad=2, offset=offset)
    check_backward(x, t, 1.3, w, None, pad=pad, offset=offset)
    check_backward(x, t, 1.3, w, w * 0.1, in_place=True)


@pytest.mark.parametrize("V", [40, 3000, 70_000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_entries(V, dtype):
    x, t = logits(8, V, dtype, seed=V)
    low = torch.finfo(dtype).min
    x[0, V // 2:] = -INF
    x[1, :V // 2] = -INF                          # the first entries seen are empty
    x[2, 1:] = -INF                               # one entry left
    x[3] = -INF                                   # none
    x[4, V // 3:] = low                           # the type's lowest value as a mask
    x[5] = low                                    # ... over a whole row: an even distribution
    x[6, ::2] = low
    t[0], t[1], t[2], t[3], t[4], t[5] = 1, V - 1, 0, 2, 0, 3
    t[6] = 1
    t[7] = 5
    logp, lse, ent = check_forward(x, t, 1.0)
    assert logp[2] == 0.0 and ent[2] == 0.0
    assert logp[3] == -INF and lse[3] == -INF and ent[3] == 0.0
    assert abs(logp[5] + np.log(V)) < 1e-5 * np.log(V) + 1e-6 and abs(ent[5] - np.log(V)) < 2e-5
    keep = [0, 1, 2, 3, 4, 6, 7]                  # row 5's lse is its lowest value again
    w = np.linspace(0.5, 2, 7)
    got = check_backward(x[keep].contiguous(), t[keep], 1.0, w, -0.1 * w)
    assert np.all(got[3] == 0.0) and np.all(np.isfinite(got))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_lowest_values_get_no_gradient(dtype):
    """Their lse cannot hold log V beside the lowest value, so p is not in it."""
    x, t = logits(2, 5000, dtype)
    x[0] = torch.finfo(dtype).min
    lse = torch.tensor(forward(x, t, 1.0)[1], dtype=torch.float32, device=DEV)
    dx = torch.full_like(x, 7.0)
    bg.bergson_token_logprobs_backward(x, t, 1.0, lse, None, torch.ones(2, device=DEV), None, dx)
    assert torch.all(dx[0] == 0) and torch.any(dx[1] != 0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_target_that_is_masked(dtype):
    x, t = logits(2, 300, dtype)
    x[:, 10] = -INF
    t[:] = 10
    logp, _, _ = forward(x, t, 1.0)
    assert np.all(logp == -INF)
    check_backward(x, t, 1.0, np.array([1.0, 2.0]), None)


@pytest.mark.parametrize("V", [50, 5000, 140_001])
def test_rows_left_out_are_not_read(V):
    x, t = logits(4, V, torch.bfloat16, seed=3)
    x[1] = NAN
    x[3] = INF
    t[1] = t[3] = -100
    logp, lse, ent = forward(x, t, 1.0)
    for o in (logp, lse, ent):
        assert o[1] == 0.0 and o[3] == 0.0 and np.all(np.isfinite(o))
    dx = torch.full_like(x, 7.0)
    ones = torch.ones(4, device=DEV)
    bg.bergson_token_logprobs_backward(x, t, 1.0, torch.tensor(lse, dtype=torch.float32, device=DEV),
                                       None, ones, None, dx)
    assert torch.all(dx[1] == 0) and torch.all(dx[3] == 0) and torch.all(torch.isfinite(dx))
    # no gradient asks for a row's logits
    x[0] = NAN
    ones[0] = 0.0
    bg.bergson_token_logprobs_backward(x, t, 1.0, torch.tensor(lse, dtype=torch.float32, device=DEV),
                                       None, ones, None, dx)
    assert torch.all(dx[0] == 0)


@pytest.mark.parametrize("V", [64, 3001, 90_000])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_nan_and_inf_show(V, bad):
    x, t = logits(3, V, torch.float32)
    x[1, V // 2] = bad
    logp, lse, ent = forward(x, t, 1.0)
    assert np.all(np.isnan([logp[1], lse[1], ent[1]]))
    assert np.all(np.isfinite([logp[0], logp[2], lse[0], ent[2]]))


def test_target_past_the_vocabulary_is_reported():
    x, t = logits(3, 100, torch.float32)
    t[1] = 100
    logp, lse, ent = forward(x, t, 1.0)
    assert np.isnan(logp[1]) and np.isfinite(lse[1]) and np.isfinite(logp[0])
    assert bg.bergson_sync_status() == bg.BERGSON_EINVAL
    assert "target" in bg.bergson_last_error()
    dx = torch.zeros_like(x)
    bg.bergson_token_logprobs_backward(x, t, 1.0, torch.zeros(3, device=DEV), None,
                                       torch.ones(3, device=DEV), None, dx)
    assert torch.all(torch.isnan(dx[1])) and torch.all(torch.isfinite(dx[0]))
    assert bg.bergson_sync_status() == bg.BERGSON_EINVAL
    assert bg.bergson_sync_status() == bg.BERGSON_OK


def test_large_magnitudes_and_a_late_maximum():
    """Rising logits (each new one the largest), a maximum at the very end, and sizes near 1e4."""
    V = 20_000
    x = torch.stack([torch.linspace(-50, 50, V), torch.linspace(50, -50, V),
                     torch.cat([torch.zeros(V - 1), torch.tensor([80.0])]),
                     torch.linspace(0, 1, V) + 1e4]).to(DEV)
    t = torch.tensor([V - 1, 0, V - 1, 7], device=DEV)
    check_forward(x, t, 1.0)
    check_forward(x, t, 0.5)


@pytest.mark.parametrize("V", [37, 700, 5000])
def test_gradient_against_differences(V):
    """<dx, u> against central differences of the fp64 objective along u."""
    x, t = logits(3, V, torch.float32, seed=V, scale=1.5)
    g = np.random.default_rng(V)
    w, h = g.normal(size=3), g.normal(size=3)
    got = check_backward(x, t, 0.8, w, h)
    w, h = np.float32(w).astype(np.float64), np.float32(h).astype(np.float64)
    u = g.normal(size=(3, V))

    def objective(step):
        logp, _, ent = orc.token_logprobs(np64(x) + step * u, t.tolist(), 0.8)
        return (w * logp).sum() + (h * ent).sum()
    eps = 1e-5
    diff = (objective(eps) - objective(-eps)) / (2 * eps)
    # fp32 gradient: 1e-5 of the product's size; the difference: eps^2 and 1e-15 / eps
    size = np.linalg.norm(got) * np.linalg.norm(u) / np.sqrt(u.size) + np.abs(got * u).sum()
    assert abs(diff - (got * u).sum()) <= 2e-5 * size + 1e-8


def test_same_bits_every_time_and_on_another_stream():
    x, t = logits(37, 30_011, torch.bfloat16)
    a = forward(x, t, 1.0)
    b = forward(x, t, 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = [torch.empty(37, device=DEV) for _ in range(3)]
    bg.bergson_token_logprobs(x, t, 1.0, *out, stream=side)
    side.synchronize()
    for u, v, w in zip(a, b, out):
        assert np.array_equal(u, v) and np.array_equal(u, np64(w))
    only = forward(x, t, 1.0, entropy=False)
    np.testing.assert_allclose(only[0], a[0], atol=1e-5)


def test_rows_past_32_bit_offsets():
    """Row starts beyond 2^31 elements; only the last rows are live."""
    V = 131_072
    R = (1 << 31) // V + 3
    x = torch.empty((R, V), dtype=torch.bfloat16, device=DEV)
    part, tp = logits(2, V, torch.bfloat16, seed=11)
    x[R - 2:] = part
    t = torch.full((R,), -1, dtype=torch.int64, device=DEV)
    t[R - 2:] = tp
    logp, lse, ent = forward(x, t, 1.0)
    want = forward(part, tp, 1.0)
    for got, w in zip((logp, lse, ent), want):
        assert np.all(got[:R - 2] == 0) and np.allclose(got[R - 2:], w, atol=2e-5)
    w = torch.ones(R, device=DEV)
    lse_d = torch.tensor(lse, dtype=torch.float32, device=DEV)
    bg.bergson_token_logprobs_backward(x, t, 1.0, lse_d, None, w, None, x)
    dx = torch.empty_like(part)
    bg.bergson_token_logprobs_backward(part, tp, 1.0, lse_d[R - 2:].contiguous(), None,
                                       w[:2].contiguous(), None, dx)
    assert torch.equal(x[R - 2:], dx)
    assert not torch.any(x[::997][:-1])
    assert bg.bergson_sync_status() == bg.BERGSON_OK


def test_no_rows():
    x = torch.empty((0, 8), device=DEV)
    e = torch.empty(0, device=DEV)
    bg.bergson_token_logprobs(x, torch.empty(0, dtype=torch.int64, device=DEV), 1.0, e, e, e)
    bg.bergson_token_logprobs_backward(x, torch.empty(0, dtype=torch.int64, device=DEV), 1.0, e, e,
                                       e, e, x)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", [(1300, 3001), (1217, 2561)])
def test_many_rows_of_middling_length(R, V, dtype):
    """Rows of 4 to 16 KB, enough of them to go to warps."""
    x, t = logits(R, V, dtype, seed=V)
    t[::7] = -1
    check_forward(x, t, 0.9)
    g = np.random.default_rng(R)
    w = g.normal(size=R)
    w[::5] = 0.0
    check_backward(x, t, 0.9, w, None)
    check_backward(x, t, 0.9, w, 0.1 * w)


def check_gradient_about_top(x, t, tau, w, h, in_place=False, pad=0):
    """The backward pass where lse is far from 0: what counts are the differences from
    the row's largest logit, so the bound goes by those and not by the logits' size."""
    R, V = x.shape
    ref = np64(x)
    lse, ent = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    bg.bergson_token_logprobs(x, t, tau, torch.empty(R, device=DEV), lse, ent)
    dx = x if in_place else torch.full((R, V + pad), 7.0, dtype=x.dtype, device=DEV)[:, :V]
    wd, hd = (None if y is None else torch.tensor(y, dtype=torch.float32, device=DEV) for y in (w, h))
    bg.bergson_token_logprobs_backward(x, t, tau, lse, ent, wd, hd, dx)
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()
    w64, h64 = (np.zeros(R) if y is None else np64(y) for y in (wd, hd))
    # the fp64 oracle's own lse rounds at 2^-53 |z|, so it gets the rows about their tops
    top = np.max(np.where(np.isfinite(ref), ref, -INF), axis=1, keepdims=True)
    want = orc.token_logprobs_backward(ref - top, t.tolist(), tau, w64, h64)
    z = (ref - top) / tau
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    logq = np.where(p > 0, np.abs(np.log(np.maximum(p, 1e-300))), 0.0)
    p[np.arange(R), t.tolist()] += 1
    tol = 1e-6 * (2 * np.where(p > 1e-30, np.abs(z), 0).max() + 8)
    size = (np.abs(w64)[:, None] * p + np.abs(h64)[:, None] * p * (logq + 12)) / tau
    bound = (tol + 4e-7) * size + HALF_UNIT[x.dtype] * np.abs(want) + SMALLEST[x.dtype]
    got = np64(dx)
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,pad", [(40, 0), (3000, 3), (70_001, 0), (70_000, 5)])
def test_gradients_where_lse_cannot_hold_the_sum(V, pad, dtype):
    """Rows of one large value, as a finite mask over all of them leaves (an even distribution), rows
    at a large common offset, and a large top above others: lse's last digit is larger than log V."""
    low = -6e4 if dtype == torch.float16 else -1e9
    g = np.random.default_rng(V)
    for in_place in (False, True):
        for w, h in ((g.normal(size=6), None), (g.normal(size=6), 0.1 * g.normal(size=6))):
            x, t = logits(6, V, dtype, seed=V)
            x[0] = low
            x[1] = -low
            x[2] = low
            x[2, V // 2:] = -INF
            t[2] = 1
            x[3] = -low / 4
            x[3, ::3] = -low
            x[4] = (torch.randn(V, device=DEV) * 3 + 9000).to(dtype)
            check_gradient_about_top(x, t, 1.0, w, h, in_place, pad)
            check_gradient_about_top(logits(6, V, dtype, seed=1)[0] * 0 + low / 2, t, 0.5, w, h)


def test_many_rows_where_lse_cannot_hold_the_sum():
    """... on warps, beside rows of ordinary size."""
    x, t = logits(1300, 3001, torch.float32, seed=4)
    x[::2] += 2.0 ** 20
    w = np.random.default_rng(0).normal(size=1300)
    check_gradient_about_top(x, t, 1.0, w, 0.1 * w)
    check_gradient_about_top(x, t, 1.0, w, None, in_place=True)


@pytest.mark.parametrize("V", [301, 20_001])
def test_rows_at_moderate_offsets(V):
    """Offsets of 600 to 3000, where half of lse's last digit, up to 1.2e-4, would be p's error."""
    x, t = logits(120, V, torch.float32, seed=V)
    x += torch.linspace(600, 3000, 120, device=DEV)[:, None]
    w = np.random.default_rng(0).normal(size=120)
    check_gradient_about_top(x, t, 1.0, w, None)
    check_gradient_about_top(x, t, 1.0, w, 0.1 * w)
