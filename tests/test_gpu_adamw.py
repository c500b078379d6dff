"""GPU parity of the AdamW step against the fp64 oracle.

Tolerances: m and v take three and four fp32 operations (2^-24 each of terms
no larger than the sums of magnitudes); the step a division, a square root
and a few products (some 1e-6 of its size), a 16-bit parameter its half unit.
8-bit codes follow from the fp32 m and v exactly, so they are compared as codes
against the rule applied to m and v formed in fp32 with each operation rounded.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


def n64(x):
    return x.detach().cpu().double().numpy()


def make(n, p=torch.float32, g=torch.float32, master=False, eight=False, seed=0, offset=0, wd=0.1,
         lr_scale=1.0):
    """A tensor of n elements that starts `offset` elements into its buffers."""
    r = np.random.default_rng(seed)

    def dev(x, dtype):
        flat = torch.zeros(n + offset, dtype=dtype, device=DEV)
        flat[offset:] = torch.as_tensor(x).to(dtype).to(DEV)
        return flat[offset:]
    param = dev(0.5 * r.normal(size=n), p)
    grad = dev(1e-2 * r.normal(size=n) * np.exp(r.normal(size=n)), g)
    mm = 1e-2 * r.normal(size=n)
    vv = 1e-4 * r.exponential(size=n)
    mas = dev(n64(param) + 1e-4 * r.normal(size=n), torch.float32) if master else None
    if not eight:
        return bg.AdamWTensor(param, grad, dev(mm, torch.float32), dev(vv, torch.float32), mas,
                              lr_scale=lr_scale, weight_decay=wd)
    mc, ms = orc.quantise(np.float32(mm), False, np.zeros(n))
    vc, vs = orc.quantise(np.float32(vv), True, np.zeros(n))
    return bg.AdamWTensor(param, grad, dev(mc, torch.uint8), dev(vc, torch.uint8), mas,
                          torch.tensor(ms, device=DEV), torch.tensor(vs, device=DEV),
                          lr_scale=lr_scale, weight_decay=wd)


def snapshot(t):
    return {k: None if getattr(t, k) is None else getattr(t, k).clone()
            for k in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")}


def check(t, old, index, step, seed=0, gs=1.0, hyper=HYPER):
    """t after a step from `old`, as tensor `index` of the call."""
    lr, b1, b2, eps = (hyper[k] for k in ("lr", "beta1", "beta2", "eps"))
    eight = t.m_scale is not None
    g32 = np.float32(n64(old["grad"])) * np.float32(gs)
    if eight:
        m0 = np.float32(orc.code_values(False)[old["m"].cpu().numpy()]) * np.repeat(
            old["m_scale"].cpu().numpy(), 256)[:t.param.numel()]
        v0 = np.float32(orc.code_values(True)[old["v"].cpu().numpy()]) * np.repeat(
            old["v_scale"].cpu().numpy(), 256)[:t.param.numel()]
    else:
        m0, v0 = old["m"].cpu().numpy(), old["v"].cpu().numpy()
    w0 = n64(old["param"] if t.master is None else old["master"])
    wd32 = float(np.float32(t.weight_decay))
    p, m, v = orc.adamw(w0, g32.astype(np.float64), m0.astype(np.float64), v0.astype(np.float64),
                        lr * float(np.float32(t.lr_scale)), b1, b2, eps, step, wd32)
    ulp = 2.0 ** -23
    m_off = ulp * (np.abs(b1 * m0) + np.abs((1 - b1) * g32)) * 1.5
    v_off = ulp * v * 2.5
    if eight:
        m32 = m0 * np.float32(b1) + g32 * np.float32(1 - b1)
        v32 = v0 * np.float32(b2) + (g32 * g32) * np.float32(1 - b2)
        rnd = orc.chance(t.param.numel(), seed, step, index)
        for got_c, got_s, x, second in ((t.m, t.m_scale, m32, False), (t.v, t.v_scale, v32, True)):
            codes, scales = orc.quantise(x, second, rnd)
            assert np.array_equal(got_s.cpu().numpy(), scales)
            assert np.array_equal(got_c.cpu().numpy(), codes)
            out = torch.empty(t.param.numel(), device=DEV)
            bg.bergson_adamw_state_values(
                got_c, got_s, bg.BERGSON_MOMENT_SECOND if second else bg.BERGSON_MOMENT_FIRST, out)
            np.testing.assert_allclose(n64(out), orc.dequantise(codes, scales, second), rtol=1.2e-7,
                                       atol=1e-44)
    else:
        assert np.all(np.abs(n64(t.m) - m) <= m_off + 1e-45)
        assert np.all(np.abs(n64(t.v) - v) <= v_off + 1e-45)
    up = np.abs(p - w0)
    # m's own rounding, magnified where m is a small difference of large terms
    root = np.sqrt(v / (1 - b2 ** step)) + eps
    off = 4e-7 * (np.abs(w0) + up) + lr * abs(t.lr_scale) * (m_off / (1 - b1 ** step) / root + 2e-6 * up)
    wide = n64(t.param if t.master is None else t.master)
    half = HALF_UNIT[t.param.dtype] * np.abs(p) if t.master is None else 0.0
    assert np.all(np.abs(wide - p) <= off + half + 1e-7 * (t.param.dtype == torch.float16))
    if t.master is not None:
        assert torch.equal(t.param, t.master.to(t.param.dtype))


SIZES = [1, 2, 7, 31, 255, 256, 257, 511, 1000, 2048, 2049, 5003, 70_001]
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("p", DTYPES)
@pytest.mark.parametrize("g", DTYPES)
@pytest.mark.parametrize("master", [False, True])
def test_types(p, g, master, eight):
    ts = [make(n, p, g, master, eight, seed=n) for n in (1, 256, 777, 4096)]
    old = [snapshot(t) for t in ts]
    bg.bergson_adamw_step(ts, step=3, seed=5, **HYPER)
    for i, (t, o) in enumerate(zip(ts, old)):
        check(t, o, i, 3, 5)


@pytest.mark.parametrize("eight", [False, True])
def test_sizes_in_one_call(eight):
    ts = [make(n, torch.bfloat16, torch.bfloat16, n % 2 == 0, eight, seed=n, wd=0.01 * (n % 3),
               lr_scale=1 + n % 2) for n in SIZES]
    old = [snapshot(t) for t in ts]
    bg.bergson_adamw_step(ts, step=100, seed=9, **HYPER)
    for i, (t, o) in enumerate(zip(ts, old)):
        check(t, o, i, 100, 9)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("offset", [1, 2, 3, 8])
@pytest.mark.parametrize("p", DTYPES)
def test_starts_off_vector_boundaries(p, offset, eight):
    t = make(3001, p, p, True, eight, seed=offset, offset=offset)
    o = snapshot(t)
    bg.bergson_adamw_step([t], step=2, **HYPER)
    check(t, o, 0, 2)


@pytest.mark.parametrize("eight", [False, True])
def test_mixed_tensors_and_hundreds_of_them(eight):
    """More tensors than one launch's records, of mixed types, states and sizes."""
    r = np.random.default_rng(0)
    ts = []
    for i in range(700):
        ts.append(make(int(r.integers(1, 700)), DTYPES[i % 3], DTYPES[(i // 3) % 3], i % 2 == 0,
                       eight if i % 5 else not eight, seed=i, offset=i % 2))
    old = [snapshot(t) for t in ts]
    arr = bg.bergson_adamw_tensors(ts)
    bg.bergson_adamw_step(arr, step=11, seed=2 ** 63 + 5, **HYPER)
    for i in range(0, 700, 13):
        check(ts[i], old[i], i, 11, 2 ** 63 + 5)
    for i in (298, 299, 300, 301, 599, 600, 601, 699):
        check(ts[i], old[i], i, 11, 2 ** 63 + 5)


def test_empty_tensors_between_others():
    ts = [make(0), make(300, seed=1), make(0), make(5, seed=2)]
    old = [snapshot(t) for t in ts]
    bg.bergson_adamw_step(ts, step=1, **HYPER)
    check(ts[1], old[1], 1, 1)
    check(ts[3], old[3], 3, 1)
    bg.bergson_adamw_step([], step=1, **HYPER)


def test_first_step_from_zeros():
    """State zeros (codes and scales): p moves by lr times the gradient's sign."""
    hyper = dict(HYPER, eps=1e-15)                # far below every gradient but the zero
    for eight in (False, True):
        t = make(1000, eight=eight, wd=0.0)
        for x in (t.m, t.v, t.m_scale, t.v_scale):
            if x is not None:
                x.zero_()
        t.grad[5] = 0.0
        o = snapshot(t)
        bg.bergson_adamw_step([t], step=1, **hyper)
        check(t, o, 0, 1, hyper=hyper)
        moved = n64(t.param - o["param"])
        assert moved[5] == 0
        keep = np.arange(1000) != 5
        np.testing.assert_allclose(moved[keep], -1e-2 * np.sign(n64(o["grad"]))[keep], rtol=2e-3)


def test_gradient_scale_and_step_lengths():
    gs = torch.full((1,), 0.25, device=DEV)
    for step in (1, 2, 1000, 10 ** 7):
        t = make(900, torch.bfloat16, torch.bfloat16, True, True, seed=step % 97)
        o = snapshot(t)
        bg.bergson_adamw_step([t], step=step, seed=1, grad_scale=gs, **HYPER)
        check(t, o, 0, step, 1, gs=0.25)


def test_zero_betas_and_eps():
    hyper = dict(lr=1e-3, beta1=0.0, beta2=0.0, eps=0.0)
    t = make(500, wd=0.0)
    o = snapshot(t)
    bg.bergson_adamw_step([t], step=1, **hyper)
    np.testing.assert_allclose(n64(t.m), n64(o["grad"]), rtol=1e-6)
    np.testing.assert_allclose(n64(t.param - o["param"]), -1e-3 * np.sign(n64(o["grad"])), rtol=2e-4)


def test_blocks_of_extreme_values():
    """Zeros, one large value among tiny ones, values whose squares are below the normal range."""
    t = make(256 * 4, eight=True, wd=0.0)
    t.m.zero_(), t.v.zero_(), t.m_scale.zero_(), t.v_scale.zero_()
    t.grad[:256] = 0.0
    t.grad[256:512] = 1e-9
    t.grad[300] = 1e3
    t.grad[512:768] = 1e-21
    t.grad[768:] = 3e37 * torch.sign(t.grad[768:])
    t.grad[768:] = torch.clamp(t.grad[768:], -1e18, 1e18)
    o = snapshot(t)
    bg.bergson_adamw_step([t], step=1, **HYPER)
    check(t, o, 0, 1)
    assert torch.all(t.m[:256] == 0) and torch.all(t.v[:256] == 0) and t.m_scale[0] == 0
    assert torch.all(t.v[256:512] >= 1)           # a v > 0 never becomes 0
    assert torch.equal(t.param[:256], o["param"][:256])


def test_nan_stays_in_its_block():
    for eight in (False, True):
        t = make(1024, eight=eight)
        t.grad[300] = float("nan")
        o = snapshot(t)
        bg.bergson_adamw_step([t], step=2, **HYPER)
        p = n64(t.param)
        assert np.isnan(p[300]) and np.isfinite(np.delete(p, 300)).all()
        if eight:
            s = n64(t.m_scale)
            assert np.isnan(s[1]) and np.isfinite(s[[0, 2, 3]]).all()


def test_small_changes_are_not_lost():
    """With beta2 = 0.999 a code's step is far above one update of v; by chance the mean still follows."""
    n = 1 << 16
    t = make(n, eight=True, wd=0.0)
    v32 = torch.full((n,), 1.0)
    v32[::256] = 8.0                              # holds the block's scale
    codes, scales = orc.quantise(v32.numpy(), True, np.zeros(n))
    t.v.copy_(torch.tensor(codes)), t.v_scale.copy_(torch.tensor(scales))
    t.grad.fill_(3.0)
    t.grad[::256] = float(np.sqrt(8.0))
    inner = torch.ones(n, dtype=torch.bool, device=DEV)
    inner[::256] = False
    out = torch.empty(n, device=DEV)
    bg.bergson_adamw_state_values(t.v, t.v_scale, bg.BERGSON_MOMENT_SECOND, out)
    want = float(out[inner].double().mean())      # 1 takes the code below it
    for step in range(1, 41):
        bg.bergson_adamw_step([t], 0.0, 0.9, 0.999, 1e-8, step, seed=7)
        want = 0.999 * want + 0.001 * 9.0
    bg.bergson_adamw_state_values(t.v, t.v_scale, bg.BERGSON_MOMENT_SECOND, out)
    got = float(out[inner].double().mean())
    # 65,280 elements of independent error below a code's step (1/8): 4 sigma is 0.002
    assert abs(got - want) < 0.01, (got, want)


def test_same_bits_every_time_and_graph_replay():
    def fresh():
        return make(9001, torch.bfloat16, torch.bfloat16, True, True, seed=3)
    a, b, c = fresh(), fresh(), fresh()
    bg.bergson_adamw_step([a], step=5, seed=1, **HYPER)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    bg.bergson_adamw_step([b], step=5, seed=1, stream=side, **HYPER)
    graph = torch.cuda.CUDAGraph()
    arr = bg.bergson_adamw_tensors([c])
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        bg.bergson_adamw_step(arr, step=5, seed=1, **HYPER)
    graph.replay()
    torch.cuda.synchronize()
    for k in ("param", "master", "m", "v", "m_scale", "v_scale"):
        assert torch.equal(getattr(a, k), getattr(b, k))
        assert torch.equal(getattr(a, k), getattr(c, k))


def test_tensor_past_32_bit_offsets():
    """2^31 + 600 elements with 8-bit states: the last block against one of its own."""
    n = (1 << 31) + 600
    big = bg.AdamWTensor(torch.zeros(n, dtype=torch.bfloat16, device=DEV),
                         torch.zeros(n, dtype=torch.bfloat16, device=DEV),
                         torch.zeros(n, dtype=torch.uint8, device=DEV),
                         torch.zeros(n, dtype=torch.uint8, device=DEV),
                         m_scale=torch.zeros(-(-n // 256), device=DEV),
                         v_scale=torch.zeros(-(-n // 256), device=DEV))
    tail = (1 << 31)
    g = torch.randn(600, device=DEV).bfloat16()
    big.grad[tail:] = g
    bg.bergson_adamw_step([big], step=1, seed=4, **HYPER)
    moved = n64(big.param[tail:])
    np.testing.assert_allclose(moved, -1e-2 * np.sign(n64(g)), rtol=1e-2)
    assert not torch.any(big.param[tail - 4096:tail]) and not torch.any(big.m[:4096])
    out = torch.empty(600, device=DEV)
    bg.bergson_adamw_state_values(big.v[tail:], big.v_scale[tail // 256:], bg.BERGSON_MOMENT_SECOND, out)
    g32 = n64(g)
    assert np.all(np.abs(n64(out) - 0.01 * g32 ** 2) <= 0.126 * 0.01 * g32 ** 2 + 1e-10)


@pytest.mark.parametrize("second", [False, True])
def test_every_code_has_its_value(second):
    codes = torch.arange(256, dtype=torch.int32, device=DEV).to(torch.uint8).repeat(3)[:700]
    scale = torch.tensor([1.0, 0.5, 3.0], device=DEV)
    out = torch.empty(700, device=DEV)
    bg.bergson_adamw_state_values(codes, scale,
                                  bg.BERGSON_MOMENT_SECOND if second else bg.BERGSON_MOMENT_FIRST, out)
    want = orc.dequantise(codes.cpu().numpy(), scale.cpu().numpy(), second)
    assert np.array_equal(n64(out), want)


@pytest.mark.parametrize("offset", [0, 1])
def test_tiny_moments_without_eps(offset):
    """eps = 0: the step is m / sqrt(v) down to the smallest normal v (5 roundings and the two
    approximations' units: 1e-6), and 0 where both are 0."""
    hyper = dict(lr=1.0, beta1=0.9, beta2=0.99, eps=0.0)
    t = make(600, wd=0.0, offset=offset)
    v = 10.0 ** np.linspace(-37, -20, 600)
    t.v.copy_(torch.tensor(v)), t.m.copy_(torch.tensor(0.5 * np.sqrt(v)))
    t.param.zero_(), t.grad.zero_()
    t.m[7] = t.v[7] = 0.0
    m32, v32 = n64(t.m), n64(t.v)
    bg.bergson_adamw_step([t], step=100_000, **hyper)
    got = n64(t.param)
    assert got[7] == 0.0
    keep = np.arange(600) != 7
    want = -(0.9 * m32) / np.sqrt(0.99 * np.where(keep, v32, 1.0))
    np.testing.assert_allclose(got[keep], want[keep], rtol=1e-6)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("y", [2.0 ** -17, 2.0 ** -15, 1.06 * 2.0 ** -15, -1.2 * 2.0 ** -15])
def test_small_first_moments_keep_the_stated_mean(y, offset):
    """From the smallest code's value on, 1.125 * 2^-15 of the scale, m keeps its mean; 2^-15 and less
    becomes 0, and between them the smallest code is taken with a probability that rises from 0 to 1."""
    n = 256 * 512
    t = make(n, eight=True, wd=0.0, offset=offset)
    t.m.zero_(), t.v.zero_(), t.m_scale.zero_(), t.v_scale.zero_()
    t.grad.fill_(y)
    t.grad[::256] = 1.875                         # the scale is 1 within a unit
    hyper = dict(HYPER, beta1=0.0)
    o = snapshot(t)
    bg.bergson_adamw_step([t], step=1, seed=3, **hyper)
    check(t, o, 0, 1, seed=3, hyper=hyper)
    out = torch.empty(n, device=DEV)
    bg.bergson_adamw_state_values(t.m, t.m_scale, bg.BERGSON_MOMENT_FIRST, out)
    inner = torch.ones(n, dtype=torch.bool, device=DEV)
    inner[::256] = False
    low, first = 2.0 ** -15, 1.125 * 2.0 ** -15
    want = abs(y) if abs(y) >= first else first * max(0.0, (abs(y) - low) / (first - low))
    # 130,560 draws of 0 or `first`: half of that, over the root, is 1.4e-3 of it; 4 sigma
    assert abs(float(out[inner].double().mean()) - np.sign(y) * want) < 4 * 1.4e-3 * first
