"""GPU parity of the Muon step with the fp64 oracle.

Tolerances of the orthogonalised update X.  How roundings grow over the iterations
follows from the singular values, so they are carried through the iteration as the kernels
take it (A + h I, c (..)^2 + (a - c h^2) I with h = b / 2c, times X): with what an operand holds
rounded as the kernels round it (one fp16 plane, or two, of 1024 times the value), with
every product in fp32 (whose random roundings are those of sums of any order), and with
every product lowered by what sums rounded toward zero lose: n MMAs one after the
other round partial sums, half of the whole on average, by up to 2^-23 each, and n is 12 a
stage of 64 columns and 48 at most with two planes, 4 a stage with one.  The deviations
from the exact X, added, are allowed four times over in the Frobenius norm, and that norm's
eight times the share of an entry in any entry.  m takes two roundings; a weight two more and
half a unit of its type.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import model_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
QUINTIC = (3.4445, -4.7750, 2.0315)
FIVE = [QUINTIC] * 5


def np64(x):
    return x.detach().cpu().double().numpy()


def ok():
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()


def step(tensors, lr, beta, nesterov, k, products, gs=None):
    arr = bg.bergson_muon_tensors(tensors)
    ws = bg.workspace_tensor(bg.bergson_muon_step_workspace(arr, products), DEV)
    ws.fill_(255)                                  # NaN in every place that nothing was written to
    bg.bergson_muon_step(arr, lr, beta, nesterov, k, products, ws, gs)
    ok()


def hold(planes):
    def f(x):
        y = np.float64(1024) * x
        hi = y.astype(np.float16).astype(np.float64)
        lo = (y - hi).astype(np.float16).astype(np.float64) if planes == 2 else 0.0
        return (hi + lo) / 1024
    return f


def carried(u, k, hold=lambda x, inner=0: x, product=lambda p, inner: p):
    n = np.linalg.norm(u)
    x = hold(u / n if n > 0 else np.zeros_like(u))
    tall, one = u.shape[0] > u.shape[1], np.eye(min(u.shape))
    for a, b, c in k:
        y = x.T if tall else x
        g = product(y @ y.T, y.shape[1])
        h = b / (2 * c) if c != 0 else 0.0
        if c != 0:
            s = hold(g + h * one)
            q = hold(c * product(s @ s, len(s)) + (a - c * h * h) * one)
        else:
            q = hold(b * g + a * one)
        x = hold(product(x @ q if tall else q @ x, len(q)))
    return x


def x_error(u, k, products):
    """(X, its allowed deviation in the Frobenius norm)."""
    x = orc.newton_schulz(u, k)
    planes = 2 if products == 3 else 1

    def lowered(p, inner):
        stages = -(-inner // 64)
        return p * (1 - 0.5 * (min(12 * stages, 48) if planes == 2 else 4 * stages) * 2.0 ** -23)
    e = [np.linalg.norm(carried(u, k, **kw) - x) for kw in (
        dict(hold=hold(planes)), dict(product=lambda p, _: p.astype(np.float32).astype(np.float64)),
        dict(product=lowered))]
    n = np.linalg.norm(u)
    xf = (u / n if n > 0 else u).astype(np.float32)
    for a, b, c in np.float32(k):
        y = xf.T if u.shape[0] > u.shape[1] else xf
        g = y @ y.T
        q = b * g + c * (g @ g)
        xf = a * xf + (xf @ q if u.shape[0] > u.shape[1] else q @ xf)
    e.append(np.linalg.norm(xf - x))
    return x, 4 * sum(e) + 1e-7 * np.linalg.norm(x)


def check_x(got, u, k, products):
    x, tol = x_error(u, k, products)
    d = got - x
    assert np.linalg.norm(d) <= tol, (np.linalg.norm(d), tol, u.shape)
    assert np.abs(d).max() <= 8 * tol * max(1.0 / np.sqrt(d.size), np.abs(x).max() / np.linalg.norm(x)), (
        np.abs(d).max(), tol, u.shape, np.unravel_index(np.abs(d).argmax(), d.shape))
    return np.linalg.norm(d) / max(np.linalg.norm(x), 1e-300)


def gradient(o, i, seed=0, scale=1e-3):
    g = torch.Generator().manual_seed(seed + 1000 * o + i)
    r = min(4, o, i)
    x = torch.randn((o, i), generator=g) + 0.5 * torch.randn((o, r), generator=g) @ torch.randn(
        (r, i), generator=g)
    return (scale * x).to(DEV)


def orthogonalised(grads, k, products, beta=0.0, nesterov=False):
    """X of every gradient: the step's weights from zeros at lr 1."""
    w = [torch.zeros_like(g) for g in grads]
    m = [torch.zeros_like(g) for g in grads]
    step([bg.MuonTensor(a, g, b) for a, g, b in zip(w, grads, m)], -1.0, beta, nesterov, k, products)
    return w


SHAPES = [(1, 1), (1, 40), (40, 1), (24, 24), (33, 70), (70, 33), (64, 64), (128, 256), (256, 128),
          (256, 256), (257, 257), (264, 264), (300, 520), (520, 300), (640, 640), (513, 1000), (1000, 513),
          (792, 264), (264, 1056), (900, 900)]


@pytest.mark.parametrize("products", [3, 1])
@pytest.mark.parametrize("o,i", SHAPES)
def test_orthogonalisation(o, i, products):
    g = gradient(o, i)
    for k in ([QUINTIC], [QUINTIC] * 2, FIVE):
        x, = orthogonalised([g], k, products)
        check_x(np64(x), np64(g), k, products)


@pytest.mark.parametrize("products", [3, 1])
def test_shapes_together(products):
    """Matrices of several shapes and several of one, in one call."""
    grads = [gradient(o, i, seed) for seed in range(3) for o, i in [(70, 300), (300, 70), (260, 260), (33, 40)]]
    for x, g in zip(orthogonalised(grads, FIVE, products), grads):
        check_x(np64(x), np64(g), FIVE, products)


@pytest.mark.parametrize("products", [3, 1])
@pytest.mark.parametrize("shapes,count", [(6, 2), (30, 1), (3, 130)])
def test_many_matrices(shapes, count, products):
    """More shapes and matrices than a launch takes."""
    grads = [gradient(20 + 7 * s, 60 + s, c) for c in range(count) for s in range(shapes)]
    got = orthogonalised(grads, FIVE, products)
    for x, g in list(zip(got, grads))[::1 if shapes != 3 else 29]:
        check_x(np64(x), np64(g), FIVE, products)


@pytest.mark.parametrize("products", [3, 1])
@pytest.mark.parametrize("o,i", [(8, 70_000), (70_000, 8), (1100, 1300), (1300, 1100)])
def test_long_and_wide(o, i, products):
    """Sums over many stages; several rows of tiles, the last ones short."""
    g = gradient(o, i)
    k = [QUINTIC] * (2 if min(o, i) > 1000 else 5)
    x, = orthogonalised([g], k, products)
    check_x(np64(x), np64(g), k, products)


@pytest.mark.parametrize("products", [3, 1])
@pytest.mark.parametrize("o,i,count", [(1024, 1280, 10), (1290, 1030, 10), (700, 2000, 16)])
def test_enough_to_fill_the_device(o, i, count, products):
    """So many that tiles are at their widest, and a CTA pair has several."""
    grads = [gradient(o, i, c) for c in range(count)]
    k = [QUINTIC] * 2
    got = orthogonalised(grads, k, products)
    for z in (0, count - 1):
        check_x(np64(got[z]), np64(grads[z]), k, products)
    # the others against torch's products in 64 bits, to the bound of the last
    _, tol = x_error(np64(grads[-1]), k, products)
    for x, g in zip(got, grads):
        y = g.double() / torch.linalg.matrix_norm(g.double())
        y = y.t() if o > i else y
        for a, b, c in k:
            s = y @ y.t()
            y = a * y + (b * s + c * s @ s) @ y
        assert float(torch.linalg.matrix_norm(x.double() - (y.t() if o > i else y))) <= tol


def test_other_coefficients():
    g = gradient(200, 333)
    for k in ([(1.5, -0.5, 0.0)] * 12, [(2.0, -1.5, 0.5)] * 8, [QUINTIC, (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)],
              [(1.0, 0.0, 0.0)]):
        x, = orthogonalised([g], k, 3)
        check_x(np64(x), np64(g), k, 3)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e12, 1e25])
def test_sizes_of_gradients(scale):
    """The norm of any update that fp32 holds."""
    g = gradient(100, 140, scale=scale)
    x, = orthogonalised([g], FIVE, 3)
    check_x(np64(x), np64(g), FIVE, 3)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("p,g,master,o,i,offset,scaled", [
    (torch.bfloat16, torch.bfloat16, True, 96, 160, 0, True), (torch.bfloat16, torch.float32, False, 160, 96, 0, False),
    (torch.float16, torch.float16, False, 33, 70, 0, True), (torch.float32, torch.float32, False, 128, 128, 0, False),
    (torch.float32, torch.bfloat16, True, 128, 64, 0, True), (torch.float16, torch.float16, True, 272, 272, 1, True),
    (torch.float32, torch.float32, False, 80, 48, 1, False), (torch.bfloat16, torch.bfloat16, True, 70, 33, 3, True)])
def test_step(p, g, master, o, i, offset, scaled, nesterov):
    """Two steps of all the state, for types and starts; what lies around it keeps its value."""
    def place(x, dtype):
        flat = torch.full((offset + o * i + 40,), 7.0, dtype=dtype, device=DEV)
        v = flat[offset:offset + o * i].view(o, i)
        v.copy_(x)
        return flat, v
    rng = torch.Generator().manual_seed(o + i)
    fw, w = place(0.02 * torch.randn((o, i), generator=rng), p)
    fm, m = place(1e-3 * torch.randn((o, i), generator=rng), torch.float32)
    fs, ms = place(w.float(), torch.float32) if master else (None, None)
    gs = torch.full((1,), 0.7, device=DEV) if scaled else None
    f = float(gs) if scaled else 1.0
    lr, beta, os_, wd = 0.02, 0.95, 1.7, 0.1
    for turn in range(2):
        fg, grad = place(gradient(o, i, turn), g)
        w0, m0, g64 = np64(ms if master else w), np64(m), np64(grad) * f
        t = bg.MuonTensor(w, grad, m, ms, os_, wd, 0.5)
        step([t], lr, beta, nesterov, FIVE, 3, gs)
        want, wm, x = orc.muon_step(w0, g64, m0, lr * 0.5, beta, nesterov, FIVE, os_, wd)
        # beta and 1 - beta round to fp32 once too
        assert np.all(np.abs(np64(m) - wm) <= 6 * U * (np.abs(m0) + np.abs(g64))), "m"
        u = beta * np64(m) + (1 - beta) * g64 if nesterov else np64(m)
        _, tol = x_error(u, FIVE, 3)
        # u's own two roundings stand in x_error's fp32 part
        entry = 8 * tol * max(1 / np.sqrt(x.size), np.abs(x).max() / np.linalg.norm(x))
        tol_w = lr * 0.5 * os_ * (entry + 4 * U * np.abs(x)) + 4 * U * np.abs(w0)
        got = np64(ms) if master else np64(w)
        unit = 0.0 if master else 1.01 * HALF_UNIT[p] * np.abs(want) + 2.0 ** -25 * (p == torch.float16)
        assert np.all(np.abs(got - want) <= tol_w + unit), "w"
        if master:
            assert torch.equal(w, ms.to(p))
    for flat in (fw, fm, fs, fg):
        if flat is not None:
            flat[offset:offset + o * i] = 7.0
            assert bool((flat == 7.0).all())


@pytest.mark.parametrize("products", [3, 1])
def test_zeros_and_spoiled_matrices(products):
    grads = [gradient(80, 120, s) for s in range(4)]
    grads[1].zero_()
    grads[2][3, 5] = float("nan")
    grads[3][0, 0] = float("inf")
    x = orthogonalised(grads, FIVE, products)
    check_x(np64(x[0]), np64(grads[0]), FIVE, products)
    assert not bool(x[1].any())
    assert bool(x[2].isnan().all()) and bool(x[3].isnan().any())


def test_rank_deficient_and_orthogonal():
    """Singular values of 0 stay, those of an orthogonal matrix move together."""
    g = torch.Generator().manual_seed(5)
    low = (torch.randn((200, 3), generator=g) @ torch.randn((3, 150), generator=g)).to(DEV)
    q = torch.linalg.qr(torch.randn((256, 256), generator=g)).Q.contiguous().to(DEV)
    for a in (low, q, torch.eye(130, device=DEV)):
        x, = orthogonalised([a], FIVE, 3)
        check_x(np64(x), np64(a), FIVE, 3)


def test_same_bits_graph_and_streams():
    """A step in a CUDA graph and steps on two streams at once give what single calls give."""
    shapes = [(200, 328), (328, 200), (264, 264)]

    def build():
        out = []
        for n, (o, i) in enumerate(shapes):
            w = gradient(o, i, 50 + n).bfloat16()
            out.append(bg.MuonTensor(w, gradient(o, i, n).bfloat16(), torch.zeros((o, i), device=DEV),
                                     w.float(), 3.0, 0.1))
        arr = bg.bergson_muon_tensors(out)
        return out, arr, bg.workspace_tensor(bg.bergson_muon_step_workspace(arr, 3), DEV)

    def run(arr, ws):
        bg.bergson_muon_step(arr, 0.02, 0.9, True, FIVE, 3, ws)
    ref, arr, ws = build()
    run(arr, ws)
    torch.cuda.synchronize()
    first = [t.master.clone() for t in ref]
    run(arr, ws)
    torch.cuda.synchronize()
    captured, arr2, ws2 = build()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(arr2, ws2)
    graph.replay()
    torch.cuda.synchronize()
    for a, t in zip(first, captured):
        assert torch.equal(a, t.master)
    graph.replay()
    two = [build() for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in two]
    for _ in range(2):
        for s, (_, b, w) in zip(streams, two):
            with torch.cuda.stream(s):
                run(b, w)
    torch.cuda.synchronize()
    ok()
    for others in [captured] + [t for t, _, _ in two]:
        for a, b in zip(ref, others):
            assert torch.equal(a.master, b.master) and torch.equal(a.m, b.m) and torch.equal(a.param, b.param)


def test_refused_tensors():
    w = torch.zeros((8, 16), device=DEV)
    with pytest.raises(ValueError):
        bg.bergson_muon_tensors([bg.MuonTensor(w, w.t().contiguous(), w)])
    with pytest.raises(ValueError):
        bg.bergson_muon_tensors([bg.MuonTensor(w, w, w.bfloat16())])
    with pytest.raises(ValueError):
        bg.bergson_muon_tensors([bg.MuonTensor(w.t(), w.t(), w.t())])
    with pytest.raises(ValueError):
        bg.bergson_muon_tensors([bg.MuonTensor(w, w.cpu(), w)])
    with pytest.raises(TypeError):
        bg.bergson_muon_tensors([bg.MuonTensor(w.long(), w, w)])
    arr = bg.bergson_muon_tensors([bg.MuonTensor(w, w.clone(), w.clone())])
    with pytest.raises(bg.BergsonError) as e:
        bg.bergson_muon_step(arr, 1.0, 0.9, True, FIVE, 3, bg.workspace_tensor(256, DEV))
    assert e.value.status == bg.BERGSON_EWORKSPACE
    with pytest.raises(ValueError):
        bg.bergson_muon_step(arr, 1.0, 0.9, True, [(1.0, 2.0)], 3, bg.workspace_tensor(1 << 20, DEV))
