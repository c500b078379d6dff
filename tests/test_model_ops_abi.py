"""Host-side checks of the entry points around a model's linear layers that need no GPU:
refusals of arguments, workspace sizes, records."""
import ctypes
import struct

import pytest

import paper_2606_11660_gb300 as bg

FAKE = 0x7F0000000000  # aligned, never dereferenced: validation fails first or no device
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def built_library():
    from paper_2606_11660_gb300 import _build
    _build.build()
    yield


def accepted(st):
    """Past validation: without a device the pointers' lookup fails."""
    return st == bg.BERGSON_ECUDA


@pytest.fixture(autouse=True)
def no_launch():
    """What passes validation returns an injected status and enqueues nothing."""
    bg.bergson_debug_inject_status(bg.BERGSON_ECUDA, 1 << 20)
    yield
    bg.bergson_debug_inject_status(0, 0)


def pack(layout, **values):
    """A C record of 8-byte pointers and integers, doubles, and 32-bit integers, in that order."""
    return struct.pack(layout, *[0 if v is None else v for v in values.values()])


def norm(**kw):
    a = dict(x=FAKE, w=FAKE, b=FAKE, y=FAKE + 4096, mean=FAKE, rstd=FAKE, rows=4, d=100, ld_x=100,
             ld_y=100, eps=1e-5, dtype=bg.BERGSON_BF16, wt=0, kind=0, reserved=0)
    a.update(kw)
    return bg.lib().bergson_norm(pack("=6Q4qd4i", **a), None)


def dnorm(ws=FAKE, ws_bytes=1 << 24, **kw):
    a = dict(x=FAKE, w=FAKE, mean=FAKE, rstd=FAKE, dy=FAKE + 4096, dx=FAKE + 8192, dw=FAKE, db=FAKE, rows=4,
             d=100, ld_x=100, ld_dy=100, ld_dx=100, dtype=bg.BERGSON_BF16, wt=0, kind=0, reserved=0)
    a.update(kw)
    return bg.lib().bergson_norm_backward(pack("=8Q5q4i", **a), ws, ws_bytes, None)


NORM_BAD = [
    (dict(dtype=3), bg.BERGSON_EINVAL), (dict(wt=-1), bg.BERGSON_EINVAL),
    (dict(rows=-1), bg.BERGSON_EINVAL), (dict(rows=1 << 31), bg.BERGSON_EINVAL),
    (dict(d=0), bg.BERGSON_EINVAL), (dict(d=(1 << 24) + 1, ld_x=1 << 25), bg.BERGSON_EUNSUPPORTED),
    (dict(ld_x=99), bg.BERGSON_EINVAL), (dict(ld_x=1 << 41), bg.BERGSON_EUNSUPPORTED),
    (dict(x=None), bg.BERGSON_EINVAL), (dict(x=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(dtype=0, x=FAKE + 2), bg.BERGSON_EALIGN), (dict(w=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(kind=2), bg.BERGSON_EINVAL), (dict(mean=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(rstd=FAKE + 1), bg.BERGSON_EALIGN), (dict(reserved=1), bg.BERGSON_EINVAL),
]


@pytest.mark.parametrize("kw,code", NORM_BAD + [
    (dict(eps=-1e-9), bg.BERGSON_EINVAL), (dict(eps=NAN), bg.BERGSON_EINVAL),
    (dict(eps=INF), bg.BERGSON_EINVAL), (dict(eps=1e60), bg.BERGSON_EINVAL),
    (dict(y=None), bg.BERGSON_EINVAL), (dict(y=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(ld_y=99), bg.BERGSON_EINVAL), (dict(y=FAKE, ld_y=104), bg.BERGSON_EINVAL),
    (dict(b=FAKE + 2), bg.BERGSON_EALIGN)])
def test_norm_refusals(kw, code):
    assert norm(**kw) == code and bg.bergson_last_error() != ""


@pytest.mark.parametrize("kw,code", NORM_BAD + [
    (dict(mean=None), bg.BERGSON_EINVAL), (dict(rstd=None), bg.BERGSON_EINVAL),
    (dict(dy=None), bg.BERGSON_EINVAL), (dict(ld_dy=99), bg.BERGSON_EINVAL),
    (dict(dx=None), bg.BERGSON_EINVAL), (dict(ld_dx=-1), bg.BERGSON_EINVAL),
    (dict(dx=FAKE, ld_dx=104), bg.BERGSON_EINVAL), (dict(dx=FAKE + 4096, ld_dx=104), bg.BERGSON_EINVAL),
    (dict(dw=FAKE + 2), bg.BERGSON_EALIGN), (dict(db=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(ws=None), bg.BERGSON_EINVAL), (dict(ws=FAKE + 16), bg.BERGSON_EALIGN),
    (dict(ws_bytes=64), bg.BERGSON_EWORKSPACE)])
def test_norm_backward_refusals(kw, code):
    assert dnorm(**kw) == code and bg.bergson_last_error() != ""


def test_norm_calls_that_pass():
    need = bg.bergson_norm_backward_workspace(4, 100)
    assert need > 0 and need % 256 == 0
    for st in (norm(), norm(w=None, b=None), norm(mean=None, rstd=None), norm(y=FAKE), norm(eps=0.0),
               norm(x=FAKE + 2, ld_x=101), norm(rows=0, x=None, y=None), norm(kind=1, mean=None),
               dnorm(), dnorm(ws_bytes=need), dnorm(dw=None, db=None), dnorm(kind=1, mean=None),
               dnorm(dx=FAKE), dnorm(dx=FAKE + 4096), dnorm(w=None),
               dnorm(rows=0, x=None, dy=None, dx=None, mean=None, rstd=None)):
        assert accepted(st), bg.bergson_last_error()
    assert bg.lib().bergson_norm(None, None) == bg.BERGSON_EINVAL
    assert bg.lib().bergson_norm_backward(None, FAKE, 1 << 20, None) == bg.BERGSON_EINVAL
    assert bg.lib().bergson_norm_backward_workspace(4, 4, None) == bg.BERGSON_EINVAL
    for rows, d in ((-1, 4), (4, 0), (1 << 31, 4)):
        with pytest.raises(bg.BergsonError):
            bg.bergson_norm_backward_workspace(rows, d)
    # a row of dw and db a CTA at most
    assert all(bg.bergson_norm_backward_workspace(1 << 30, d) <= 152 * 8 * 2 * 4 * max(d, 512)
               for d in (1, 24, 512, 513, 2048, 8192, 16_384, 16_385, 1 << 20))


def embed(**kw):
    a = dict(table=FAKE, ids=FAKE, out=FAKE + 65_536, V=50, d=100, rows=4, ld_t=100, ld_o=100, scale=1.0,
             dtype=bg.BERGSON_BF16, reserved=0)
    a.update(kw)
    return bg.lib().bergson_embedding(pack("=3Q5qd2i", **a), None)


def dembed(ws=FAKE, ws_bytes=1 << 30, **kw):
    a = dict(dy=FAKE, ids=FAKE, dt=FAKE + 65_536, V=50, d=100, rows=4, ld_dy=100, ld_t=100, scale=1.0,
             dtype=bg.BERGSON_BF16, tt=0, add=0, reserved=0)
    a.update(kw)
    return bg.lib().bergson_embedding_backward(pack("=3Q5qd4i", **a), ws, ws_bytes, None)


EMBED_BAD = [
    (dict(dtype=7), bg.BERGSON_EINVAL), (dict(rows=-1), bg.BERGSON_EINVAL),
    (dict(rows=1 << 31), bg.BERGSON_EINVAL), (dict(V=0), bg.BERGSON_EINVAL),
    (dict(V=1 << 31), bg.BERGSON_EINVAL), (dict(d=0), bg.BERGSON_EINVAL),
    (dict(d=1 << 25), bg.BERGSON_EUNSUPPORTED), (dict(d=(1 << 20) + 1), bg.BERGSON_EUNSUPPORTED),
    (dict(rows=1 << 30, d=1024), bg.BERGSON_EUNSUPPORTED),
    (dict(scale=INF), bg.BERGSON_EINVAL), (dict(scale=NAN), bg.BERGSON_EINVAL),
    (dict(scale=1e39), bg.BERGSON_EINVAL), (dict(ids=None), bg.BERGSON_EINVAL),
    (dict(ids=FAKE + 4), bg.BERGSON_EALIGN), (dict(ld_t=99), bg.BERGSON_EINVAL),
    (dict(reserved=1), bg.BERGSON_EINVAL),
]


@pytest.mark.parametrize("kw,code", EMBED_BAD + [
    (dict(table=None), bg.BERGSON_EINVAL), (dict(table=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(out=None), bg.BERGSON_EINVAL), (dict(out=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(ld_o=99), bg.BERGSON_EINVAL)])
def test_embedding_refusals(kw, code):
    assert embed(**kw) == code and bg.bergson_last_error() != ""


@pytest.mark.parametrize("kw,code", EMBED_BAD + [
    (dict(tt=3), bg.BERGSON_EINVAL), (dict(dy=None), bg.BERGSON_EINVAL),
    (dict(dy=FAKE + 1), bg.BERGSON_EALIGN), (dict(ld_dy=99), bg.BERGSON_EINVAL),
    (dict(dt=None), bg.BERGSON_EINVAL), (dict(dt=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(ws=None), bg.BERGSON_EINVAL), (dict(ws=FAKE + 128), bg.BERGSON_EALIGN),
    (dict(ws_bytes=1), bg.BERGSON_EWORKSPACE)])
def test_embedding_backward_refusals(kw, code):
    assert dembed(**kw) == code and bg.bergson_last_error() != ""


def test_embedding_calls_that_pass():
    for st in (embed(), embed(table=FAKE + 2, ld_t=101), embed(rows=0, table=None, ids=None, out=None),
               embed(scale=-2.0), dembed(), dembed(add=1, tt=1), dembed(rows=0, dy=None, ids=None),
               dembed(rows=5000, ws_bytes=bg.bergson_embedding_backward_workspace(5000, 50, 100))):
        assert accepted(st), bg.bergson_last_error()
    assert dembed(rows=5000, ws_bytes=4096) == bg.BERGSON_EWORKSPACE
    assert bg.lib().bergson_embedding(None, None) == bg.BERGSON_EINVAL
    assert bg.lib().bergson_embedding_backward(None, FAKE, 1 << 20, None) == bg.BERGSON_EINVAL
    assert bg.lib().bergson_embedding_backward_workspace(4, 4, 4, None) == bg.BERGSON_EINVAL
    for sizes in ((0, 1, 1), (4096, 50_000, 64), (4097, 50_000, 64), (1 << 20, 1 << 18, 100)):
        need = bg.bergson_embedding_backward_workspace(*sizes)
        assert need > 0 and need % 256 == 0


QUINTIC = (3.4445, -4.7750, 2.0315)


def muon(ws=FAKE, ws_bytes=1 << 40, n=1, lr=1e-3, beta=0.9, k=(QUINTIC,) * 5, products=3, gs=None,
         **kw):
    a = dict(param=FAKE, grad=FAKE, master=FAKE, m=FAKE, rows=64, cols=100, lr_scale=1.0, ortho_scale=1.0,
             weight_decay=0.1, param_dtype=1, grad_dtype=1, reserved=0)
    a.update(kw)
    rec = (bg.bergson_muon_tensor * max(n, 1))(*[bg.bergson_muon_tensor(**a)] * max(n, 1))
    flat = [x for abc in k for x in abc] if k is not None else []
    c = (ctypes.c_double * len(flat))(*flat) if k is not None else None
    return bg.lib().bergson_muon_step(rec if n is not None else None, n, lr, beta, 1, c,
                                      len(flat) // 3 if k is not None else 1, products, gs, ws, ws_bytes,
                                      None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), bg.BERGSON_EINVAL), (dict(lr=INF), bg.BERGSON_EINVAL), (dict(beta=1.0), bg.BERGSON_EINVAL),
    (dict(beta=-0.1), bg.BERGSON_EINVAL), (dict(beta=NAN), bg.BERGSON_EINVAL),
    (dict(products=2), bg.BERGSON_EINVAL), (dict(k=()), bg.BERGSON_EINVAL), (dict(k=None), bg.BERGSON_EINVAL),
    (dict(k=(QUINTIC,) * 65), bg.BERGSON_EINVAL), (dict(k=((NAN, 0, 0),)), bg.BERGSON_EINVAL),
    (dict(k=((60.0, 0.0, 0.0),)), bg.BERGSON_EUNSUPPORTED),
    (dict(k=((3.0, 0.0, 0.0),) * 4), bg.BERGSON_EUNSUPPORTED),
    (dict(k=((0.0, 400.0, -399.0),)), bg.BERGSON_EUNSUPPORTED), (dict(gs=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(ws=None), bg.BERGSON_EINVAL), (dict(ws=FAKE + 64), bg.BERGSON_EALIGN),
    (dict(ws_bytes=4096), bg.BERGSON_EWORKSPACE), (dict(param=None), bg.BERGSON_EINVAL),
    (dict(grad=None), bg.BERGSON_EINVAL), (dict(m=None), bg.BERGSON_EINVAL),
    (dict(param=FAKE + 1), bg.BERGSON_EALIGN), (dict(grad=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(m=FAKE + 2), bg.BERGSON_EALIGN), (dict(master=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(rows=0), bg.BERGSON_EINVAL), (dict(cols=-1), bg.BERGSON_EINVAL),
    (dict(cols=(1 << 20) + 1), bg.BERGSON_EUNSUPPORTED),
    (dict(rows=(1 << 16) + 1, cols=(1 << 16) + 1), bg.BERGSON_EUNSUPPORTED),
    (dict(param_dtype=3), bg.BERGSON_EINVAL), (dict(grad_dtype=-1), bg.BERGSON_EINVAL),
    (dict(reserved=1), bg.BERGSON_EINVAL), (dict(lr_scale=INF), bg.BERGSON_EINVAL),
    (dict(ortho_scale=NAN), bg.BERGSON_EINVAL), (dict(weight_decay=INF), bg.BERGSON_EINVAL),
])
def test_muon_refusals(kw, code):
    assert muon(**kw) == code and bg.bergson_last_error() != ""


def test_muon_calls_that_pass():
    for st in (muon(), muon(master=None), muon(n=0), muon(products=1), muon(k=(QUINTIC,) * 64),
               muon(k=((1.5, -0.5, 0.0),) * 20), muon(k=((1.0, 0.0, 0.0),)), muon(gs=FAKE),
               muon(rows=1, cols=1), muon(param_dtype=0, grad_dtype=2), muon(n=700),
               muon(k=((40.0, 0.0, 0.0),))):
        assert accepted(st), bg.bergson_last_error()


def test_muon_workspace():
    def need(shapes, products):
        recs = [bg.bergson_muon_tensor(rows=r, cols=c, param_dtype=1, grad_dtype=1) for r, c in shapes]
        return bg.bergson_muon_step_workspace((bg.bergson_muon_tensor * len(recs))(*recs), products)
    one = need([(64, 100)], 3)
    assert one % 256 == 0 and one > need([(64, 100)], 1) > 0
    assert need([], 3) > 0
    # two planes of X twice, of A and of B: 16 bytes an element of a square matrix, and no more
    # than a batch's however many matrices there are
    assert need([(1024, 1024)] * 4, 3) <= 16 * 4 * 1024 ** 2 + 65_536
    many = need([(4096, 4096)] * 300, 3)
    assert many <= 16 * 2 ** 29 + 65_536
    assert need([(1 + i, 300 - i) for i in range(200)], 3) >= one
    assert bg.lib().bergson_muon_step_workspace(None, 0, 3, None) == bg.BERGSON_EINVAL
    with pytest.raises(bg.BergsonError):
        need([(64, 0)], 3)
