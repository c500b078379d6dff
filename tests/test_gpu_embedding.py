"""GPU parity of embedding lookups and the table's gradient with the fp64 oracle.

A lookup is one product and one rounding: half a unit of the output's type, and 2^-24
of the product's.  A sum over the n rows of a token is off by at most n 2^-24 of the
sum of magnitudes (each addition rounds once), with the scale and the addition to the
table two more; then half a unit of the table's type.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_gb300 as bg
from oracle import model_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 1e-42, torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}


def np64(x):
    return x.detach().cpu().double().numpy()


def matrix(R, d, dtype, pad=0, offset=0, fill=7.0):
    flat = torch.full((offset + R * (d + pad) + 16,), fill, dtype=dtype, device=DEV)
    return flat, flat[offset:offset + R * (d + pad)].view(R, d + pad)[:, :d]


def ok():
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()


def near(got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


def tokens(R, V, seed=0, skewed=True, ignored=0.2):
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(R, generator=g, dtype=torch.float64)
    t = (torch.exp(u * np.log(V + 1)) - 1) if skewed else u * V
    t = t.long().clamp(0, V - 1)
    t[torch.rand(R, generator=g) < ignored] = -1
    return t.to(DEV)


def check_lookup(R, V, d, dtype, scale=1.0, pad=0, offset=0):
    g = torch.Generator().manual_seed(R + V + d)
    _, table = matrix(V, d, dtype, pad, offset)
    table.copy_(torch.randn((V, d), generator=g))
    flat, out = matrix(R, d, dtype, pad, offset)
    ids = tokens(R, V)
    bg.bergson_embedding(table, ids, scale, out)
    ok()
    want = orc.embedding(np64(table), ids.tolist(), float(np.float32(scale)))
    near(np64(out), want, (HALF_UNIT[dtype] + U) * 1.01 * np.abs(want) + SMALLEST[dtype])
    if scale == 1.0:
        assert np.array_equal(np64(out), want)
    out.fill_(7.0)
    assert bool((flat == 7.0).all())


def check_gradient(ids, V, d, dtype, tt, add, scale=1.0, pad=0, offset=0, poison=False):
    R = len(ids)
    g = torch.Generator().manual_seed(R + V + d)
    _, dy = matrix(R, d, dtype, pad, offset)
    dy.copy_(torch.randn((R, d), generator=g))
    if poison:                                    # what is left out may hold anything
        dy[ids < 0] = float("nan")
    flat, dt = matrix(V, d, tt, pad, offset)
    if add:
        dt.copy_(torch.randn((V, d), generator=g))
    before = dt.clone()
    ws = bg.workspace_tensor(bg.bergson_embedding_backward_workspace(R, V, d), DEV)
    ws.fill_(255)
    bg.bergson_embedding_backward(dy, ids, scale, dt, add, ws)
    ok()
    ids_list = ids.tolist()
    want, size = orc.embedding_backward(np64(dy), ids_list, float(np.float32(scale)), V)
    n = np.bincount(ids[ids >= 0].cpu().numpy(), minlength=V)[:, None]
    tol = (n + 2) * U * size
    if add:
        untouched = torch.from_numpy(n[:, 0] == 0).to(DEV)
        assert torch.equal(dt[untouched], before[untouched])
        want = want + np64(before)
        tol = tol + U * np.abs(want)
    near(np64(dt), want, tol + HALF_UNIT[tt] * 1.01 * np.abs(want) + SMALLEST[tt])
    got = dt.clone()
    dt.fill_(7.0)
    assert bool((flat == 7.0).all())
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V,d", [(1, 1, 1), (5, 96, 24), (33, 1000, 768), (7, 50, 1025), (3, 20, 5000),
                                   (1000, 300, 260)])
@pytest.mark.parametrize("scale,pad,offset", [(1.0, 0, 0), (27.7, 3, 0), (1.0, 8, 8), (1.0, 0, 1)])
def test_lookup(R, V, d, dtype, scale, pad, offset):
    check_lookup(R, V, d, dtype, scale, pad, offset)


@pytest.mark.parametrize("dtype,tt", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                      (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
                                      (torch.float32, torch.bfloat16), (torch.float16, torch.float32)])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("R,V,d", [(1, 1, 1), (1, 700, 40), (97, 600, 24), (776, 1500, 768), (300, 96, 1100),
                                   (4096, 500, 65), (4097, 500, 65), (5000, 3000, 96), (4100, 96, 1032)])
def test_gradient(R, V, d, dtype, tt, add):
    check_gradient(tokens(R, V, seed=R), V, d, dtype, tt, add, scale=1.0 if d % 2 else 3.3, poison=True)


@pytest.mark.parametrize("R", [400, 5000])
@pytest.mark.parametrize("pad,offset", [(3, 0), (8, 8), (0, 1)])
@pytest.mark.parametrize("d", [40, 1027])
@pytest.mark.parametrize("tt", DTYPES)
def test_rows_apart(R, d, pad, offset, tt):
    for add in (False, True):
        check_gradient(tokens(R, 200), 200, d, torch.bfloat16, tt, add, 0.5, pad, offset)


@pytest.mark.parametrize("R", [64, 2048, 4100, 6000, 9000])
@pytest.mark.parametrize("kind", ["one", "two", "apart", "none", "last", "falling"])
def test_orders_of_tokens(R, kind):
    """One token for all, tokens that come once, none at all, runs that end at their limits."""
    V = R + 40
    i = torch.arange(R, device=DEV)
    ids = {"one": torch.full_like(i, 5), "two": (i >= R // 2 + 7).long() * 9,
           "apart": (i * 7919) % R, "none": torch.full_like(i, -3),
           "last": torch.where(i % 32 < 31, i, V - 1), "falling": (R - 1 - i) // 32}[kind]
    for add in (False, True):
        check_gradient(ids, V, 72, torch.bfloat16, torch.float32, add)


@pytest.mark.parametrize("R", [17_000, 40_000, 70_001])
@pytest.mark.parametrize("kind", ["one", "apart", "last", "falling", "skewed"])
def test_orders_of_many_tokens(R, kind):
    """The longer runs, and tokens that cross their ends or fill them."""
    V = 4000
    i = torch.arange(R, device=DEV)
    ids = {"one": torch.full_like(i, 5), "apart": (i * 7919) % V,
           "last": torch.where(i % 64 < 63, i % (V - 1), V - 1), "falling": ((R - 1 - i) // 64) % V,
           "skewed": tokens(R, V, seed=R)}[kind]
    for add in (False, True):
        check_gradient(ids, V, 24, torch.bfloat16, torch.float32, add)


@pytest.mark.parametrize("R,V", [(5000, 511), (5000, 512), (5000, 513), (5000, 262_143), (5000, 262_144),
                                 (300_000, 5000)])
def test_sort_passes(R, V):
    """The digits' borders, and tiles of several steps."""
    check_gradient(tokens(R, V, skewed=False), V, 8, torch.float32, torch.float32, False)


def test_wide_vocabulary():
    """Three passes of the sort; a table of 2^27 rows and one column."""
    V, R = 1 << 27, 5000
    ids = torch.randint(0, V, (R,), device=DEV)
    ids[:3] = torch.tensor([0, V - 1, V - 1], device=DEV)
    dy = torch.randn((R, 1), device=DEV)
    dt = torch.full((V, 1), 7.0, device=DEV)
    ws = bg.workspace_tensor(bg.bergson_embedding_backward_workspace(R, V, 1), DEV)
    bg.bergson_embedding_backward(dy, ids, 1.0, dt, False, ws)
    ok()
    want = torch.zeros((V, 1), dtype=torch.float64, device=DEV).index_add_(0, ids, dy.double())
    assert float((dt - want).abs().max()) <= 8 * 4 * U       # a token comes a few times


def test_ids_out_of_range():
    table = torch.randn((10, 64), device=DEV)
    ids = torch.tensor([3, 10, -1, 9], device=DEV)
    out = torch.zeros((4, 64), device=DEV)
    bg.bergson_embedding(table, ids, 1.0, out)
    assert bg.bergson_sync_status() == bg.BERGSON_EINVAL
    assert bool(out[1].isnan().all()) and not bool(out[2].any()) and torch.equal(out[3], table[9])
    for R in (4, 5000):
        many = ids.repeat(R // 4)
        dy = torch.ones((len(many), 64), device=DEV)
        ws = bg.workspace_tensor(bg.bergson_embedding_backward_workspace(len(many), 10, 64), DEV)
        dt = torch.full((10, 64), 7.0, device=DEV)
        bg.bergson_embedding_backward(dy, many, 1.0, dt, False, ws)
        assert bg.bergson_sync_status() == bg.BERGSON_EINVAL
        want = torch.zeros((10, 64), device=DEV)
        want[3] = want[9] = R // 4
        assert torch.equal(dt, want)


def test_no_rows():
    ids = torch.empty(0, dtype=torch.int64, device=DEV)
    dy = torch.empty((0, 30), device=DEV)
    dt = torch.full((70, 30), 7.0, device=DEV)
    ws = bg.workspace_tensor(bg.bergson_embedding_backward_workspace(0, 70, 30), DEV)
    bg.bergson_embedding(dt, ids, 1.0, dy)
    bg.bergson_embedding_backward(dy, ids, 1.0, dt, True, ws)
    ok()
    assert bool((dt == 7.0).all())
    bg.bergson_embedding_backward(dy, ids, 1.0, dt, False, ws)
    ok()
    assert not bool(dt.any())


def test_same_bits_every_time():
    ids = tokens(20_000, 700)
    first = check_gradient(ids, 700, 40, torch.bfloat16, torch.float32, False)
    for _ in range(3):
        assert torch.equal(first, check_gradient(ids, 700, 40, torch.bfloat16, torch.float32, False))


def test_refused_tensors():
    t = torch.zeros((10, 64), device=DEV)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    ws = bg.workspace_tensor(256, DEV)
    with pytest.raises(ValueError):
        bg.bergson_embedding(t, ids.int(), 1.0, t[:4])
    with pytest.raises(ValueError):
        bg.bergson_embedding(t, ids, 1.0, t[:5])
    with pytest.raises(ValueError):
        bg.bergson_embedding(t, ids, 1.0, t[:4].bfloat16())
    with pytest.raises(ValueError):
        bg.bergson_embedding(t.cpu(), ids, 1.0, t[:4])
    with pytest.raises(ValueError):
        bg.bergson_embedding_backward(t[:4], ids, 1.0, t[:, :32], False, ws)
    with pytest.raises(TypeError):
        bg.bergson_embedding_backward(t[:4], ids, 1.0, t.long(), False, ws)
    with pytest.raises(bg.BergsonError) as e:
        bg.bergson_embedding_backward(torch.zeros((5000, 64), device=DEV), ids.repeat(1250), 1.0, t,
                                      False, ws)
    assert e.value.status == bg.BERGSON_EWORKSPACE
