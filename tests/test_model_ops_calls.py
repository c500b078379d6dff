"""Calls of the operators around a model's linear layers that need no GPU: what the documentation allows
passes, what it does not is refused by name."""
import pytest
import torch

import paper_2606_11660_gb300 as bg
from tests.test_model_ops_abi import QUINTIC, accepted, built_library, muon, no_launch  # noqa: F401


@pytest.mark.parametrize("k", [
    ((10.0, 0.0, 0.0), (0.1, 0.0, 0.0)), ((9.0, -2.0, 0.0), (0.25, 0.0, 0.0)), ((40.0, 0.0, 0.0), (1.0, 0.0, 0.0))])
def test_coefficients_without_a_square(k):
    """c = 0: |X| up to 48 as the header has it, whatever A = X X^T is."""
    assert accepted(muon(k=k)), bg.bergson_last_error()


@pytest.mark.parametrize("k", [
    ((10.0, 0.0, 0.0), (10.0, 0.0, 0.0)), ((10.0, 0.0, 0.0), (0.1, 0.5, 0.0)),
    ((10.0, 0.0, 0.0), (0.0, 0.0, 0.001)), ((0.0, -60.0, 0.0),)])
def test_coefficients_that_pass_the_limits(k):
    """|X| = 100; b A = 50; A = 100 beside a square; b = 60."""
    assert muon(k=k) == bg.BERGSON_EUNSUPPORTED and bg.bergson_last_error() != ""


def test_workspace_of_thin_matrices():
    """Rows stand apart by whole chunks of 64 columns: a batch ends by what its planes take."""
    def need(shapes, products):
        recs = [bg.bergson_muon_tensor(rows=r, cols=c, param_dtype=1, grad_dtype=1) for r, c in shapes]
        return bg.bergson_muon_step_workspace((bg.bergson_muon_tensor * len(recs))(*recs), products)
    for shape in ((1 << 20, 1), (1 << 18, 3), (1 << 20, 65), (1, 1 << 20)):
        for products, each in ((3, 16), (1, 8)):
            assert need([shape] * 300, products) <= each * 2 ** 29 + 65_536
    # one alone may take more
    assert need([(1 << 20, 600)], 1) >= 2 * 2 * 640 * 2 ** 20


def test_products_that_pass_a_count():
    """Refused before anything is enqueued: m keeps its value."""
    big = dict(rows=1 << 16, cols=1 << 20, ws_bytes=1 << 62)
    assert muon(k=(QUINTIC,) * 64, **big) == bg.BERGSON_EUNSUPPORTED and "iterations" in bg.bergson_last_error()
    for st in (muon(k=(QUINTIC,) * 60, **big), muon(k=(QUINTIC,) * 64, products=1, **big),
               muon(k=(QUINTIC,) * 64, rows=1 << 16, cols=1 << 16, ws_bytes=1 << 62),
               muon(k=(QUINTIC,) * 64, n=300, rows=1, cols=1 << 20)):
        assert accepted(st), bg.bergson_last_error()


@pytest.mark.parametrize("what,call", [
    ("x", lambda t: bg.bergson_norm(t, None, None, bg.BERGSON_NORM_LAYER, 1e-5, t)),
    ("x", lambda t: bg.bergson_norm_backward(t, None, bg.BERGSON_NORM_RMS, None, None, t, t, None, None, t)),
    ("table", lambda t: bg.bergson_embedding(t, torch.zeros(2, dtype=torch.int64), 1.0, t)),
    ("dy", lambda t: bg.bergson_embedding_backward(t, torch.zeros(6, dtype=torch.int64), 1.0, t[0], False, t)),
    ("param", lambda t: bg.bergson_muon_tensors([bg.MuonTensor(t, t, t)])),
])
@pytest.mark.parametrize("shape", [(2, 3, 8), (8,)])
def test_tensors_that_are_no_matrices(what, call, shape):
    with pytest.raises(ValueError, match=rf"^{what} must be a matrix .*{shape[0]}"):
        call(torch.zeros(shape))


@pytest.mark.parametrize("k", [[(1.0, 2.0)], [(1.0, 2.0), (3.0, 4.0, 5.0, 6.0)], [(1.0, 2.0, 3.0, 4.0)]])
def test_coefficients_that_are_no_triples(k):
    with pytest.raises(ValueError, match="triples"):
        bg.bergson_muon_step([], 1.0, 0.9, True, k, 3, torch.zeros(256))
