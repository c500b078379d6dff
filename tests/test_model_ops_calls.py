"""Calls of the operators around a model's linear layers that need no GPU: what the documentation allows
passes, what it does not is refused by name."""
import paper_2606_11660_gb300 as bg
from tests.test_model_ops_abi import built_library  # noqa: F401


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
