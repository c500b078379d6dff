"""A training step of a small model through the library's operators, against torch's autograd in
64 bits, in a CUDA graph, and on two streams at once.

The model: embedding lookups (scaled), a layer norm, a linear layer with a residual, a norm
without a mean, and an output layer tied to the embedding.  The products of its linear layers
are torch's.  fp32 throughout, so that what is allowed is roundings of sums: gradients are off by at
most some 1e-6 of the sums of magnitudes behind them, a few hundred terms deep through four
layers; 2e-5 of a gradient's largest entry holds that many times over.
"""
import pytest
import torch

import paper_2606_11660_gb300 as bg

pytestmark = pytest.mark.gpu
DEV = "cuda"
LAYER, RMS = bg.BERGSON_NORM_LAYER, bg.BERGSON_NORM_RMS
EPS = 1e-5
QUINTIC = [(3.4445, -4.7750, 2.0315)] * 5


class Model:
    def __init__(self, R, V, d, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def randn(*s, scale=1.0):
            return scale * torch.randn(s, generator=g, device=DEV)
        self.R, self.V, self.d, self.scale = R, V, d, d ** 0.5
        self.ids = torch.randint(-1, V, (R,), generator=g, device=DEV)
        self.targets = torch.randint(-1, V, (R,), generator=g, device=DEV)
        self.E, self.W = randn(V, d, scale=0.05), randn(d, d, scale=d ** -0.5)
        self.w1, self.b1, self.w2 = 1 + randn(d, scale=0.1), randn(d, scale=0.1), 1 + randn(d, scale=0.1)
        new = lambda *s: torch.zeros(s, device=DEV)  # noqa: E731
        self.x0, self.n1, self.x1, self.n2 = (new(R, d) for _ in range(4))
        self.mean, self.r1, self.r2 = new(R), new(R), new(R)
        self.logits = new(R, V)
        self.logp, self.lse = new(R), new(R)
        self.d_logp = torch.full((R,), -1.0 / R, device=DEV)      # of the mean loss
        self.dx, self.dn = new(R, d), new(R, d)
        self.dE, self.dW = new(V, d), new(d, d)
        self.dw1, self.db1, self.dw2 = new(d), new(d), new(d)
        self.nws = bg.workspace_tensor(bg.bergson_norm_backward_workspace(R, d), DEV)
        self.ews = bg.workspace_tensor(bg.bergson_embedding_backward_workspace(R, V, d), DEV)
        self.mW, self.mE, self.vE = new(d, d), new(V * d), new(V * d)
        self.muon = bg.bergson_muon_tensors([bg.MuonTensor(self.W, self.dW, self.mW, None, 0.2 * d ** 0.5, 0.1)])
        self.mws = bg.workspace_tensor(bg.bergson_muon_step_workspace(self.muon, 3), DEV)
        self.adamw = bg.bergson_adamw_tensors([
            bg.AdamWTensor(self.E.view(-1), self.dE.view(-1), self.mE, self.vE)])

    def gradients(self):
        bg.bergson_embedding(self.E, self.ids, self.scale, self.x0)
        bg.bergson_norm(self.x0, self.w1, self.b1, LAYER, EPS, self.n1, self.mean, self.r1)
        torch.addmm(self.x0, self.n1, self.W.t(), out=self.x1)
        bg.bergson_norm(self.x1, self.w2, None, RMS, EPS, self.n2, None, self.r2)
        torch.mm(self.n2, self.E.t(), out=self.logits)
        bg.bergson_token_logprobs(self.logits, self.targets, 1.0, self.logp, self.lse)
        bg.bergson_token_logprobs_backward(self.logits, self.targets, 1.0, self.lse, None, self.d_logp, None,
                                           self.logits)
        G = self.logits                                            # gradients now
        torch.mm(G.t(), self.n2, out=self.dE)
        torch.mm(G, self.E, out=self.dn)
        bg.bergson_norm_backward(self.x1, self.w2, RMS, None, self.r2, self.dn, self.dx, self.dw2, None,
                                 self.nws)
        torch.mm(self.dx.t(), self.n1, out=self.dW)
        torch.mm(self.dx, self.W, out=self.dn)
        bg.bergson_norm_backward(self.x0, self.w1, LAYER, self.mean, self.r1, self.dn, self.dn, self.dw1,
                                 self.db1, self.nws)
        self.dx.add_(self.dn)
        bg.bergson_embedding_backward(self.dx, self.ids, self.scale, self.dE, True, self.ews)

    def step(self):
        self.gradients()
        bg.bergson_muon_step(self.muon, 0.02, 0.95, True, QUINTIC, 3, self.mws)
        bg.bergson_adamw_step(self.adamw, 1e-3, 0.9, 0.99, 1e-8, 1)

    def results(self):
        return {k: v for k, v in vars(self).items()
                if isinstance(v, torch.Tensor) and k not in ("nws", "ews", "mws")}

    def reference(self):
        """Gradients of the loss by autograd in 64 bits."""
        E, W, w1, b1, w2 = (t.double().requires_grad_() for t in (self.E, self.W, self.w1, self.b1, self.w2))
        on = (self.ids >= 0)[:, None]
        x0 = torch.where(on, E[self.ids.clamp(min=0)] * self.scale, 0.0)
        c = x0 - x0.mean(1, keepdim=True)
        n1 = c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * w1 + b1
        x1 = x0 + n1 @ W.t()
        n2 = x1 / torch.sqrt((x1 * x1).mean(1, keepdim=True) + EPS) * w2
        logp = torch.log_softmax(n2 @ E.t(), 1)
        take = logp.gather(1, self.targets.clamp(min=0)[:, None])[:, 0]
        (-(take * (self.targets >= 0)).sum() / self.R).backward()
        return dict(dE=E.grad, dW=W.grad, dw1=w1.grad, db1=b1.grad, dw2=w2.grad)


@pytest.mark.parametrize("R,V,d", [(37, 61, 48), (300, 500, 264), (4500, 1000, 520)])
def test_gradients_of_a_model(R, V, d):
    m = Model(R, V, d)
    m.gradients()
    assert bg.bergson_sync_status() == bg.BERGSON_OK, bg.bergson_last_error()
    for k, want in m.reference().items():
        off = (getattr(m, k).double() - want).abs().max()
        assert float(off) <= 2e-5 * float(want.abs().max()), (k, float(off), float(want.abs().max()))


def test_steps_run():
    m = Model(400, 200, 128)
    losses = []
    for _ in range(6):
        m.step()
        losses.append(-float(m.logp.sum()) / m.R)
    assert bg.bergson_sync_status() == bg.BERGSON_OK and all(x == x for x in losses)


@pytest.mark.parametrize("R,V,d", [(37, 61, 48), (4500, 1000, 264)])
def test_graph_of_a_step(R, V, d):
    one, two = Model(R, V, d), Model(R, V, d)
    one.step()
    two.step()
    torch.cuda.synchronize()
    one, two = Model(R, V, d), Model(R, V, d)
    one.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.step()
    graph.replay()
    torch.cuda.synchronize()
    assert bg.bergson_sync_status() == bg.BERGSON_OK
    for k, v in one.results().items():
        assert torch.equal(v, two.results()[k]), k
    one.step()
    graph.replay()
    torch.cuda.synchronize()
    for k, v in one.results().items():
        assert torch.equal(v, two.results()[k]), k


def test_steps_on_two_streams_at_once():
    alone = [Model(600, 300, 136, seed=k) for k in range(2)]
    again = [Model(600, 300, 136, seed=k) for k in range(2)]
    for m in alone:
        m.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for stream, m in zip(streams, again):
        with torch.cuda.stream(stream):
            m.step()
    torch.cuda.synchronize()
    for a, b in zip(alone, again):
        for k, v in a.results().items():
            assert torch.equal(v, b.results()[k]), k
