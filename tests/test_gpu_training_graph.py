"""A training step's operators captured in one CUDA graph give what single calls give."""
import pytest
import torch

import paper_2606_11660_gb300 as bg

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Step:
    """Log-probabilities, both losses, gradients, an AdamW step and its factors."""

    def __init__(self, B, T, V, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def new(*shape, dtype=torch.float32):
            return torch.zeros(shape, dtype=dtype, device=DEV)
        self.B, self.T = B, T
        self.x = torch.randn((B * T, V), generator=g, device=DEV).bfloat16()
        self.t = torch.randint(-1, V, (B * T,), generator=g, device=DEV)
        self.old = -5 - torch.rand((B, T), generator=g, device=DEV)
        self.mask = (torch.rand((B, T), generator=g, device=DEV) < 0.7).to(torch.uint8)
        self.adv = torch.randn(B, generator=g, device=DEV)
        self.logp, self.lse, self.ent = new(B * T), new(B * T), new(B * T)
        self.loss, self.seq, self.stats, self.d, self.dh = new(1), new(B), new(3), new(B, T), new(B, T)
        self.loss2, self.pair, self.rewards, self.d2 = new(1), new(B // 2), new(B), new(B, T)
        self.dx = torch.zeros_like(self.x)
        self.ws = bg.workspace_tensor(bg.bergson_policy_loss_workspace(B, T), DEV)
        n = B * T * V
        self.p = torch.randn(n, generator=g, device=DEV).bfloat16()
        self.m, self.v = new(n, dtype=torch.uint8), new(n, dtype=torch.uint8)
        self.ms, self.vs = new(-(-n // 256)), new(-(-n // 256))
        self.tensors = bg.bergson_adamw_tensors([
            bg.AdamWTensor(self.p, self.dx.view(-1), self.m, self.v, None, self.ms, self.vs)])
        self.r, self.c, self.values = new(B * T), new(V), new(n)
        self.mats = bg.bergson_moment_matrices([
            bg.MomentMatrix(self.v.view(B * T, V), self.r, self.c, self.vs)])
        self.mws = bg.workspace_tensor(bg.bergson_factor_moments_workspace(self.mats), DEV)

    def run(self):
        B, T = self.B, self.T
        bg.bergson_token_logprobs(self.x, self.t, 0.9, self.logp, self.lse, self.ent)
        lp = self.logp.view(B, T)
        bg.bergson_policy_loss(lp, self.old, self.old, self.ent.view(B, T), self.adv, self.mask, 0.2,
                               0.2, 0.1, 0.01, bg.BERGSON_POLICY_TOKEN_MEAN, 1.0, self.loss, self.seq,
                               self.stats, self.d, self.dh, self.ws)
        bg.bergson_preference_loss(lp, self.old, self.mask, bg.BERGSON_PREFERENCE_SIGMOID, 0.1, 0.0,
                                   0.1, False, self.loss2, self.pair, self.rewards, self.d2)
        bg.bergson_token_logprobs_backward(self.x, self.t, 0.9, self.lse, self.ent, self.d.view(-1),
                                           self.dh.view(-1), self.dx)
        bg.bergson_adamw_step(self.tensors, 1e-3, 0.9, 0.99, 1e-8, 1, seed=3)
        bg.bergson_adamw_state_values(self.v, self.vs, bg.BERGSON_MOMENT_SECOND, self.values)
        bg.bergson_factor_moments(self.mats, 100.0, 1e-12, self.mws)

    def results(self):
        return {k: v for k, v in vars(self).items()
                if isinstance(v, torch.Tensor) and k not in ("ws", "mws")}


@pytest.mark.parametrize("B,T,V", [(4, 24, 512), (24, 3000, 130), (700, 40, 72), (2, 3, 40_000)])
def test_graph_of_a_step(B, T, V):
    one, two = Step(B, T, V), Step(B, T, V)
    one.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.run()
    graph.replay()
    torch.cuda.synchronize()
    assert bg.bergson_sync_status() == bg.BERGSON_OK
    for k, v in one.results().items():
        assert torch.equal(v, two.results()[k]), k
    assert float(one.loss) != 0 and float(one.d.abs().sum()) > 0


def test_steps_on_two_streams_at_once():
    steps = [Step(16, 200, 300, seed=k) for k in range(2)]
    again = [Step(16, 200, 300, seed=k) for k in range(2)]
    for s in steps:
        s.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for stream, s in zip(streams, again):
        with torch.cuda.stream(stream):
            s.run()
    torch.cuda.synchronize()
    for a, b in zip(steps, again):
        for k, v in a.results().items():
            assert torch.equal(v, b.results()[k]), k
