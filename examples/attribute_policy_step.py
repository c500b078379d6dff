"""Fine-tunes a small output layer on answers' rewards and on preferred answers, then asks which
of the training answers drove it.

    python examples/attribute_policy_step.py

A "model" of one linear layer maps hidden states A [B, T, d] to logits over V
tokens.  Per step: token log-probabilities and entropies of the sampled
tokens, the clipped policy loss with its KL term (or, afterwards, the preference
loss over pairs of answers), gradients at the logits, the weight's gradient and
one AdamW step with 8-bit moments.  The last step's gradients at the logits
are the G of the layer, AdamW's second moments give its r and c, and the
projected per-answer gradients go to a store that each answer then queries.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_11660_gb300 as bg  # noqa: E402

B, T, D, V = 16, 96, 256, 512
LR, BETA1, BETA2, EPS = 2e-4, 0.9, 0.99, 1e-8


class OutputLayer:
    """W [V, D] with its gradient, AdamW's 8-bit moments and an fp32 master copy."""

    def __init__(self, g):
        self.W = (0.02 * torch.randn((V, D), generator=g, device="cuda")).bfloat16()
        self.dW = torch.empty_like(self.W)
        master = self.W.float()
        n, blocks = V * D, V * D // bg.BERGSON_STATE_BLOCK
        self.m, self.v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.ms, self.vs = (torch.zeros(blocks, device="cuda") for _ in range(2))
        self.tensors = bg.bergson_adamw_tensors([
            bg.AdamWTensor(self.W, self.dW, self.m, self.v, master, self.ms, self.vs,
                           weight_decay=0.01)])
        self.master, self.steps = master, 0

    def logits(self, A):
        return A.view(-1, D) @ self.W.t()

    def step(self, A, G):
        """The weight's gradient from its inputs and output gradients, and one AdamW step."""
        torch.mm(G.t(), A.view(-1, D), out=self.dW)
        self.steps += 1
        bg.bergson_adamw_step(self.tensors, LR, BETA1, BETA2, EPS, self.steps, seed=1)

    def moments(self):
        """r [V] and c [D] of the second moments, bias-corrected."""
        r, c = torch.empty(V, device="cuda"), torch.empty(D, device="cuda")
        mats = bg.bergson_moment_matrices([bg.MomentMatrix(self.v.view(V, D), r, c, self.vs)])
        ws = bg.workspace_tensor(bg.bergson_factor_moments_workspace(mats))
        bg.bergson_factor_moments(mats, 1 / (1 - BETA2 ** self.steps), 1e-12, ws)
        return r, c


def logprobs(x, tokens):
    """(logp, lse, entropy) of the tokens, [B*T] each; tokens < 0 are left out."""
    out = [torch.empty(tokens.numel(), device="cuda") for _ in range(3)]
    bg.bergson_token_logprobs(x, tokens.view(-1), 1.0, *out)
    return out


def policy_step(layer, A, tokens, mask, old, ref, advantages, ws):
    """One clipped policy step; returns (loss, gradients at the logits)."""
    x = layer.logits(A)
    logp, lse, entropy = logprobs(x, tokens)
    loss, stats = torch.empty(1, device="cuda"), torch.empty(3, device="cuda")
    d, dh = torch.empty((B, T), device="cuda"), torch.empty((B, T), device="cuda")
    bg.bergson_policy_loss(logp.view(B, T), old, ref, entropy.view(B, T), advantages, mask, 0.2,
                           0.28, 0.02, 0.001, bg.BERGSON_POLICY_TOKEN_MEAN, 1.0, loss, None, stats,
                           d, dh, ws)
    # in place of the logits
    bg.bergson_token_logprobs_backward(x, tokens.view(-1), 1.0, lse, entropy, d.view(-1),
                                       dh.view(-1), x)
    layer.step(A, x)
    return loss, x


def preference_step(layer, A, tokens, mask, ref):
    """One preference step: answers 0 .. B/2 - 1 are preferred to B/2 .. B - 1."""
    x = layer.logits(A)
    logp, lse, _ = logprobs(x, tokens)
    loss, pair = torch.empty(1, device="cuda"), torch.empty(B // 2, device="cuda")
    d = torch.empty((B, T), device="cuda")
    bg.bergson_preference_loss(logp.view(B, T), ref, mask, bg.BERGSON_PREFERENCE_SIGMOID, 0.1, 0.0,
                               0.0, False, loss, pair, None, d)
    bg.bergson_token_logprobs_backward(x, tokens.view(-1), 1.0, lse, None, d.view(-1), None, x)
    layer.step(A, x)
    return loss, x


def attribute(layer, A, G, mask):
    """Every answer's most similar training answers under the normalised gradients."""
    r, c = layer.moments()
    s_in, s_out = bg.bergson_module_seeds(0, 0)
    layers = [bg.Layer(A, G.view(B, T, V), 16, 16, s_in, s_out, r, c)]
    K = 256
    ws = bg.workspace_tensor(bg.bergson_project_grads_workspace(layers, B, T))
    proj = torch.empty((B, K), device="cuda")
    bg.bergson_project_grads(layers, B, T, mask, proj, ws)
    store = torch.empty((B, K), dtype=torch.float16, device="cuda")
    bg.bergson_build_store(proj, B, K, True, store, 0)
    ws = bg.workspace_tensor(bg.bergson_score_topk_workspace(B, K, B, 3))
    scores = torch.empty((B, 3), device="cuda")
    index = torch.empty((B, 3), dtype=torch.int64, device="cuda")
    bg.bergson_score_topk(store, B, K, proj, 3, scores, index, ws)
    return scores, index


def main(steps: int = 12) -> dict:
    g = torch.Generator(device="cuda").manual_seed(0)
    layer = OutputLayer(g)
    A = torch.randn((B, T, D), generator=g, device="cuda").bfloat16()
    lengths = torch.randint(T // 2, T + 1, (B,), generator=g, device="cuda")
    mask = (torch.arange(T, device="cuda") < lengths[:, None]).to(torch.uint8)
    tokens = torch.randint(0, V, (B, T), generator=g, device="cuda")
    tokens = torch.where(mask != 0, tokens, -1)            # padding: left out
    # of the policy that sampled, which is the reference too
    old = logprobs(layer.logits(A), tokens)[0].view(B, T)
    advantages = torch.linspace(-1, 1, B, device="cuda")
    ws = bg.workspace_tensor(bg.bergson_policy_loss_workspace(B, T))

    out = {"policy": [], "preference": []}
    for _ in range(steps):
        loss, G = policy_step(layer, A, tokens, mask, old, old, advantages, ws)
        out["policy"].append(float(loss))
    ref = logprobs(layer.logits(A), tokens)[0].view(B, T)
    for _ in range(steps):
        loss, G = preference_step(layer, A, tokens, mask, ref)
        out["preference"].append(float(loss))
    out["scores"], out["index"] = (x.cpu() for x in attribute(layer, A, G, mask))
    status = bg.bergson_sync_status()
    if status != bg.BERGSON_OK:
        raise RuntimeError(f"device status {status}: {bg.bergson_last_error()}")
    return out


if __name__ == "__main__":
    result = main()
    print("policy loss     %.4f -> %.4f" % (result["policy"][0], result["policy"][-1]))
    print("preference loss %.4f -> %.4f" % (result["preference"][0], result["preference"][-1]))
    for b in range(4):
        print("answer %d: " % b + ", ".join(
            "%d (%.3f)" % (i, s) for i, s in zip(result["index"][b].tolist(),
                                                 result["scores"][b].tolist())))
