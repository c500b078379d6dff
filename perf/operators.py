"""Timed cases of the training-side operators: what a program that fine-tunes a
model and attributes the result calls next to the collection.

  logprobs    token log-probabilities (and entropies) of a batch of logits
  dlogits     their backward pass: gradients at the logits, which are also the
              output gradients G of the model's last linear layer
  policy      clipped policy loss with a KL term, forward and backward
  preference  preference loss over pairs of answers, forward and backward
  adamw       one AdamW step over many tensors, states in 32 or 8 bits
  moments     factored second moments r, c of AdamW's v, as a layer takes them

`own` selects the library's kernels; otherwise `run` computes the same in
elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                       # elements that share a scale of an 8-bit state
GAMMA = 0x9E3779B97F4A7C15
MAX_LOGITS_BYTES = 8192 * 131072 * 2
MAX_TOKENS = 2048 * 16384
MAX_PAIR_TOKENS = 2 * 256 * 32768
MAX_PARAMS = 8 * 50_364_416
MAX_MOMENTS_BYTES = 4 * 8 * 50_331_648


def listed():
    return [
        # The last position of a few prompts: one decoding step's log-probabilities and
        # entropies over an odd vocabulary.
        dict(name="logprobs_step", op="logprobs", R=5, V=50_257, dtype="bf16", pad=0, masked=0,
             ignored=0.0, entropy=True, tau=0.7),
        # A full scoring pass over a training batch with a vocabulary padded to a round
        # size, whose padding columns are masked with -inf; a tenth of the tokens are prompt.
        dict(name="logprobs_batch", op="logprobs", R=8192, V=131_072, dtype="bf16", pad=0, masked=60,
             ignored=0.1, entropy=True, tau=1.0),
        # The backward pass of a small unaligned batch in 16-bit floats, as test runs make it.
        dict(name="dlogits_odd", op="dlogits", R=1031, V=32_003, dtype="f16", pad=0, masked=0,
             ignored=0.25, entropy=True, tau=0.9),
        # Gradients at the logits of a training batch, half of whose tokens are prompt.
        dict(name="dlogits_batch", op="dlogits", R=8192, V=65_536, dtype="bf16", pad=0, masked=0,
             ignored=0.5, entropy=False, tau=1.0),
        # A debugging batch: a handful of short answers, one of them empty.
        dict(name="policy_tiny", op="policy", B=8, T=97, pad=3, reduction="seq_mean", kl=0.04,
             ent=0.0, token_adv=False, fill=0.7),
        # The long answers of a policy-optimisation step, KL and entropy terms on.
        dict(name="policy_long", op="policy", B=2048, T=16_384, pad=0, reduction="token_mean",
             kl=0.04, ent=0.001, token_adv=False, fill=0.6),
        # A micro-batch of preference pairs.
        dict(name="preference_micro", op="preference", P=4, T=383, pad=1, kind="sigmoid", ref=True,
             mean=False, smooth=0.0, margin=0.0, fill=0.7),
        # Length-normalised preference over long documents without a reference model.
        dict(name="preference_long", op="preference", P=256, T=32_768, pad=0, kind="sigmoid",
             ref=False, mean=True, smooth=0.1, margin=0.5, fill=0.6),
        # Low-rank adapters of a 24-layer model: hundreds of small tensors, 8-bit states.
        dict(name="adamw_adapters", op="adamw", layout="adapters", d=2048, ff=8192, layers=24,
             rank=16, p="bf16", g="bf16", master=True, bits=8, scaled=True),
        # Full fine-tuning of four wide transformer blocks, 32-bit states and master copies.
        dict(name="adamw_blocks", op="adamw", layout="blocks", d=2048, ff=8192, layers=4, rank=0,
             p="bf16", g="bf16", master=True, bits=32, scaled=True),
        # Second moments of one small layer.
        dict(name="moments_tiny", op="moments", layout="blocks", d=72, ff=280, layers=1, bits=8),
        # Second moments of the modules of four wide blocks, before their collection.
        dict(name="moments_blocks", op="moments", layout="blocks", d=2048, ff=8192, layers=4,
             bits=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "dlogits", "policy", "preference", "adamw", "moments"])
    if op in ("logprobs", "dlogits"):
        while True:
            c = dict(op=op, R=_log(rng, 1, 8192), V=_log(rng, 96, 262_144),
                     dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), pad=rng.choice([0, 0, 5, 64]),
                     masked=0, ignored=rng.choice([0.0, 0.1, 0.5]), entropy=rng.random() < 0.5,
                     tau=rng.choice([1.0, 1.0, 0.6, 1.3]))
            c["masked"] = rng.choice([0, 0, 37])
            if c["R"] * (c["V"] + c["pad"]) * SIZE[c["dtype"]] <= MAX_LOGITS_BYTES // (
                    1 if op == "logprobs" else 2):
                return c
    if op == "policy":
        while True:
            c = dict(op=op, B=_log(rng, 1, 2048), T=_log(rng, 1, 32_768), pad=rng.choice([0, 0, 3, 8]),
                     reduction=rng.choice(["token_mean", "seq_mean", "sum_norm"]),
                     kl=rng.choice([0.0, 0.04]), ent=rng.choice([0.0, 0.001]),
                     token_adv=rng.random() < 0.3, fill=rng.choice([0.3, 0.6, 1.0]))
            if c["B"] * c["T"] <= MAX_TOKENS:
                return c
    if op == "preference":
        while True:
            c = dict(op=op, P=_log(rng, 1, 2048), T=_log(rng, 1, 32_768), pad=rng.choice([0, 0, 1, 8]),
                     kind=rng.choice(["sigmoid", "sigmoid", "hinge", "squared"]),
                     ref=rng.random() < 0.7, mean=False, smooth=rng.choice([0.0, 0.1]),
                     margin=0.0, fill=rng.choice([0.3, 0.6, 1.0]))
            c["mean"] = c["kind"] == "squared" or rng.random() < 0.3
            c["margin"] = 0.5 if c["mean"] and c["kind"] == "sigmoid" else 0.0
            if 2 * c["P"] * c["T"] <= MAX_PAIR_TOKENS:
                return c
    while True:
        layout = rng.choice(["adapters", "blocks"])
        c = dict(op=op, layout=layout, d=_log(rng, 24, 2048), ff=0, layers=_log(rng, 1, 24))
        c["ff"] = c["d"] * rng.choice([2, 4]) + rng.choice([0, 0, 1, 8])
        if op == "adamw":
            p = rng.choice(["bf16", "bf16", "f16", "f32"])
            c.update(rank=rng.choice([4, 8, 16, 31]), p=p, g=rng.choice([p, p, "f32"]),
                     master=p != "f32" and rng.random() < 0.6, bits=rng.choice([8, 32]),
                     scaled=rng.random() < 0.5)
            if c["layout"] == "blocks":
                c["rank"] = 0
            if _params(c) <= MAX_PARAMS // 2:
                return c
        else:
            c.update(layout="blocks", bits=rng.choice([8, 32]))
            if work(c)["bytes"] <= MAX_MOMENTS_BYTES // 2:
                return c


# ------------------------------------------------------------------ shapes

def _matrices(c):
    """(rows, columns) of a block's weight matrices, all layers."""
    d, ff = c["d"], c["ff"]
    return [(3 * d, d), (d, d), (ff, d), (d, ff)] * c["layers"]


def _tensors(c):
    """(elements, weight decay) of every trained tensor."""
    if c["layout"] == "adapters":
        return [(n, 0.0) for o, i in _matrices(c) for n in (c["rank"] * i, o * c["rank"])]
    out = []
    for o, i in _matrices(c):
        out += [(o * i, 0.1), (o, 0.0)]                   # weight and bias
    return out + [(c["d"], 0.0)] * (4 * c["layers"])      # two norms' gains and shifts


def _params(c):
    return sum(n for n, _ in _tensors(c))


def _starts(sizes):
    """Where each tensor begins in a flat buffer that starts every one on a scale block."""
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += -(-n // BLOCK) * BLOCK
    return out, at


# ------------------------------------------------------------------ work

def work(case):
    c, op = case, case["op"]
    if op in ("logprobs", "dlogits"):
        live = c["R"] - _n_ignored(c)
        n = c["R"] * c["V"]
        if op == "logprobs":
            return dict(bytes=live * c["V"] * SIZE[c["dtype"]] + c["R"] * (8 + 4 * (3 if c["entropy"] else 2)),
                        flops=(7 if c["entropy"] else 4) * live * c["V"])
        return dict(bytes=(live * c["V"] + n) * SIZE[c["dtype"]] + c["R"] * (16 + (8 if c["entropy"] else 0)),
                    flops=(8 if c["entropy"] else 5) * live * c["V"])
    if op == "policy":
        n = c["B"] * c["T"]
        words = 3 + bool(c["kl"]) + 2 * bool(c["ent"]) + bool(c["token_adv"])
        return dict(bytes=n * (4 * words + 1), flops=30 * n)
    if op == "preference":
        n = 2 * c["P"] * c["T"]
        return dict(bytes=n * (9 + 4 * bool(c["ref"])), flops=4 * n)
    if op == "adamw":
        n = _params(c)
        state = 16 if c["bits"] == 32 else 4 + 8 + 32 / BLOCK   # 8 bits: returned as values too
        return dict(bytes=n * (2 * SIZE[c["p"]] * (1 if not c["master"] else 0.5) + SIZE[c["g"]]
                               + 8 * bool(c["master"]) + state), flops=(15 if c["bits"] == 32 else 30) * n)
    m = _matrices(c)
    each = 4 if c["bits"] == 32 else 1 + 4 / BLOCK
    return dict(bytes=sum(o * i * each + 4 * (o + i) for o, i in m), flops=sum(2 * o * i for o, i in m))


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _n_ignored(c):
    return int(c["ignored"] * c["R"])


def _logits(c, g):
    """Logits of a language model (scale 2.5, the target lifted by up to 12), and targets."""
    R, V, dt = c["R"], c["V"], DTYPES[c["dtype"]]
    x = torch.empty((R, V + c["pad"]), dtype=dt, device=DEV)
    for at in range(0, R, 1024):
        part = x[at:at + 1024]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV).mul_(2.5))
    x = x[:, :V]
    live = V - c["masked"]
    x[:, live:] = -math.inf
    t = torch.randint(0, live, (R,), generator=g, device=DEV)
    lift = 12 * torch.rand(R, generator=g, device=DEV)
    rows = torch.arange(R, device=DEV)
    x[rows, t] = (x[rows, t].float() + lift).to(dt)
    t[torch.randperm(R, generator=g, device=DEV)[:_n_ignored(c)]] = -1
    return x, t


def _prefix_mask(lengths, T):
    """[rows, T]: a prompt of a tenth of the answer's length is masked, then what follows the answer."""
    at = torch.arange(T, device=DEV)
    return ((at >= (lengths // 10)[:, None]) & (at < lengths[:, None])).to(torch.uint8)


def _lengths(rows, T, fill, g):
    n = (T * (1 - (1 - fill) * 2 * torch.rand(rows, generator=g, device=DEV))).long().clamp(0, T)
    if rows > 5:
        n[rows // 2] = 0                                  # an empty answer
    return n


def _padded(x, pad):
    """The same values in rows `pad` elements apart."""
    if not pad:
        return x
    out = torch.empty((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=DEV)[:, :x.shape[1]]
    return out.copy_(x)


def prepare(case, seed):
    c, op, g = case, case["op"], _gen(seed)
    s = dict(case=c)
    if op in ("logprobs", "dlogits"):
        x, t = _logits(c, g)
        R = c["R"]
        s.update(x=x, t=t, logp=torch.empty(R, device=DEV), lse=torch.empty(R, device=DEV),
                 entropy=torch.empty(R, device=DEV) if c["entropy"] else None)
        if op == "dlogits":
            for at in range(0, R, 1024):
                z = x[at:at + 1024].float() / c["tau"]
                lse = torch.logsumexp(z, 1)
                s["lse"][at:at + 1024] = lse
                if c["entropy"]:
                    p = torch.exp(z - lse[:, None])
                    s["entropy"][at:at + 1024] = lse - (p * z).nan_to_num_(0.0, 0.0, 0.0).sum(1)
            s["w"] = torch.randn(R, generator=g, device=DEV) / R
            s["h"] = torch.full((R,), -0.001 / R, device=DEV) if c["entropy"] else None
            s["dx"] = torch.empty((R, x.stride(0)), dtype=x.dtype, device=DEV)[:, :c["V"]]
        return s
    if op == "policy":
        B, T = c["B"], c["T"]
        old = -torch.empty((B, T), device=DEV).exponential_(1.0, generator=g)
        logp = old + 0.2 * torch.randn((B, T), generator=g, device=DEV)
        ref = logp + 0.3 * torch.randn((B, T), generator=g, device=DEV) if c["kl"] else None
        ent = 2 * torch.rand((B, T), generator=g, device=DEV) if c["ent"] else None
        adv = torch.randn((B, T) if c["token_adv"] else (B,), generator=g, device=DEV)
        mask = _prefix_mask(_lengths(B, T, c["fill"], g), T)
        logp[mask == 0] = -math.inf                       # what padding may hold
        s.update(logp=_padded(logp, c["pad"]), old=_padded(old, c["pad"]),
                 ref=None if ref is None else _padded(ref, c["pad"]),
                 ent=None if ent is None else _padded(ent, c["pad"]), adv=adv,
                 mask=_padded(mask, c["pad"]), loss=torch.empty(1, device=DEV),
                 seq=torch.empty(B, device=DEV), stats=torch.empty(3, device=DEV),
                 d=torch.empty((B, T), device=DEV),
                 dh=torch.empty((B, T), device=DEV) if c["ent"] else None)
        if own:
            import paper_2606_11660_gb300 as bg
            s["ws"] = bg.workspace_tensor(bg.bergson_policy_loss_workspace(B, T), DEV)
        return s
    if op == "preference":
        P, T = c["P"], c["T"]
        logp = -torch.empty((2 * P, T), device=DEV).exponential_(1.0, generator=g)
        ref = logp + 0.1 * torch.randn((2 * P, T), generator=g, device=DEV) if c["ref"] else None
        mask = _prefix_mask(_lengths(2 * P, T, c["fill"], g), T)
        logp[mask == 0] = -math.inf
        s.update(logp=_padded(logp, c["pad"]), ref=None if ref is None else _padded(ref, c["pad"]),
                 mask=_padded(mask, c["pad"]), loss=torch.empty(1, device=DEV),
                 pair=torch.empty(P, device=DEV), rewards=torch.empty(2 * P, device=DEV),
                 d=torch.empty((2 * P, T), device=DEV), beta=2.0 if c["mean"] else 0.1)
        return s
    if op == "adamw":
        return _prepare_adamw(c, s, g, seed)
    mats = _matrices(c)
    starts, n = _starts([o * i for o, i in mats])
    v = _moments_like(n, g).square_()
    s["r"] = torch.empty(sum(o for o, _ in mats), device=DEV)
    s["c"] = torch.empty(sum(i for _, i in mats), device=DEV)
    s["views"] = []
    codes = scales = None
    if c["bits"] == 8:
        codes, scales = _encode_v(v, torch.zeros(n, dtype=torch.int32, device=DEV))
    ro = co = 0
    for (o, i), at in zip(mats, starts):
        view = dict(rows=o, cols=i, at=at, n=o * i, r=s["r"][ro:ro + o], c=s["c"][co:co + i],
                    v=(v if codes is None else codes)[at:at + o * i].view(o, i),
                    scale=None if codes is None else scales[at // BLOCK:(at + o * i - 1) // BLOCK + 1])
        s["views"].append(view)
        ro, co = ro + o, co + i
    s.update(correction=1 / (1 - 0.999 ** 250), floor=1e-12)
    if own:
        import paper_2606_11660_gb300 as bg
        s["mats"] = bg.bergson_moment_matrices(
            [bg.MomentMatrix(w["v"], w["r"], w["c"], w["scale"]) for w in s["views"]])
        s["ws"] = bg.workspace_tensor(bg.bergson_factor_moments_workspace(s["mats"]), DEV)
    return s


def _moments_like(n, g):
    """Magnitudes of gradients: normal, with a spread of two decades between neighbourhoods."""
    x = torch.randn(n, generator=g, device=DEV)
    scale = torch.exp(1.2 * torch.randn(-(-n // 64), generator=g, device=DEV) - 7)
    return x * scale.repeat_interleave(64)[:n]


def _prepare_adamw(c, s, g, seed):
    tensors = _tensors(c)
    sizes = [n for n, _ in tensors]
    starts, n = _starts(sizes)
    blocks = torch.tensor([-(-k // BLOCK) for k in sizes], device=DEV)
    of = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), blocks)   # a block's tensor
    first = torch.tensor(starts, device=DEV)[of]
    at = torch.arange(n // BLOCK, device=DEV) * BLOCK - first                   # its place in it
    inside = ((at[:, None] + torch.arange(BLOCK, device=DEV))
              < torch.tensor(sizes, device=DEV)[of][:, None]).view(-1)
    p = 0.02 * torch.randn(n, generator=g, device=DEV) * inside
    grad = _moments_like(n, g) * inside
    m = 0.3 * grad + 0.2 * _moments_like(n, g) * inside
    v = (grad.square() + _moments_like(n, g).square() + 1e-12) * inside
    s.update(p=p.to(DTYPES[c["p"]]), g=grad.to(DTYPES[c["g"]]),
             master=p.clone() if c["master"] else None,
             wd=torch.tensor([w for _, w in tensors], device=DEV)[of], tensor_of=of, at=at,
             lr=3e-4, b1=0.9, b2=0.99, eps=1e-8, step=250, seed=int(seed) & 0xFFFF,
             gs=torch.full((1,), 0.731, device=DEV) if c["scaled"] else None,
             m_val=None, v_val=None, m_scale=None, v_scale=None)
    if c["bits"] == 8:
        zero = torch.zeros(n, dtype=torch.int32, device=DEV)
        s["m"], s["m_scale"] = _encode_m(m, zero)
        s["v"], s["v_scale"] = _encode_v(v, zero)
        s["m_val"], s["v_val"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    else:
        s["m"], s["v"] = m, v
    if own:
        import paper_2606_11660_gb300 as bg

        def part(key, a, b, each=1):
            return None if s[key] is None else s[key][a // each:-(-b // each)]
        s["tensors"] = bg.bergson_adamw_tensors([
            bg.AdamWTensor(param=part("p", a, a + k), grad=part("g", a, a + k),
                           master=part("master", a, a + k), m=part("m", a, a + k),
                           v=part("v", a, a + k), m_scale=part("m_scale", a, a + k, BLOCK),
                           v_scale=part("v_scale", a, a + k, BLOCK), weight_decay=w)
            for a, (k, w) in zip(starts, tensors)])
    return s


# ------------------------------------------------------- 8-bit states, plain

def _wrap(x):
    """A 64-bit pattern as the int64 that holds it."""
    x &= (1 << 64) - 1
    return x - (1 << 64) if x >> 63 else x


def _mix_host(x):
    x &= (1 << 64) - 1
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & ((1 << 64) - 1)
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & ((1 << 64) - 1)
    return x ^ (x >> 31)


def _shift(x, k):
    return (x >> k) & ((1 << (64 - k)) - 1)


def _mix(x):
    """The SplitMix64 finaliser of int64 patterns."""
    x = (x ^ _shift(x, 30)) * _wrap(0xBF58476D1CE4E5B9)
    x = (x ^ _shift(x, 27)) * _wrap(0x94D049BB133111EB)
    return x ^ _shift(x, 31)


def _dither(s):
    """16 random bits an element: four elements share an output of the SplitMix64
    sequence whose start is a function of (seed, step, tensor)."""
    base = _mix_host(s["seed"] ^ _mix_host(s["step"]))
    key = _mix(s["tensor_of"] ^ _wrap(base))
    quad = _shift(s["at"], 2)[:, None] + torch.arange(BLOCK // 4, device=DEV)
    h = _mix(key[:, None] + (quad + 1) * _wrap(GAMMA))
    h = torch.stack([h & 0xFFFF, _shift(h, 16) & 0xFFFF, _shift(h, 32) & 0xFFFF, _shift(h, 48)], 2)
    return h.view(-1).to(torch.int32)


def _block_scale(top):
    """(scale, 1 / scale) of blocks whose largest magnitude is `top`; 0 for a block of zeros."""
    scale = torch.where(top > 0, torch.clamp(top * (1 / 1.875), min=2.0 ** -126), top)
    return scale, torch.where(scale > 0, torch.reciprocal(scale), torch.zeros_like(scale))


def _encode_m(m, dither):
    """Sign, four bits of exponent, three of mantissa; `dither` (16 bits) rounds up by chance."""
    b = m.view(-1, BLOCK)
    scale, inv = _block_scale(b.abs().amax(1))
    y = (b.abs() * inv[:, None]).view(-1)
    code = ((y.view(torch.int32) + (dither << 4)) >> 20) - (112 << 3)
    code = code.clamp(0, 127) | torch.where(m < 0, 128, 0).to(torch.int32)
    return code.to(torch.uint8), scale


def _decode_m(code, scale):
    k = code.to(torch.int32)
    y = torch.where((k & 127) > 0, (((k & 127) + (112 << 3)) << 20).view(torch.float32), 0.0)
    y = torch.where(k > 127, -y, y)
    return (y.view(-1, BLOCK) * scale[:, None]).view(-1)


def _encode_v(v, dither):
    """Five bits of exponent, three of mantissa; only zero takes code 0."""
    b = v.view(-1, BLOCK)
    scale, inv = _block_scale(b.amax(1))
    y = (b * inv[:, None]).view(-1)
    code = ((y.view(torch.int32) + (dither << 4)) >> 20) - (96 << 3)
    code = torch.where(v > 0, code.clamp(1, 255), 0)
    return code.to(torch.uint8), scale


def _decode_v(code, scale):
    k = code.to(torch.int32)
    y = torch.where(k > 0, ((k + (96 << 3)) << 20).view(torch.float32), 0.0)
    return (y.view(-1, BLOCK) * scale[:, None]).view(-1)


# ------------------------------------------------------------------ passes

def run(state):
    return {"logprobs": _logprobs, "dlogits": _dlogits, "policy": _policy,
            "preference": _preference, "adamw": _adamw, "moments": _moments}[state["case"]["op"]](state)


def _logprobs(s):
    c = s["case"]
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_token_logprobs(s["x"], s["t"], c["tau"], s["logp"], s["lse"], s["entropy"])
        return {k: s[k] for k in ("logp", "lse", "entropy")}
    z = s["x"].float() * (1.0 / c["tau"])
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1)
    lse = top[:, 0] + torch.log(total)
    live = s["t"] >= 0
    logp = z.gather(1, s["t"].clamp(min=0)[:, None])[:, 0] - lse
    entropy = None
    if c["entropy"]:
        shifted = torch.where(e > 0, e * (z - top), 0.0).sum(1)
        entropy = torch.where(live, torch.log(total) - shifted / total, 0.0)
    return {"logp": torch.where(live, logp, 0.0), "lse": torch.where(live, lse, 0.0), "entropy": entropy}


def _dlogits(s):
    c = s["case"]
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_token_logprobs_backward(s["x"], s["t"], c["tau"], s["lse"], s["entropy"], s["w"],
                                           s["h"], s["dx"])
        return s["dx"]
    live = (s["t"] >= 0)[:, None]
    logq = s["x"].float() * (1.0 / c["tau"]) - s["lse"][:, None]
    q = torch.exp(logq)
    d = -s["w"][:, None] * q
    if c["entropy"]:
        d = d - torch.where(q > 0, s["h"][:, None] * q * (logq + s["entropy"][:, None]), 0.0)
    d.scatter_add_(1, s["t"].clamp(min=0)[:, None], s["w"][:, None])
    return torch.where(live, d * (1.0 / c["tau"]), 0.0).to(s["x"].dtype)


CLIP = (0.2, 0.28)
NORM_TOKENS = 1024.0


def _policy(s):
    c = s["case"]
    if own:
        import paper_2606_11660_gb300 as bg
        kind = {"token_mean": bg.BERGSON_POLICY_TOKEN_MEAN, "seq_mean": bg.BERGSON_POLICY_SEQ_MEAN,
                "sum_norm": bg.BERGSON_POLICY_SUM_NORM}[c["reduction"]]
        bg.bergson_policy_loss(s["logp"], s["old"], s["ref"], s["ent"], s["adv"], s["mask"], CLIP[0],
                               CLIP[1], c["kl"], c["ent"], kind, NORM_TOKENS, s["loss"], s["seq"],
                               s["stats"], s["d"], s["dh"], s["ws"])
        return {k: s[k] for k in ("loss", "seq", "stats", "d", "dh")}
    on = s["mask"] != 0
    adv = s["adv"] if c["token_adv"] else s["adv"][:, None]
    ratio = torch.exp(torch.where(on, s["logp"] - s["old"], 0.0))
    held = ratio.clamp(1 - CLIP[0], 1 + CLIP[1])
    plain, clipped = ratio * adv, held * adv
    loss = -torch.minimum(plain, clipped)
    grad = torch.where(plain <= clipped, -plain, 0.0)
    kl = torch.zeros_like(loss)
    if c["kl"]:
        gap = torch.where(on, s["ref"] - s["logp"], 0.0)
        up = torch.exp(gap)
        kl = up - gap - 1
        loss = loss + c["kl"] * kl
        grad = grad + c["kl"] * (1 - up)
    if c["ent"]:
        loss = loss - c["ent"] * s["ent"]
    n_row = on.sum(1).float()
    n = n_row.sum()
    if c["reduction"] == "token_mean":
        w = (1 / n.clamp(min=1)).expand(c["B"])
    elif c["reduction"] == "seq_mean":
        w = 1 / (c["B"] * n_row.clamp(min=1))
    else:
        w = torch.full((c["B"],), 1 / (c["B"] * NORM_TOKENS), device=DEV)
    seq = torch.where(on, loss, 0.0).sum(1) * w
    apart = on & (plain > clipped)
    stats = torch.stack([torch.where(on, kl, 0.0).sum() / n.clamp(min=1),
                         apart.sum().float() / n.clamp(min=1), n])
    return {"loss": seq.sum().view(1), "seq": seq, "stats": stats,
            "d": torch.where(on, grad * w[:, None], 0.0),
            "dh": torch.where(on, -c["ent"] * w[:, None], 0.0) if c["ent"] else None}


def _preference(s):
    c, P = s["case"], s["case"]["P"]
    if own:
        import paper_2606_11660_gb300 as bg
        kind = {"sigmoid": bg.BERGSON_PREFERENCE_SIGMOID, "hinge": bg.BERGSON_PREFERENCE_HINGE,
                "squared": bg.BERGSON_PREFERENCE_SQUARED}[c["kind"]]
        bg.bergson_preference_loss(s["logp"], s["ref"], s["mask"], kind, s["beta"], c["margin"],
                                   c["smooth"], c["mean"], s["loss"], s["pair"], s["rewards"],
                                   s["d"])
        return {k: s[k] for k in ("loss", "pair", "rewards", "d")}
    on, beta = s["mask"] != 0, s["beta"]
    gap = s["logp"] - s["ref"] if c["ref"] else s["logp"]
    total = torch.where(on, gap, 0.0).sum(1)
    share = torch.ones_like(total)
    if c["mean"]:
        share = 1 / on.sum(1).float().clamp(min=1)
    mean = total * share
    x = beta * (mean[:P] - mean[P:]) - c["margin"]
    up, down = 1 - c["smooth"], c["smooth"]

    def softplus(y):
        return torch.clamp(y, min=0) + torch.log1p(torch.exp(-y.abs()))
    if c["kind"] == "sigmoid":
        pair = up * softplus(-x) + down * softplus(x)
        slope = down / (1 + torch.exp(-x)) - up / (1 + torch.exp(x))
    elif c["kind"] == "hinge":
        pair = up * torch.clamp(1 - x, min=0) + down * torch.clamp(1 + x, min=0)
        slope = down * (x > -1).float() - up * (x < 1).float()
    else:
        a, b = (x - 0.5) / beta, (x + 0.5) / beta
        pair = up * a * a + down * b * b
        slope = 2 * (up * a + down * b) / beta
    per = slope * beta / P
    per = torch.cat([per, -per]) * share
    return {"loss": pair.mean().view(1), "pair": pair, "rewards": beta * mean,
            "d": torch.where(on, per[:, None], 0.0)}


def _adamw(s):
    c = s["case"]
    eight = c["bits"] == 8
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_adamw_step(s["tensors"], s["lr"], s["b1"], s["b2"], s["eps"], s["step"],
                              seed=s["seed"], grad_scale=s["gs"])
        if eight:
            bg.bergson_adamw_state_values(s["m"], s["m_scale"], bg.BERGSON_MOMENT_FIRST, s["m_val"])
            bg.bergson_adamw_state_values(s["v"], s["v_scale"], bg.BERGSON_MOMENT_SECOND, s["v_val"])
    else:
        g = s["g"].float()
        if s["gs"] is not None:
            g = g * s["gs"]
        b1, b2 = s["b1"], s["b2"]
        m = _decode_m(s["m"], s["m_scale"]) if eight else s["m"]
        v = _decode_v(s["v"], s["v_scale"]) if eight else s["v"]
        m = m * b1 + g * (1 - b1)
        v = v * b2 + g * g * (1 - b2)
        w = s["master"] if c["master"] else s["p"].float()
        step = (m * (1 / (1 - b1 ** s["step"]))) / (torch.sqrt(v * (1 / (1 - b2 ** s["step"]))) + s["eps"])
        wd = (s["lr"] * s["wd"])[:, None]
        w = w - ((w.view(-1, BLOCK) * wd).view(-1) + s["lr"] * step)
        s["p"].copy_(w)
        if c["master"]:
            s["master"].copy_(w)
        if eight:
            dither = _dither(s)
            code, scale = _encode_m(m, dither)
            s["m"].copy_(code), s["m_scale"].copy_(scale)
            code, scale = _encode_v(v, dither)
            s["v"].copy_(code), s["v_scale"].copy_(scale)
            s["m_val"].copy_(_decode_m(s["m"], s["m_scale"]))
            s["v_val"].copy_(_decode_v(s["v"], s["v_scale"]))
        else:
            s["m"].copy_(m), s["v"].copy_(v)
    return {"p": s["p"], "master": s["master"], "m": s["m_val" if eight else "m"],
            "v": s["v_val" if eight else "v"]}


def _moments(s):
    c = s["case"]
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_factor_moments(s["mats"], s["correction"], s["floor"], s["ws"])
    else:
        [_factor(w, c["bits"], s["correction"], s["floor"]) for w in s["views"]]
    return {"r": s["r"], "c": s["c"]}


def _factor(w, bits, correction, floor):
    v = w["v"]
    if bits == 8:
        k = v.reshape(-1).to(torch.int32)
        y = torch.where(k > 0, ((k + (96 << 3)) << 20).view(torch.float32), 0.0)
        v = (y * w["scale"].repeat_interleave(BLOCK)[:k.numel()]).view(v.shape)
    v = v * correction + floor
    rows, cols = v.mean(1), v.mean(0)
    w["r"].copy_(rows)
    w["c"].copy_(cols / rows.mean())


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    return {"logprobs": _exact_logprobs, "dlogits": _exact_dlogits, "policy": _exact_policy,
            "preference": _exact_preference, "adamw": _exact_adamw, "moments": _exact_moments}[case["op"]](s)


def _exact_logprobs(s):
    c, outs = s["case"], []
    for x, t in zip(s["x"].split(512), s["t"].split(512)):
        z = x.double() / c["tau"]
        lse = torch.logsumexp(z, 1)
        q = torch.softmax(z, 1)
        logp = z[torch.arange(len(t), device=DEV), t.clamp(min=0)] - lse
        h = -torch.special.xlogy(q, q).sum(1)
        dead = t < 0
        outs.append([y.masked_fill(dead, 0.0) for y in (logp, lse, h)])
    logp, lse, h = (torch.cat(y) for y in zip(*outs))
    return {"logp": logp, "lse": lse, "entropy": h if c["entropy"] else None}


def _exact_dlogits(s):
    c, outs = s["case"], []
    if c["R"] * c["V"] > 600_000_000:
        return None
    for at in range(0, c["R"], 512):
        part = slice(at, at + 512)
        t = s["t"][part]
        q = torch.exp(s["x"][part].double() / c["tau"] - s["lse"][part].double()[:, None])
        w = s["w"][part].double()[:, None]
        d = -w * q
        d[torch.arange(len(t), device=DEV), t.clamp(min=0)] += w[:, 0]
        if c["entropy"]:
            d -= s["h"][part].double()[:, None] * (torch.special.xlogy(q, q) + q * s["entropy"][part].double()[:, None])
        outs.append((d / c["tau"]).masked_fill((t < 0)[:, None], 0.0))
    return torch.cat(outs)


def _exact_policy(s):
    c = s["case"]
    rows = []
    n = float(s["mask"].sum(dtype=torch.int64))
    for b in torch.arange(c["B"], device=DEV).split(max(1, (1 << 22) // c["T"])):
        on = s["mask"][b].bool()
        l = s["logp"][b].double().masked_fill(~on, 0.0)
        old = s["old"][b].double().masked_fill(~on, 0.0)
        a = s["adv"][b].double().view(len(b), -1).expand(l.shape)
        r = (l - old).exp()
        limit = torch.where(a > 0, torch.full_like(a, 1 + CLIP[1]), torch.full_like(a, 1 - CLIP[0]))
        off = torch.where(a > 0, r > limit, (a < 0) & (r < limit))
        surrogate = torch.where(off, limit, r) * a
        value, slope, kl = -surrogate, -(r * a).masked_fill(off, 0.0), torch.zeros_like(l)
        if c["kl"]:
            u = s["ref"][b].double().masked_fill(~on, 0.0) - l
            kl = torch.expm1(u) - u
            value, slope = value + c["kl"] * kl, slope - c["kl"] * torch.expm1(u)
        if c["ent"]:
            value = value - c["ent"] * s["ent"][b].double()
        k = on.sum(1).double()
        if c["reduction"] == "token_mean":
            w = torch.full_like(k, 1 / max(n, 1.0))
        elif c["reduction"] == "seq_mean":
            w = 1 / (k.clamp(min=1) * c["B"])
        else:
            w = torch.full_like(k, 1 / (c["B"] * NORM_TOKENS))
        rows.append(((value * on).sum(1) * w, (kl * on).sum(), (off & on).sum().double(),
                     slope * on * w[:, None], -c["ent"] * on * w[:, None]))
    seq, kl, off, d, dh = zip(*rows)
    seq = torch.cat(seq)
    stats = torch.stack([sum(kl) / max(n, 1.0), sum(off) / max(n, 1.0), torch.tensor(n, device=DEV).double()])
    return {"loss": seq.sum().view(1), "seq": seq, "stats": stats, "d": torch.cat(d),
            "dh": torch.cat(dh) if c["ent"] else None}


def _exact_preference(s):
    c, P, beta = s["case"], s["case"]["P"], s["beta"]
    on = s["mask"].bool()
    gap = s["logp"].double().masked_fill(~on, 0.0)
    if c["ref"]:
        gap = gap - s["ref"].double().masked_fill(~on, 0.0)
    k = on.sum(1).clamp(min=1).double() if c["mean"] else torch.ones(2 * P, device=DEV).double()
    score = gap.sum(1) / k
    x = (beta * (score[:P] - score[P:]) - c["margin"]).requires_grad_(True)
    f = torch.nn.functional
    one = {"sigmoid": lambda y: -f.logsigmoid(y), "hinge": lambda y: f.relu(1 - y),
           "squared": lambda y: ((y - 0.5) / beta) ** 2}[c["kind"]]
    pair = (1 - c["smooth"]) * one(x) + c["smooth"] * one(-x)
    pair.sum().backward()
    d = torch.cat([x.grad, -x.grad]) * beta / P / k
    pair = pair.detach()
    return {"loss": pair.mean().view(1), "pair": pair, "rewards": beta * score, "d": d[:, None] * on}


def _exact_adamw(s):
    """For 8-bit states m and v before their rounding."""
    c = s["case"]
    m, v = s["m"], s["v"]
    if c["bits"] == 8:
        k = m.double().view(-1, BLOCK)
        mag = k % 128
        size = torch.where(mag > 0, torch.exp2(torch.floor(mag / 8) - 15) * (1 + (mag % 8) / 8), 0.0)
        m = (torch.where(k >= 128, -size, size) * s["m_scale"].double()[:, None]).view(-1)
        k = v.double().view(-1, BLOCK)
        size = torch.where(k > 0, torch.exp2(torch.floor(k / 8) - 31) * (1 + (k % 8) / 8), 0.0)
        v = (size * s["v_scale"].double()[:, None]).view(-1)
    g = s["g"].double() * (1.0 if s["gs"] is None else s["gs"].double())
    m = s["b1"] * m.double() + (1 - s["b1"]) * g
    v = s["b2"] * v.double() + (1 - s["b2"]) * g ** 2
    w = (s["master"] if c["master"] else s["p"]).double()
    up = m / (1 - s["b1"] ** s["step"]) / ((v / (1 - s["b2"] ** s["step"])).sqrt() + s["eps"])
    w = w - s["lr"] * (up + s["wd"].double().repeat_interleave(BLOCK) * w)
    return {"p": w, "master": w if c["master"] else None, "m": m, "v": v}


def _exact_moments(s):
    rows, cols = [], []
    for w in s["views"]:
        v = w["v"].double()
        if w["scale"] is not None:
            v = torch.where(v > 0, torch.exp2(torch.floor(v / 8) - 31) * (1 + (v % 8) / 8), 0.0)
            v = v * w["scale"].double().repeat_interleave(BLOCK)[:v.numel()].view(v.shape)
        v = v * s["correction"] + s["floor"]
        rows.append(v.sum(1) / w["cols"])
        cols.append(v.sum(0) / w["rows"] / v.mean())
    return {"r": torch.cat(rows), "c": torch.cat(cols)}
