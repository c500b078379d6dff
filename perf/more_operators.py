"""Timed cases of the operators that a training step has around its linear
layers: the model's ends and the optimiser of its matrices.

  norm     layer norm (or its form without a mean): outputs and row statistics
  dnorm    its backward pass: gradients at the input, the weight and the bias
  embed    embedding lookup with a scale
  dembed   its backward pass: the table's gradient, dense or added to one
  muon     one Muon step over many matrices: momentum, orthogonalisation by
           Newton-Schulz products, weight update

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
EPS = 1e-5
QUINTIC = (3.4445, -4.7750, 2.0315)
ITERATIONS = 5
MAX_NORM_ELEMENTS = 65_536 * 2048
MAX_DNORM_ELEMENTS = 65_536 * 2048
MAX_EMBED_ELEMENTS = 65_536 * 4096
MAX_DEMBED_ELEMENTS = 65_536 * 2048 + 50_304 * 2048
MAX_MUON_FLOPS = 6.9e12             # times the products at work


def listed():
    return [
        # The last positions of a few prompts on their way to the output layer.
        dict(name="norm_step", op="norm", R=5, d=768, dtype="bf16", w="bf16", pad=0, kind="layer"),
        # One norm of a training batch of 32 sequences of 2048 tokens.
        dict(name="norm_batch", op="norm", R=65_536, d=2048, dtype="bf16", w="f32", pad=0,
             kind="layer"),
        # The backward pass of a small ragged batch without a mean, rows apart, 16-bit floats.
        dict(name="dnorm_odd", op="dnorm", R=1031, d=1029, dtype="f16", w="f16", pad=3, kind="rms"),
        # The backward pass of the training batch.
        dict(name="dnorm_batch", op="dnorm", R=65_536, d=2048, dtype="bf16", w="f32", pad=0,
             kind="layer"),
        # One decoding step's lookups.
        dict(name="embed_step", op="embed", R=5, V=50_257, d=768, dtype="bf16", pad=0, ignored=0.0,
             scaled=False),
        # A training batch's lookups in a wide table with a scale; a tenth of the tokens is padding.
        dict(name="embed_batch", op="embed", R=65_536, V=131_072, d=4096, dtype="bf16", pad=0,
             ignored=0.1, scaled=True),
        # The output layer's gradient is there already and the lookups' is added: tied weights in a
        # debugging batch of 8 answers of 97 tokens.
        dict(name="dembed_tied", op="dembed", R=776, V=50_257, d=768, dtype="bf16", t="f32", pad=0,
             ignored=0.3, scaled=False, add=True),
        # The table's whole gradient of a training batch.
        dict(name="dembed_batch", op="dembed", R=65_536, V=50_304, d=2048, dtype="bf16", t="bf16",
             pad=0, ignored=0.1, scaled=True, add=False),
        # The matrices of one small block with master copies, at fp32 accuracy.
        dict(name="muon_small", op="muon", d=264, ff=1056, layers=1, p="bf16", g="bf16",
             master=True, nesterov=True, products=3, scaled=False),
        # Ten blocks of a small model with master copies, at fp32 accuracy.
        dict(name="muon_model", op="muon", d=640, ff=2560, layers=10, p="bf16", g="bf16",
             master=True, nesterov=True, products=3, scaled=True),
        # Four wide blocks, weights held in bf16 alone, at 16-bit products.
        dict(name="muon_blocks", op="muon", d=2048, ff=8192, layers=4, p="bf16", g="bf16",
             master=False, nesterov=True, products=1, scaled=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "dnorm", "embed", "dembed", "muon"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("norm", "dnorm"):
        while True:
            c = dict(op=op, R=_log(rng, 1, 131_072), d=_log(rng, 24, 16_384), dtype=dtype,
                     w=rng.choice([dtype, "f32"]), pad=rng.choice([0, 0, 3, 8]),
                     kind=rng.choice(["layer", "rms"]))
            if rng.random() < 0.6:
                c["d"] = -(-c["d"] // 32) * 32
            if c["R"] * (c["d"] + c["pad"]) * SIZE[dtype] <= 2 * MAX_NORM_ELEMENTS:
                return c
    if op == "embed":
        while True:
            c = dict(op=op, R=_log(rng, 1, 131_072), V=_log(rng, 96, 262_144), d=_log(rng, 24, 8192),
                     dtype=dtype, pad=rng.choice([0, 0, 3, 8]), ignored=rng.choice([0.0, 0.1, 0.5]),
                     scaled=rng.random() < 0.5)
            if rng.random() < 0.6:
                c["d"] = -(-c["d"] // 32) * 32
            if work(c)["bytes"] <= 2 * SIZE["bf16"] * MAX_EMBED_ELEMENTS // 2 and (
                    c["V"] * c["d"] <= 2 * MAX_EMBED_ELEMENTS):
                return c
    if op == "dembed":
        while True:
            c = dict(op=op, R=_log(rng, 1, 262_144), V=_log(rng, 96, 262_144), d=_log(rng, 24, 8192),
                     dtype=dtype, t=rng.choice([dtype, "f32"]), pad=rng.choice([0, 0, 3, 8]),
                     ignored=rng.choice([0.0, 0.1, 0.5]), scaled=rng.random() < 0.5,
                     add=rng.random() < 0.4)
            if rng.random() < 0.6:
                c["d"] = -(-c["d"] // 32) * 32
            if (c["R"] * SIZE[dtype] + c["V"] * SIZE[c["t"]]) * c["d"] <= 2 * MAX_DEMBED_ELEMENTS:
                return c
    while True:
        c = dict(op=op, d=_log(rng, 24, 2048), ff=0, layers=_log(rng, 1, 12),
                 p=rng.choice(["bf16", "bf16", "f32"]), g="", master=False,
                 nesterov=rng.random() < 0.7, products=rng.choice([3, 3, 1]),
                 scaled=rng.random() < 0.5)
        c["ff"] = c["d"] * rng.choice([2, 4]) + rng.choice([0, 0, 1, 8])
        if c["products"] == 1:
            c["p"] = "bf16"
        c["g"] = rng.choice([c["p"], c["p"], "f32"])
        c["master"] = c["p"] != "f32" and c["products"] == 3 and rng.random() < 0.7
        if work(c)["flops"] * c["products"] <= MAX_MUON_FLOPS:
            return c


# ------------------------------------------------------------------ shapes and work

def _kinds(c):
    """(rows, columns) of a block's weight matrices."""
    d, ff = c["d"], c["ff"]
    return [(3 * d, d), (d, d), (ff, d), (d, ff)]


def _matrices(c):
    """(rows, columns) of all layers' weight matrices, kind by kind."""
    return [k for k in _kinds(c) for _ in range(c["layers"])]


def _starts(sizes):
    """Where each matrix begins in a flat buffer that starts every one on 256 elements."""
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += -(-n // 256) * 256
    return out, at


def _n_ignored(c):
    return int(c["ignored"] * c["R"])


def _distinct(c):
    """Rows of the table that R lookups of Zipf's law are expected to meet."""
    live, V = c["R"] - _n_ignored(c), c["V"]
    k = torch.arange(V, dtype=torch.float64)
    p = torch.log1p(1 / (k + 1)) / math.log(V + 1)
    return int((1 - torch.exp(live * torch.log1p(-p))).sum())


def work(case):
    c, op = case, case["op"]
    if op in ("norm", "dnorm"):
        n, e, w = c["R"] * c["d"], SIZE[c["dtype"]], c["d"] * SIZE[c["w"]]
        stats = 4 * c["R"] * (2 if c["kind"] == "layer" else 1)
        sides = 2 if c["kind"] == "layer" else 1
        if op == "norm":
            return dict(bytes=2 * n * e + sides * w + stats, flops=8 * n)
        return dict(bytes=3 * n * e + w + 4 * c["d"] * sides + stats, flops=14 * n)
    if op == "embed":
        n, e = c["R"] * c["d"], SIZE[c["dtype"]]
        return dict(bytes=n * e + _distinct(c) * c["d"] * e + 8 * c["R"], flops=n)
    if op == "dembed":
        live = c["R"] - _n_ignored(c)
        rows = 2 * _distinct(c) if c["add"] else c["V"]
        return dict(bytes=live * c["d"] * SIZE[c["dtype"]] + 8 * c["R"] + rows * c["d"] * SIZE[c["t"]],
                    flops=live * c["d"])
    flops = elements = 0
    for o, i in _matrices(c):
        m, n = min(o, i), max(o, i)
        elements += m * n
        flops += ITERATIONS * (3 * m * m * n + m ** 3)    # symmetric products by their half
    weights = 2 * SIZE[c["p"]] if not c["master"] else SIZE[c["p"]] + 8
    return dict(bytes=elements * (weights + SIZE[c["g"]] + 8), flops=flops)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(R, d, pad, dtype):
    """[R, d] whose rows are `pad` elements apart."""
    return torch.empty((R, d + pad), dtype=DTYPES[dtype], device=DEV)[:, :d]


def _stream(c, g):
    """Rows of a residual stream: a scale a row, some offset, a few channels far above the rest."""
    R, d = c["R"], c["d"]
    x = _rows(R, d, c["pad"], c["dtype"])
    far = torch.ones(d, device=DEV)
    far[torch.randperm(d, generator=g, device=DEV)[:max(1, d // 256)]] = 20.0
    for at in range(0, R, 16_384):
        part = x[at:at + 16_384]
        y = torch.randn(part.shape, generator=g, device=DEV).mul_(far).add_(0.3)
        part.copy_(y.mul_(torch.exp(0.5 * torch.randn((len(y), 1), generator=g, device=DEV))))
    return x


def _noise(R, d, pad, dtype, scale, g):
    x = _rows(R, d, pad, dtype)
    for at in range(0, R, 16_384):
        part = x[at:at + 16_384]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV).mul_(scale))
    return x


def _ids(c, g):
    """Tokens by Zipf's law; the left-out ones are -1."""
    R, V = c["R"], c["V"]
    u = torch.rand(R, generator=g, device=DEV, dtype=torch.float64)
    t = (torch.exp(u * math.log(V + 1)) - 1).long().clamp(0, V - 1)
    t[torch.randperm(R, generator=g, device=DEV)[:_n_ignored(c)]] = -1
    return t


def prepare(case, seed):
    c, op, g = case, case["op"], _gen(seed)
    s = dict(case=c)
    if op in ("norm", "dnorm"):
        R, d = c["R"], c["d"]
        layer = c["kind"] == "layer"
        s["x"] = _stream(c, g)
        s["w"] = (1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(DTYPES[c["w"]])
        s["b"] = (0.1 * torch.randn(d, generator=g, device=DEV)).to(DTYPES[c["w"]]) if layer else None
        s["mean"] = torch.empty(R, device=DEV) if layer else None
        s["rstd"] = torch.empty(R, device=DEV)
        if op == "norm":
            s["y"] = _rows(R, d, c["pad"], c["dtype"])
            return s
        s["dy"] = _noise(R, d, c["pad"], c["dtype"], 0.05, g)
        s["dx"] = _rows(R, d, c["pad"], c["dtype"])
        s["dw"] = torch.empty(d, device=DEV)
        s["db"] = torch.empty(d, device=DEV) if layer else None
        for at in range(0, R, 16_384):
            x = s["x"][at:at + 16_384].float()
            mean = x.mean(1, keepdim=True) if layer else 0.0
            s["rstd"][at:at + 16_384] = torch.rsqrt((x - mean).square().mean(1) + EPS)
            if layer:
                s["mean"][at:at + 16_384] = mean[:, 0]
        if own:
            import paper_2606_11660_gb300 as bg
            s["ws"] = bg.workspace_tensor(bg.bergson_norm_backward_workspace(R, d), DEV)
        return s
    if op in ("embed", "dembed"):
        R, V, d = c["R"], c["V"], c["d"]
        s["ids"] = _ids(c, g)
        s["scale"] = math.sqrt(d) if c["scaled"] else 1.0
        if op == "embed":
            s["table"] = _noise(V, d, c["pad"], c["dtype"], 0.02, g)
            s["out"] = _rows(R, d, c["pad"], c["dtype"])
            return s
        s["dy"] = _noise(R, d, c["pad"], c["dtype"], 0.05, g)
        s["dt"] = (_noise(V, d, c["pad"], c["t"], 0.05, g) if c["add"]
                   else _rows(V, d, c["pad"], c["t"]))
        if own:
            import paper_2606_11660_gb300 as bg
            s["ws"] = bg.workspace_tensor(bg.bergson_embedding_backward_workspace(R, V, d), DEV)
        return s
    return _prepare_muon(c, s, g)


def _gradients(mats, starts, n, g):
    """Gradients of weights: a few strong directions above noise; zeros between the matrices."""
    x = torch.zeros(n, device=DEV)
    for (o, i), at in zip(mats, starts):
        r = min(8, o, i)
        left, right = (torch.randn((k, r), generator=g, device=DEV) for k in (o, i))
        part = torch.randn((o, i), generator=g, device=DEV)
        x[at:at + o * i] = part.addmm_(left, right.t(), alpha=0.5).mul_(1e-3).view(-1)
    return x


def _prepare_muon(c, s, g):
    mats = _matrices(c)
    starts, n = _starts([o * i for o, i in mats])
    grad = _gradients(mats, starts, n, g)
    s["m"] = _gradients(mats, starts, n, g).mul_(0.5).add_(grad, alpha=0.3)
    s["g"] = grad.to(DTYPES[c["g"]])
    p = torch.zeros(n, device=DEV)
    for (o, i), at in zip(mats, starts):
        p[at:at + o * i] = 0.02 * torch.randn(o * i, generator=g, device=DEV)
    s["p"] = p.to(DTYPES[c["p"]])
    s["master"] = p if c["master"] else None
    s["views"] = [dict(o=o, i=i, a=at, z=at + o * i, scale=0.2 * math.sqrt(max(o, i)))
                  for (o, i), at in zip(mats, starts)]
    s["kinds"] = [dict(o=o, i=i, a=starts[k * c["layers"]], scale=0.2 * math.sqrt(max(o, i)))
                  for k, (o, i) in enumerate(_kinds(c))]
    s.update(lr=3e-4, beta=0.95, wd=0.1,
             gs=torch.full((1,), 0.731, device=DEV) if c["scaled"] else None)
    if own:
        import paper_2606_11660_gb300 as bg

        def part(key, v):
            return None if s[key] is None else s[key][v["a"]:v["z"]].view(v["o"], v["i"])
        s["tensors"] = bg.bergson_muon_tensors([
            bg.MuonTensor(param=part("p", v), grad=part("g", v), m=part("m", v),
                          master=part("master", v), ortho_scale=v["scale"], weight_decay=s["wd"])
            for v in s["views"]])
        s["coefficients"] = [QUINTIC] * ITERATIONS
        s["ws"] = bg.workspace_tensor(bg.bergson_muon_step_workspace(s["tensors"], c["products"]), DEV)
    return s


# ------------------------------------------------------------------ passes

def run(state):
    return {"norm": _norm, "dnorm": _dnorm, "embed": _embed, "dembed": _dembed,
            "muon": _muon}[state["case"]["op"]](state)


def _norm(s):
    c = s["case"]
    layer = c["kind"] == "layer"
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_norm(s["x"], s["w"], s["b"], bg.BERGSON_NORM_LAYER if layer else bg.BERGSON_NORM_RMS,
                        EPS, s["y"], s["mean"], s["rstd"])
        return {k: s[k] for k in ("y", "mean", "rstd")}
    x = s["x"].float()
    mean = None
    if layer:
        mean = x.mean(1)
        x = x - mean[:, None]
    rstd = torch.rsqrt((x * x).mean(1) + EPS)
    y = x * rstd[:, None] * s["w"].float()
    if layer:
        y = y + s["b"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _dnorm(s):
    c = s["case"]
    layer = c["kind"] == "layer"
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_norm_backward(s["x"], s["w"], bg.BERGSON_NORM_LAYER if layer else bg.BERGSON_NORM_RMS,
                                 s["mean"], s["rstd"], s["dy"], s["dx"], s["dw"], s["db"], s["ws"])
        return {k: s[k] for k in ("dx", "dw", "db")}
    x, dy = s["x"].float(), s["dy"].float()
    if layer:
        x = x - s["mean"][:, None]
    x = x * s["rstd"][:, None]
    h = dy * s["w"].float()
    along = (h * x).mean(1, keepdim=True)
    dx = h - x * along
    if layer:
        dx = dx - h.mean(1, keepdim=True)
    return {"dx": (dx * s["rstd"][:, None]).to(s["x"].dtype), "dw": (dy * x).sum(0),
            "db": dy.sum(0) if layer else None}


def _embed(s):
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_embedding(s["table"], s["ids"], s["scale"], s["out"])
        return s["out"]
    y = s["table"][s["ids"].clamp(min=0)].float() * s["scale"]
    return torch.where((s["ids"] >= 0)[:, None], y, 0.0).to(s["table"].dtype)


def _dembed(s):
    c = s["case"]
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_embedding_backward(s["dy"], s["ids"], s["scale"], s["dt"], c["add"], s["ws"])
        return s["dt"]
    live = s["ids"] >= 0
    dy = torch.where(live[:, None], s["dy"].float(), 0.0)
    total = torch.zeros((c["V"], c["d"]), device=DEV).index_add_(0, s["ids"].clamp(min=0), dy)
    total = total * s["scale"]
    if c["add"]:
        total = total + s["dt"].float()
    s["dt"].copy_(total)
    return s["dt"]


def _layers(flat, v, layers):
    """[layers, rows, columns]: the matrices of one kind."""
    o, i = v["o"], v["i"]
    return flat.as_strided((layers, o, i), (-(-o * i // 256) * 256, i, 1), flat.storage_offset() + v["a"])


def _muon(s):
    c = s["case"]
    if own:
        import paper_2606_11660_gb300 as bg
        bg.bergson_muon_step(s["tensors"], s["lr"], s["beta"], c["nesterov"], s["coefficients"],
                             c["products"], s["ws"], grad_scale=s["gs"])
        return {k: s[k] for k in ("p", "master", "m")}
    g = s["g"].float()
    if s["gs"] is not None:
        g = g * s["gs"]
    b = s["beta"]
    s["m"].mul_(b).add_(g, alpha=1 - b)
    u = s["m"] * b + g * (1 - b) if c["nesterov"] else s["m"]
    w = s["master"] if c["master"] else s["p"].float()
    for v in s["kinds"]:
        x, part = _layers(u, v, c["layers"]), _layers(w, v, c["layers"])
        tall = v["o"] > v["i"]
        if tall:
            x = x.mT
        x = x / torch.sqrt((x * x).sum((1, 2), keepdim=True))
        for _ in range(ITERATIONS):
            a = x @ x.mT
            x = QUINTIC[0] * x + (QUINTIC[1] * a + QUINTIC[2] * (a @ a)) @ x
        if tall:
            x = x.mT
        part.sub_(s["lr"] * (v["scale"] * x + s["wd"] * part))
    s["p"].copy_(w)
    return {"p": s["p"], "master": s["master"], "m": s["m"]}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    return {"norm": _exact_norm, "dnorm": _exact_dnorm, "embed": _exact_embed,
            "dembed": _exact_dembed, "muon": _exact_muon}[case["op"]](s)


def _exact_norm(s):
    layer = s["case"]["kind"] == "layer"
    outs = []
    for x in s["x"].split(8192):
        x = x.double()
        mean = x.sum(1) / x.shape[1] if layer else torch.zeros(len(x), device=DEV).double()
        var = x.square().sum(1) / x.shape[1] - mean ** 2
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(-mean * rstd, x.t(), rstd).t() * s["w"].double()
        outs.append((y + s["b"].double() if layer else y, mean, rstd))
    y, mean, rstd = (torch.cat(k) for k in zip(*outs))
    return {"y": y, "mean": mean if layer else None, "rstd": rstd}


def _exact_dnorm(s):
    """The adjoint of the normalisation as a projection: what is along the row's unit vectors goes."""
    layer, outs, d = s["case"]["kind"] == "layer", [], s["case"]["d"]
    dw = torch.zeros(d, device=DEV).double()
    db = torch.zeros(d, device=DEV).double()
    for at in range(0, s["case"]["R"], 8192):
        x, dy = (s[k][at:at + 8192].double() for k in ("x", "dy"))
        r = s["rstd"][at:at + 8192].double()
        if layer:
            x = x - s["mean"][at:at + 8192].double()[:, None]
        x = torch.einsum("rd,r->rd", x, r)
        dw += torch.einsum("rd,rd->d", x, dy)
        db += dy.sum(0)
        h = dy * s["w"].double()
        out = h - torch.einsum("rd,r->rd", x, torch.einsum("rd,rd->r", h, x) / d)
        if layer:
            out -= h.sum(1, keepdim=True) / d
        outs.append(torch.einsum("rd,r->rd", out, r))
    return {"dx": torch.cat(outs), "dw": dw, "db": db if layer else None}


def _exact_embed(s):
    out = torch.zeros(s["out"].shape, device=DEV).double()
    on = torch.nonzero(s["ids"] >= 0)[:, 0]
    for rows in on.split(16_384):
        out[rows] = s["table"].index_select(0, s["ids"][rows]).double() * s["scale"]
    return out


def _exact_dembed(s):
    c = s["case"]
    if c["V"] * c["d"] > 1 << 30:
        return None
    out = torch.zeros((c["V"], c["d"]), device=DEV).double()
    order = torch.argsort(s["ids"])
    order = order[s["ids"][order] >= 0]
    for rows in order.split(16_384):
        out.index_add_(0, s["ids"][rows], s["dy"].index_select(0, rows).double(), alpha=s["scale"])
    return out + s["dt"].double() if c["add"] else out


def _exact_muon(s):
    """The iteration as a polynomial in the eigenvalues of the smaller Gram matrix."""
    c = s["case"]
    if work(c)["flops"] > 2e12 or sum(min(o, i) ** 3 for o, i in _matrices(c)) > 40 * 640 ** 3:
        return None
    g = s["g"].double() * (1.0 if s["gs"] is None else s["gs"].double())
    m = s["m"].double().lerp(g, 1 - s["beta"])
    u = m.lerp(g, 1 - s["beta"]) if c["nesterov"] else m
    w = (s["master"] if c["master"] else s["p"]).double()
    for v in s["views"]:
        x = u[v["a"]:v["z"]].view(v["o"], v["i"])
        x = x / torch.linalg.matrix_norm(x)
        wide = v["i"] >= v["o"]
        value, q = torch.linalg.eigh(x @ x.t() if wide else x.t() @ x)
        grown, value = torch.ones_like(value), value.clamp(min=0)
        for k in range(ITERATIONS):
            by = QUINTIC[0] + value * (QUINTIC[1] + value * QUINTIC[2])
            grown, value = grown * by, value * by * by
        p = (q * grown) @ q.t()
        o = p @ x if wide else x @ p
        part = w[v["a"]:v["z"]].view(v["o"], v["i"])
        w[v["a"]:v["z"]] = (part * (1 - s["lr"] * s["wd"]) - s["lr"] * v["scale"] * o).view(-1)
    return {"p": w, "master": w if c["master"] else None, "m": m}
