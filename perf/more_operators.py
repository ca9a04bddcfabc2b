"""Operators of a token model's input side and inner layers, as measurable cases: the lookup of token embeddings with a scale (and the table's gradient), the
layer norm with the residual's addition (and its gradient), and the update that orthogonalises a matrix's momentum by Newton-Schulz products, by itself and as
an optimizer's step over a list of matrices.

listed() names twelve at generic sizes and at this repository's own (ResNet-50's filters as matrices); draw() gives others of the same ranges.  prepare() makes
what a program holds before the call, run() is one pass -- elementary torch operations where `own` is false, the calls of paper_1709_05011_amd where it is
true -- and exact() the same results in 64 bits, written apart.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
LR, MOMENTUM, DECAY, NS_EPS, NS_STEPS = 0.02, 0.95, 0.1, 1e-7, 5
A, B, C = 3.4445, -4.7750, 2.0315             # of the fifth-degree polynomial that a step takes singular values through


def listed():
    return [
        # one token of an answer enters the model: the smallest call, latency
        {"name": "embed_decode", "kind": "embed", "mode": "fwd", "dtype": "bf16", "table": "bf16", "rows": 1, "vocab": 131072, "c": 4096, "pad": 0, "accumulate": False},
        # training in mixed precision: lookup and a gradient of the whole table
        {"name": "embed_train", "kind": "embed", "mode": "train", "dtype": "bf16", "table": "bf16", "rows": 16384, "vocab": 32768, "c": 2048, "pad": 0, "accumulate": False},
        # a ragged batch with padding, odd width and vocabulary, whose table is the classifier's too: its gradient is added to what is there
        {"name": "embed_tied_odd", "kind": "embed", "mode": "train", "dtype": "f32", "table": "f32", "rows": 30011, "vocab": 50021, "c": 1537, "pad": 3, "accumulate": True},
        # one token through the norm: latency
        {"name": "ln_decode", "kind": "ln", "mode": "fwd", "dtype": "bf16", "rows": 1, "c": 4096, "residual": True, "pad": 0},
        # training in mixed precision: forward and backward of a large batch of tokens
        {"name": "ln_bf16_train", "kind": "ln", "mode": "train", "dtype": "bf16", "rows": 8192, "c": 4096, "residual": True, "pad": 0},
        # odd sizes in fp32, no residual, forward and backward
        {"name": "ln_f32_odd", "kind": "ln", "mode": "train", "dtype": "f32", "rows": 1003, "c": 1537, "residual": False, "pad": 0},
        # many narrow rows (heads, small models), forward and backward
        {"name": "ln_narrow", "kind": "ln", "mode": "train", "dtype": "bf16", "rows": 65536, "c": 256, "residual": True, "pad": 0},
        # a small model's matrices: launches
        {"name": "muon_small", "kind": "muon", "list": "layers", "layers": 2, "c": 64, "grad": "f32", "lowp": False, "scaled": False},
        # ResNet-50's 53 filters as matrices of k rows and c*r*s columns, mixed precision
        {"name": "muon_resnet50", "kind": "muon", "list": "resnet50", "layers": 0, "c": 0, "grad": "f32", "lowp": True, "scaled": False},
        # two layers of a token model with bf16 gradients under a clip factor
        {"name": "muon_layers", "kind": "muon", "list": "layers", "layers": 2, "c": 2048, "grad": "bf16", "lowp": True, "scaled": True},
        # three odd wide matrices out of a wider buffer, in mixed precision
        {"name": "ns_odd", "kind": "ns", "dtype": "bf16", "batch": 3, "rows": 517, "cols": 1031, "pad": 5},
        # one large square matrix
        {"name": "ns_large", "kind": "ns", "dtype": "f32", "batch": 1, "rows": 4096, "cols": 4096, "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "ln", "muon", "ns"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "embed":
        c = _log_int(rng, 48, 8192)
        c = c if rng.random() < 0.3 else max(64, c // 64 * 64)
        vocab = min(_log_int(rng, 200, 200000), (1 << 28) // c)
        rows = min(_log_int(rng, 1, 131072), (1 << 26) // c)
        return {"kind": kind, "mode": rng.choice(["fwd", "train", "train"]), "dtype": dtype, "table": rng.choice([dtype, "f32"]), "rows": rows, "vocab": vocab, "c": c,
                "pad": rng.choice([0, 0, 8, 3]), "accumulate": rng.random() < 0.4}
    if kind == "ln":
        c = _log_int(rng, 48, 16384)
        c = c if rng.random() < 0.3 else max(64, c // 64 * 64)
        rows = min(_log_int(rng, 1, 65536), (1 << 25) // c)
        return {"kind": kind, "mode": rng.choice(["fwd", "train"]), "dtype": dtype, "rows": rows, "c": c, "residual": rng.random() < 0.7, "pad": rng.choice([0, 0, 64, 5])}
    if kind == "muon":
        layers, c = _log_int(rng, 1, 8), _log_int(rng, 32, 1536)
        c = c if rng.random() < 0.5 else max(64, c // 64 * 64)
        while layers > 1 and layers * c ** 3 > 2 * 2048 ** 3:
            layers -= 1
        return {"kind": kind, "list": "layers", "layers": layers, "c": c, "grad": dtype, "lowp": rng.random() < 0.5, "scaled": rng.random() < 0.5}
    rows, cols = _log_int(rng, 16, 3000), _log_int(rng, 16, 3000)
    if rng.random() < 0.5:
        rows, cols = max(32, rows // 32 * 32), max(32, cols // 32 * 32)
    return {"kind": kind, "dtype": dtype, "batch": rng.choice([1, 1, 2, 5]), "rows": rows, "cols": cols, "pad": rng.choice([0, 0, 8, 5])}


# ---------------------------------------------------------------------------------------------- inputs

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(std)


def _shapes(case):
    """Rows and columns of a list's matrices."""
    if case["list"] == "resnet50":
        from paper_1709_05011_amd import synth    # plain lists of sizes
        return [(cs.k, cs.weight_numel // cs.k) for cs in synth.resnet50_convs(1)]
    c = case["c"]
    return [s for _ in range(case["layers"]) for s in ((c, c), (c, c), (c, c), (c, c), (4 * c, c), (c, 4 * c))]


def _gradient(g, rows, cols, batch=()):
    """A matrix as gradients are: rows and columns of different sizes, and a few directions that stand out."""
    x = _normal(g, (*batch, rows, cols)) * torch.exp(_normal(g, (*batch, rows, 1), 0.7)) * torch.exp(_normal(g, (*batch, 1, cols), 0.7))
    return x.add_(_normal(g, (*batch, rows, 2)) @ _normal(g, (*batch, 2, cols))).mul_(1e-3)


def _flat(matrices, dtype):
    """One buffer for a list of matrices, as programs keep them, each from a multiple of 64 elements on (zeros between), and its views."""
    whole = torch.zeros(sum(_room(x.numel()) for x in matrices), dtype=dtype, device=DEV)
    views, at = [], 0
    for x in matrices:
        views.append(whole[at:at + x.numel()].view(x.shape))
        views[-1].copy_(x)
        at += _room(x.numel())
    return whole, views


def _room(n):
    return (n + 63) // 64 * 64


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = {"case": dict(case)}
    if kind == "embed":
        rows, vocab, c, t = case["rows"], case["vocab"], case["c"], _type(case["dtype"])
        often = torch.rand(rows, generator=g, device=DEV, dtype=torch.float64)       # a token's frequency falls with its rank, whose tokens lie anywhere
        rank = ((vocab / 2.7 + 1) ** often * 2.7 - 2.7).long().clamp(0, vocab - 1)
        s["tokens"] = torch.randperm(vocab, generator=g, device=DEV)[rank].int()
        if rows > 8:
            s["tokens"][torch.rand(rows, generator=g, device=DEV) < 0.05] = -1         # padding
        s["table"] = _normal(g, (vocab, c + case["pad"]), 0.02).to(_type(case["table"]))[:, :c]
        s["out"] = torch.empty((rows, c), dtype=t, device=DEV)
        if case["mode"] == "train":
            s["dout"] = _normal(g, (rows, c), 1e-2).to(t)
            s["dtable"] = _normal(g, (vocab, c), 1e-2) if case["accumulate"] else torch.empty((vocab, c), device=DEV)
        return s
    if kind == "ln":
        t, rows, c = _type(case["dtype"]), case["rows"], case["c"]
        columns = torch.exp(_normal(g, (c,), 0.7))                        # a stream whose columns differ in size and in mean
        s["x"] = _normal(g, (rows, c + case["pad"])).add_(0.3).to(t)[:, :c]
        s["r"] = (_normal(g, (rows, c), 2.0) * columns + _normal(g, (c,))).to(t) if case["residual"] else None
        s["gamma"], s["beta"] = 1.0 + _normal(g, (c,), 0.2), _normal(g, (c,), 0.1)
        s["h"], s["y"] = torch.empty((rows, c), dtype=t, device=DEV), torch.empty((rows, c), dtype=t, device=DEV)
        s["mean"], s["rstd"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        if case["mode"] == "train":
            s["dy"], s["dh"] = _normal(g, (rows, c), 1e-2).to(t), _normal(g, (rows, c), 1e-2).to(t) if case["residual"] else None
            s["dx"], s["dgamma"], s["dbeta"] = torch.empty((rows, c), dtype=t, device=DEV), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
        return s
    if kind == "ns":
        t = _type(case["dtype"])
        wide = torch.zeros((case["batch"], case["rows"], case["cols"] + case["pad"]), dtype=t, device=DEV)
        s["x"] = wide[:, :, :case["cols"]]
        s["x"].copy_(_gradient(g, case["rows"], case["cols"], (case["batch"],)))
        s["y"] = torch.empty((case["batch"], case["rows"], case["cols"]), dtype=t, device=DEV)
        return s
    shapes = _shapes(case)
    s["all_w"], s["w"] = _flat([_normal(g, n, 0.02) for n in shapes], torch.float32)
    s["all_g"], s["g"] = _flat([_gradient(g, *n) for n in shapes], _type(case["grad"]))
    s["all_m"], s["m"] = _flat([_gradient(g, *n).mul_(4.0) for n in shapes], torch.float32)
    s["all_lowp"], s["lowp"] = _flat(s["w"], torch.bfloat16) if case["lowp"] else (None, None)
    s["scale"] = torch.full((1,), 0.37, device=DEV) if case["scaled"] else None
    s["same"] = {}                                                          # the list's places by shape
    for i, n in enumerate(shapes):
        s["same"].setdefault(n, []).append(i)
    return s


# ------------------------------------------------------------------------------- the operators in plain form

def _embed(s):
    c, t = s["case"], s["tokens"].long()
    there = (t >= 0) & (t < c["vocab"])
    scale = math.sqrt(c["c"])
    rows = s["table"][t.clamp(0, c["vocab"] - 1)].float() * scale
    out = {"out": torch.where(there[:, None], rows, 0.0).to(_type(c["dtype"]))}
    if c["mode"] == "train":
        if not c["accumulate"]:
            s["dtable"].zero_()
        s["dtable"].index_add_(0, t[there], s["dout"][there].float() * scale)
        out["dtable"] = s["dtable"]
    return out


def _ln(s):
    c, x, r = s["case"], s["x"], s["r"]
    h = (x.float() + r.float()).to(x.dtype) if r is not None else x
    hf = h.float()
    mean = hf.mean(1)
    d = hf - mean[:, None]
    rstd = torch.rsqrt((d * d).mean(1) + EPS)
    n = d * rstd[:, None]
    out = {"mean": mean, "rstd": rstd, "y": (n * s["gamma"] + s["beta"]).to(h.dtype)}
    if r is not None:
        out["h"] = h
    if c["mode"] == "train":
        dy = s["dy"].float()
        a = dy * s["gamma"]
        dx = (a - a.mean(1)[:, None] - n * (a * n).mean(1)[:, None]) * rstd[:, None]
        out["dx"] = (dx if s["dh"] is None else dx + s["dh"].float()).to(h.dtype)
        out["dgamma"], out["dbeta"] = (dy * n).sum(0), dy.sum(0)
    return out


def _orthogonal(u):
    """[batch][rows][cols] in fp32 through the Newton-Schulz steps, on the shorter side."""
    x = u / (torch.sqrt((u.double() * u.double()).sum((1, 2))).float() + NS_EPS)[:, None, None]
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    for _ in range(NS_STEPS):
        a = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.bmm(B * a + C * torch.bmm(a, a), x)
    return x.transpose(1, 2) if tall else x


def _ns(s):
    return {"y": _orthogonal(s["x"].float()).to(s["x"].dtype).contiguous()}


def _muon(s):
    for (rows, cols), places in s["same"].items():
        grads = [s["g"][i].float() if s["scale"] is None else s["g"][i].float() * s["scale"] for i in places]
        for i, g in zip(places, grads):
            s["m"][i].mul_(MOMENTUM).add_(g)
        o = _orthogonal(torch.stack([g + MOMENTUM * s["m"][i] for i, g in zip(places, grads)]))
        for j, i in enumerate(places):
            s["w"][i].copy_(s["w"][i] - LR * DECAY * s["w"][i] - LR * math.sqrt(max(1.0, rows / cols)) * o[j])
            if s["lowp"] is not None:
                s["lowp"][i].copy_(s["w"][i])
    return _muon_out(s)


def _muon_out(s):
    out = {"w": s["all_w"], "m": s["all_m"]}
    return out if s["lowp"] is None else out | {"lowp": s["all_lowp"]}


# ------------------------------------------------------------------------------- the framework's calls

def _lc_type(lc, name):
    return lc.LC_BF16 if name == "bf16" else lc.LC_F32


def _own_embed(s):
    from paper_1709_05011_amd import larsconv as lc
    c = s["case"]
    if "desc" not in s:
        s["desc"] = lc.EmbeddingDesc(c["rows"], c["vocab"], c["c"], table_ld=s["table"].stride(0), scale=math.sqrt(c["c"]), table_dtype=_lc_type(lc, c["table"]),
                                     dtype=_lc_type(lc, c["dtype"]))
        if c["mode"] == "train":
            s["ws"] = torch.empty(lc.embedding_bwd_workspace_bytes(s["desc"]), dtype=torch.uint8, device=DEV)
    lc.embedding_fwd(s["desc"], s["table"], s["tokens"], s["out"])
    out = {"out": s["out"]}
    if c["mode"] == "train":
        lc.embedding_bwd(s["desc"], s["tokens"], s["dout"], s["dtable"], s["ws"], accumulate=c["accumulate"])
        out["dtable"] = s["dtable"]
    return out


def _own_ln(s):
    from paper_1709_05011_amd import larsconv as lc
    c = s["case"]
    if "desc" not in s:
        s["desc"] = lc.LayerNormDesc(c["rows"], c["c"], x_ld=s["x"].stride(0), eps=EPS, dtype=_lc_type(lc, c["dtype"]))
        if c["mode"] == "train":
            s["ws"] = torch.empty(lc.layernorm_bwd_workspace_bytes(s["desc"]), dtype=torch.uint8, device=DEV)
    d, h = s["desc"], s["h"] if s["r"] is not None else None
    lc.layernorm_fwd(d, s["x"], s["r"], s["gamma"], s["beta"], h, s["y"], s["mean"], s["rstd"])
    out = {"mean": s["mean"], "rstd": s["rstd"], "y": s["y"]}
    if h is not None:
        out["h"] = h
    if c["mode"] == "train":
        lc.layernorm_bwd(d, s["x"] if h is None else h, s["dy"], s["dh"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"],
                         h_ld=0 if h is not None else s["x"].stride(0))
        out |= {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    return out


def _own_ns(s):
    from paper_1709_05011_amd import larsconv as lc
    c = s["case"]
    if "desc" not in s:
        s["desc"] = lc.NewtonSchulzDesc(c["batch"], c["rows"], c["cols"], ld=s["x"].stride(1), iterations=NS_STEPS, eps=NS_EPS, dtype=_lc_type(lc, c["dtype"]))
        s["ws"] = torch.empty(lc.newton_schulz_workspace_bytes(s["desc"]), dtype=torch.uint8, device=DEV)
    lc.newton_schulz(s["desc"], s["x"], s["y"], s["ws"])
    return {"y": s["y"]}


def _own_muon(s):
    from paper_1709_05011_amd import larsconv as lc
    c = s["case"]
    if "args" not in s:
        s["args"] = lc.MuonArgs(s["w"], s["g"], s["m"], w_lowp=s["lowp"], g_dtype=_lc_type(lc, c["grad"]))
        s["ws"] = torch.empty(lc.muon_workspace_bytes(s["args"]), dtype=torch.uint8, device=DEV)
    lc.muon_step(s["args"], LR, MOMENTUM, DECAY, s["ws"], nesterov=True, iterations=NS_STEPS, eps=NS_EPS, grad_scale=s["scale"])
    return _muon_out(s)


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"embed": _own_embed, "ln": _own_ln, "ns": _own_ns, "muon": _own_muon}[kind](state)
    return {"embed": _embed, "ln": _ln, "ns": _ns, "muon": _muon}[kind](state)


# ---------------------------------------------------------------------------------------------- costs

def _bytes(name):
    return 2 if name == "bf16" else 4


def _ns_flops(rows, cols):
    """Products of symmetric results count their half."""
    m, n = min(rows, cols), max(rows, cols)
    return NS_STEPS * (m * m * n + m * m * m + 2 * m * m * n)


def work(case):
    kind = case["kind"]
    if kind == "embed":
        n, e, rows = case["rows"] * case["c"], _bytes(case["dtype"]), min(case["rows"], case["vocab"])
        b, f = 4 * case["rows"] + rows * case["c"] * _bytes(case["table"]) + n * e, n
        if case["mode"] == "train":                          # a fresh gradient is written whole; one that is added to, where tokens are (an eighth of the rows, about)
            b += 4 * case["rows"] + n * e + (rows * case["c"] if case["accumulate"] else 4 * case["vocab"] * case["c"])
            f += 2 * n
        return {"bytes": b, "flops": f}
    if kind == "ln":
        e, n, rows, c = _bytes(case["dtype"]), case["rows"] * case["c"], case["rows"], case["c"]
        r = 1 if case["residual"] else 0
        b, f = n * e * (2 + 2 * r) + 8 * c + 8 * rows, 8 * n
        if case["mode"] == "train":
            b, f = b + n * e * (3 + r) + 12 * c + 8 * rows, f + 13 * n
        return {"bytes": b, "flops": f}
    if kind == "ns":
        return {"bytes": 2 * _bytes(case["dtype"]) * case["batch"] * case["rows"] * case["cols"], "flops": case["batch"] * _ns_flops(case["rows"], case["cols"])}
    shapes = _shapes(case)
    return {"bytes": (16 + _bytes(case["grad"]) + (2 if case["lowp"] else 0)) * sum(r * c for r, c in shapes), "flops": sum(_ns_flops(*s) for s in shapes)}


# ------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_embed(s):
    c, t, scale = s["case"], s["tokens"].long(), c_root(s["case"])
    out = torch.zeros((c["rows"], c["c"]), dtype=torch.float64, device=DEV)
    at = torch.nonzero((t >= 0) & (t < c["vocab"]))[:, 0]
    out[at] = scale * torch.index_select(s["table"], 0, t[at]).double()
    if c["mode"] != "train":
        return {"out": out}
    sums = s["dtable"].double() if c["accumulate"] else torch.zeros((c["vocab"], c["c"]), dtype=torch.float64, device=DEV)
    order = at[torch.argsort(t[at], stable=True)]
    ids, counts = torch.unique_consecutive(t[order], return_counts=True)
    ends = torch.cumsum(counts, 0)
    for first in range(0, c["c"], 512):                       # a token's sum as the difference of running sums
        run_ = torch.cumsum(s["dout"][order, first:first + 512].double(), 0)
        upto = run_[ends - 1]
        sums[ids, first:first + 512] += scale * (upto - torch.cat([torch.zeros_like(upto[:1]), upto[:-1]]))
    return {"out": out, "dtable": sums}


def c_root(case):
    return float(case["c"]) ** 0.5


def _exact_ln(s):
    c, gamma = s["case"], s["gamma"].double()
    h = s["x"].double()
    out = {}
    if s["r"] is not None:
        out["h"] = h + s["r"].double()
        h = out["h"].float().to(s["x"].dtype).double()                       # the norm is that of the values as stored
    var, mean = torch.var_mean(h, 1, correction=0)
    out["mean"], out["rstd"] = mean, (var + EPS) ** -0.5
    n = (h - mean.unsqueeze(1)) * out["rstd"].unsqueeze(1)
    out["y"] = torch.addcmul(s["beta"].double(), n, gamma)
    if c["mode"] == "train":
        dy = s["dy"].double()
        dn = dy * gamma
        through = dn - dn.sum(1, keepdim=True) / c["c"] - n * (torch.sum(dn * n, 1, keepdim=True) / c["c"])
        out["dx"] = through * out["rstd"].unsqueeze(1) + (0.0 if s["dh"] is None else s["dh"].double())
        out["dgamma"], out["dbeta"] = torch.sum(dy * n, 0), torch.sum(dy, 0)
    return out


def _exact_orthogonal(u):
    """One matrix: aX + A (bX + c A X) with the product of the shorter side."""
    x = u / (torch.linalg.vector_norm(u) + NS_EPS)
    if x.shape[0] > x.shape[1]:
        return _exact_orthogonal(u.T.contiguous()).T
    for _ in range(NS_STEPS):
        a = x @ x.T
        x = A * x + a @ (B * x + C * (a @ x))
    return x


def _exact_ns(s):
    return {"y": torch.stack([_exact_orthogonal(x) for x in s["x"].double()])}


def _exact_muon(s):
    w, m = [], []
    for i in range(len(s["w"])):
        g = s["g"][i].double() * (1.0 if s["scale"] is None else s["scale"].double())
        m.append(MOMENTUM * s["m"][i].double() + g)
        rows, cols = g.shape
        w.append((1.0 - LR * DECAY) * s["w"][i].double() - LR * max(1.0, rows / cols) ** 0.5 * _exact_orthogonal(g + MOMENTUM * m[i]))
    w, m = _flat(w, torch.float64)[0], _flat(m, torch.float64)[0]
    out = {"w": w, "m": m}
    return out if s["lowp"] is None else out | {"lowp": w}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "ln": _exact_ln, "ns": _exact_ns, "muon": _exact_muon}[case["kind"]](s)
