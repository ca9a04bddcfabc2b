"""The operators of a token model's output side, as measurable cases: the RMS norm with the residual's addition (in the storage type or
in 8 bits with scales; with its gradient), the log probabilities of given tokens with entropy and top alternatives (and their gradient),
and the AdamW step over a list of tensors with its states in 32 or in 8 bits.

listed() names twelve at generic sizes and at this repository's own (ResNet-50's parameter list, its classifier); draw() gives others of
the same ranges.  prepare() makes what a program holds before the call, run() is one pass -- elementary torch operations where `own` is
false, the calls of paper_1709_05011_amd where it is true -- and exact() the same results in 64 bits, written apart.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP = 1e-3, 0.9, 0.95, 1e-8, 0.1, 1000
BLOCK = 256                                   # elements of a tensor that share a scale of the 8-bit states
MASKED = float("-inf")


def listed():
    return [
        # one token through the norm in front of an 8-bit product: the smallest call, latency
        {"name": "norm_q8_decode", "kind": "norm", "mode": "q8", "dtype": "bf16", "rows": 1, "c": 4096, "residual": True, "group": 0, "pad": 0},
        # a ragged batch of prompts, a scale for every 128 columns, rows of x out of a wider tensor
        {"name": "norm_q8_prompt", "kind": "norm", "mode": "q8", "dtype": "bf16", "rows": 4099, "c": 5120, "residual": True, "group": 128, "pad": 64},
        # training in mixed precision: forward and backward of a large batch of tokens
        {"name": "norm_bf16_train", "kind": "norm", "mode": "train", "dtype": "bf16", "rows": 8192, "c": 4096, "residual": True, "group": 0, "pad": 0},
        # odd sizes in fp32, no residual, forward and backward
        {"name": "norm_f32_odd", "kind": "norm", "mode": "train", "dtype": "f32", "rows": 1003, "c": 1537, "residual": False, "group": 0, "pad": 0},
        # serving: one row of a large vocabulary with 20 alternatives
        {"name": "token_decode", "kind": "token", "mode": "fwd", "dtype": "bf16", "rows": 1, "vocab": 131072, "top": 20, "pad": 0, "masked": False},
        # a batch of answers with a masked vocabulary of odd size, five alternatives
        {"name": "token_batch_odd", "kind": "token", "mode": "fwd", "dtype": "bf16", "rows": 96, "vocab": 50021, "top": 5, "pad": 27, "masked": True},
        # training in mixed precision: log probabilities, entropy and their gradient over a large vocabulary
        {"name": "token_bf16_train", "kind": "token", "mode": "train", "dtype": "bf16", "rows": 4096, "vocab": 32768, "top": 0, "pad": 0, "masked": False},
        # the classifier of this repository's networks at an ordinary batch, fp32
        {"name": "token_f32_classes", "kind": "token", "mode": "train", "dtype": "f32", "rows": 512, "vocab": 1000, "top": 0, "pad": 0, "masked": False},
        # the smallest list: a small model's tensors, latency
        {"name": "adamw_small", "kind": "adamw", "layers": 2, "c": 64, "q8": False, "grad": "f32", "lowp": False, "scaled": False, "offset": 0},
        # ResNet-50's 161 tensors, fp32 states
        {"name": "adamw_resnet50", "kind": "adamw", "layers": 0, "c": 0, "q8": False, "grad": "f32", "lowp": True, "scaled": False, "offset": 0},
        # mixed precision, 8-bit states, bf16 gradients under a clip factor, the largest list
        {"name": "adamw_q8_large", "kind": "adamw", "layers": 4, "c": 2048, "q8": True, "grad": "bf16", "lowp": True, "scaled": True, "offset": 0},
        # odd tensors off a 16-byte boundary, 8-bit states
        {"name": "adamw_q8_odd", "kind": "adamw", "layers": 6, "c": 517, "q8": True, "grad": "f32", "lowp": False, "scaled": True, "offset": 1},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "token", "adamw"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "norm":
        c = _log_int(rng, 64, 16384)
        c = c if rng.random() < 0.3 else max(64, c // 64 * 64)
        rows = min(_log_int(rng, 1, 16384), (1 << 25) // c)
        mode = rng.choice(["fwd", "q8", "train"])
        return {"kind": kind, "mode": mode, "dtype": dtype, "rows": rows, "c": c, "residual": rng.random() < 0.7,
                "group": rng.choice([0, 128]) if mode == "q8" else 0, "pad": rng.choice([0, 0, 64, 5])}
    if kind == "token":
        vocab = _log_int(rng, 100, 200000)
        vocab = vocab if rng.random() < 0.5 else max(128, vocab // 128 * 128)
        rows = min(_log_int(rng, 1, 8192), (1 << 27) // vocab)
        mode = rng.choice(["fwd", "fwd", "train"])
        return {"kind": kind, "mode": mode, "dtype": dtype, "rows": rows, "vocab": vocab,
                "top": rng.choice([0, 1, 5, 20, 32]) if mode == "fwd" else 0, "pad": rng.choice([0, 0, 8, 27]), "masked": rng.random() < 0.3}
    layers, c = _log_int(rng, 1, 24), _log_int(rng, 33, 2048)
    c = c if rng.random() < 0.5 else max(64, c // 64 * 64)
    while layers > 1 and 12 * layers * c * c > 2e8:
        layers -= 1
    return {"kind": kind, "layers": layers, "c": c, "q8": rng.random() < 0.5, "grad": dtype, "lowp": rng.random() < 0.5,
            "scaled": rng.random() < 0.5, "offset": rng.choice([0, 0, 0, 1])}


# ---------------------------------------------------------------------------------------------- inputs

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(std)


def _sizes(case):
    if not case["layers"]:
        from paper_1709_05011_amd import synth    # plain lists of sizes
        return synth.resnet50_param_numels()
    c = case["c"]
    return [m for _ in range(case["layers"]) for m in (c, c * c, c * c, c * c, c * c, c, 4 * c * c, 4 * c * c)]


def _flat(sizes, dtype, offset):
    """One buffer for a list of tensors, as programs keep them, each from a multiple of 256 elements on (zeros between), all of them
    `offset` elements past an aligned address; and its views."""
    whole = torch.zeros(sum((m + BLOCK - 1) // BLOCK * BLOCK for m in sizes) + offset, dtype=dtype, device=DEV)[offset:]
    return whole, _views(whole, sizes)


def _views(whole, sizes, per=1):
    views, at = [], 0
    for m in sizes:
        n = (m + BLOCK - 1) // BLOCK * BLOCK
        views.append(whole[at // per:(at + (m if per == 1 else n)) // per])
        at += n
    return views


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "norm":
        t, rows, c = _type(case["dtype"]), case["rows"], case["c"]
        columns = torch.exp(_normal(g, (c,), 0.7))                        # a stream whose columns differ in size, as residual streams do
        wide = (_normal(g, (rows, c + case["pad"]))).to(t)
        s = {"case": dict(case), "x": wide[:, :c], "r": (_normal(g, (rows, c), 2.0) * columns).to(t) if case["residual"] else None,
             "gamma": 1.0 + _normal(g, (c,), 0.2), "h": torch.empty((rows, c), dtype=t, device=DEV), "rstd": torch.empty(rows, device=DEV)}
        if case["mode"] == "q8":
            s["y"] = torch.empty((rows, c), dtype=torch.uint8, device=DEV)
            s["scale"] = torch.empty((rows, -(-c // case["group"]) if case["group"] else 1), device=DEV)
        else:
            s["y"] = torch.empty((rows, c), dtype=t, device=DEV)
        if case["mode"] == "train":
            s["dy"], s["dh"] = _normal(g, (rows, c), 1e-2).to(t), _normal(g, (rows, c), 1e-2).to(t) if case["residual"] else None
            s["dx"], s["dgamma"] = torch.empty((rows, c), dtype=t, device=DEV), torch.empty(c, device=DEV)
        return s
    if kind == "token":
        t, rows, k = _type(case["dtype"]), case["rows"], case["vocab"]
        z = _normal(g, (rows, k + case["pad"]), 2.0)
        tokens = torch.randint(0, k, (rows,), generator=g, device=DEV, dtype=torch.int32)
        near = torch.rand(rows, generator=g, device=DEV) < 0.6              # rows whose token the model finds likely
        z[near, tokens[near].long()] += 9.0
        if case["masked"]:                                                  # tokens that the grammar forbids; a row that forbids all
            z.masked_fill_(torch.rand(k + case["pad"], generator=g, device=DEV) < 0.3, MASKED)
            if rows > 4:
                z[3] = MASKED
        if rows > 8:
            tokens[5] = -1                                                  # a position that does not count
        s = {"case": dict(case), "z": z.to(t)[:, :k], "tokens": tokens, "lp": torch.empty(rows, device=DEV), "ent": torch.empty(rows, device=DEV),
             "lse": torch.empty(rows, device=DEV)}
        if case["top"]:
            s["top_ids"] = torch.empty((rows, case["top"]), dtype=torch.int32, device=DEV)
            s["top_lp"] = torch.empty((rows, case["top"]), device=DEV)
        if case["mode"] == "train":
            s["dlp"], s["dent"] = _normal(g, (rows,), 1.0 / rows) - 1.0 / rows, torch.full((rows,), -0.01 / rows, device=DEV)
            s["dz"] = torch.empty((rows, k), dtype=t, device=DEV)
        return s
    sizes, q8, off = _sizes(case), case["q8"], case["offset"]
    s = {"case": dict(case), "sizes": sizes, "t": STEP, "scale": torch.full((1,), 0.37, device=DEV) if case["scaled"] else None}
    live, views = _flat(sizes, torch.float32, 0)
    for v in views:
        v.fill_(1.0)
    n = live.numel()
    std = torch.exp(_normal(g, (n // BLOCK,), 1.5)).repeat_interleave(BLOCK) * 1e-3        # layers' gradients differ in size
    s["w"], s["w_views"] = _flat(sizes, torch.float32, off)
    s["g"], s["g_views"] = _flat(sizes, _type(case["grad"]), off)
    s["w"].copy_(_normal(g, (n,), 0.02).mul_(live))
    s["g"].copy_(_normal(g, (n,)).mul_(std).mul_(live))
    m, v = _normal(g, (n,), 0.3).mul_(std).mul_(live), _normal(g, (n,), 0.7).exp_().mul_(std).mul_(std).mul_(live)
    if q8:
        for key, x, t, most in (("m", m, torch.float8_e4m3fn, 448.0), ("v", v, torch.float8_e5m2, 57344.0)):
            scale = _power_scale(x.view(-1, BLOCK).abs().amax(1), most)
            s[key] = (x.view(-1, BLOCK) / scale[:, None]).to(t).view(-1).view(torch.uint8)
            s[key + "_views"], s[key + "_scale"], s[key + "_scale_views"] = _views(s[key], sizes), scale, _views(scale, sizes, BLOCK)
    else:
        (s["m"], s["m_views"]), (s["v"], s["v_views"]) = _flat(sizes, torch.float32, off), _flat(sizes, torch.float32, off)
        s["m"].copy_(m)
        s["v"].copy_(v)
    s["lowp"], s["lowp_views"] = _flat(sizes, torch.bfloat16, off) if case["lowp"] else (None, None)
    if q8:                                                                  # each element's number in its tensor, for the dither
        s["index"] = torch.cat([torch.arange((m + BLOCK - 1) // BLOCK * BLOCK, device=DEV, dtype=torch.int32) for m in sizes])
    return s


# ------------------------------------------------------------------------------- the operators in plain form

def _power_scale(amax, most):
    """The smallest power of two s, 2^-126 at least, with amax / s <= most; 1 where amax is 0."""
    f, e = torch.frexp(amax / most)
    return torch.where(amax > 0, ((torch.where(f == 0.5, e - 1, e).clamp(min=-126) + 127) << 23).view(torch.float32), 1.0)


def _norm_fwd(s):
    c, x, r = s["case"], s["x"], s["r"]
    h = (x.float() + r.float()).to(x.dtype) if r is not None else x
    hf = h.float()
    rstd = torch.rsqrt((hf * hf).mean(1) + EPS)
    return h, hf, rstd, hf * rstd[:, None] * s["gamma"]


def _norm(s):
    c = s["case"]
    h, hf, rstd, y = _norm_fwd(s)
    out = {"rstd": rstd}
    if s["r"] is not None:
        out["h"] = h
    if c["mode"] == "q8":
        rows, group = c["rows"], c["group"] or c["c"]
        groups = -(-c["c"] // group)
        padded = torch.nn.functional.pad(y, (0, groups * group - c["c"])).view(rows, groups, group)
        scale = (padded.abs().amax(2) / 448.0).clamp(min=2.0 ** -126)
        q = (padded / scale[:, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(rows, -1)
        return out | {"y": q[:, :c["c"]].contiguous(), "scale": scale}
    out["y"] = y.to(h.dtype)
    if c["mode"] == "train":
        dy, xh = s["dy"].float(), hf * rstd[:, None]
        a = dy * s["gamma"]
        dx = (a - xh * (a * xh).mean(1)[:, None]) * rstd[:, None]
        out["dx"] = (dx if s["dh"] is None else dx + s["dh"].float()).to(h.dtype)
        out["dgamma"] = (dy * xh).sum(0)
    return out


def _token(s):
    c, z = s["case"], s["z"].float()
    rows, k = z.shape
    t = s["tokens"].long()
    most = z.amax(1)
    empty = torch.isinf(most)                                               # nothing is allowed in this row
    d = z - torch.where(empty, 0.0, most)[:, None]
    e = torch.exp(d)
    total = e.sum(1)
    lse = torch.where(empty, most, most + torch.log(total))
    counts = (t >= 0) & (t < k)
    at = d.gather(1, t.clamp(0, k - 1)[:, None])[:, 0] - torch.log(total)
    lp = torch.where(counts, torch.where(empty, MASKED, at), 0.0)
    ent = torch.where(empty, 0.0, torch.log(total) - (torch.where(e > 0, d, 0.0) * e).sum(1) / total)
    out = {"lp": lp, "ent": ent, "lse": lse}
    if c["top"]:
        bits = (z + 0.0).view(torch.int32).long()                           # (the two zeros are one value)
        key = (torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits) << 32) + (k - 1 - torch.arange(k, device=DEV))
        n = min(c["top"], k)
        ids = k - 1 - (key.topk(n, 1).values & 0xFFFFFFFF)
        there = z.gather(1, ids) > MASKED
        top_lp = torch.where(there, d.gather(1, ids) - torch.log(total)[:, None], MASKED)
        out["top_ids"] = torch.nn.functional.pad(torch.where(there, ids, -1).int(), (0, c["top"] - n), value=-1)
        out["top_lp"] = torch.nn.functional.pad(top_lp, (0, c["top"] - n), value=MASKED)
    if c["mode"] == "train":
        p = e / total[:, None]
        logp = torch.where(p > 0, d - torch.log(total)[:, None], 0.0)
        glp, gent = torch.where(counts & ~empty, s["dlp"], 0.0), torch.where(empty, 0.0, s["dent"])
        dz = -p * (glp[:, None] + gent[:, None] * (logp + ent[:, None]))
        dz.scatter_add_(1, t.clamp(0, k - 1)[:, None], glp[:, None])
        out["dz"] = torch.where(empty[:, None], 0.0, dz).to(s["z"].dtype)
    return out


def _dither(index, seed):
    """21 bits for each element from its number and the call's seed: two rounds of shift and product, modulo 2^32 in 32-bit integers."""
    x = index + _signed(seed * 0x9E3779B1 + 0x7F4A7C15)
    x = (x ^ ((x >> 16) & 0xFFFF)) * _signed(0x9E3779B1)
    x = (x ^ ((x >> 15) & 0x1FFFF)) * _signed(0x6A09E667)
    return (x >> 11) & 0x1FFFFF


def _signed(v):
    v &= 0xFFFFFFFF
    return v - (1 << 32) if v >= 1 << 31 else v


def _e5m2_dithered(x, r):
    """Codes of x in [0, 57344] with the bits r added below the last place before what follows it is dropped; what is not zero takes code 1 at least."""
    bits = x.view(torch.int32)
    normal = ((bits + r) >> 21) - (112 << 2)
    small = ((x * 2.0 ** 37).clamp(max=2.0 ** 24).int() + r) >> 21
    code = torch.where(x < 2.0 ** -14, small, normal)
    return torch.where(x > 0, code.clamp(min=1), 0).to(torch.uint8)


def _adamw(s):
    c = s["case"]
    s["t"] += 1
    w, g = s["w"], s["g"].float()
    if s["scale"] is not None:
        g = g * s["scale"]
    if c["q8"]:
        m = (s["m"].view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].view(torch.float8_e5m2).float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
    else:
        m, v = s["m"], s["v"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    root = torch.sqrt(v) / math.sqrt(1 - BETA2 ** s["t"]) + ADAM_EPS
    w.copy_(w - LR * DECAY * w - (LR / (1 - BETA1 ** s["t"])) * (m / root))
    if c["q8"]:
        s["m_scale"].copy_(_power_scale(m.view(-1, BLOCK).abs().amax(1), 448.0))
        s["v_scale"].copy_(_power_scale(v.view(-1, BLOCK).amax(1), 57344.0))
        s["m"].copy_((m.view(-1, BLOCK) / s["m_scale"][:, None]).to(torch.float8_e4m3fn).view(-1).view(torch.uint8))
        s["v"].copy_(_e5m2_dithered((v.view(-1, BLOCK) / s["v_scale"][:, None]).view(-1), _dither(s["index"], s["t"])))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if s["lowp"] is not None:
        s["lowp"].copy_(w)
    return _adamw_out(s)


def _adamw_out(s):
    out = {"w": s["w"]}
    if s["case"]["q8"]:
        out |= {"m": s["m"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e5m2), "m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    else:
        out |= {"m": s["m"], "v": s["v"]}
    return out if s["lowp"] is None else out | {"lowp": s["lowp"]}


# ------------------------------------------------------------------------------- the framework's calls

def _own_norm(s):
    from paper_1709_05011_amd import larsconv as lc
    c = s["case"]
    if "desc" not in s:
        s["desc"] = lc.RmsNormDesc(c["rows"], c["c"], x_ld=s["x"].stride(0), eps=EPS, dtype=lc.LC_BF16 if c["dtype"] == "bf16" else lc.LC_F32)
        if c["mode"] == "train":
            s["ws"] = torch.empty(lc.rmsnorm_bwd_workspace_bytes(s["desc"]), dtype=torch.uint8, device=DEV)
    d, h = s["desc"], s["h"] if s["r"] is not None else None
    out = {"rstd": s["rstd"]}
    if h is not None:
        out["h"] = h
    if c["mode"] == "q8":
        lc.rmsnorm_fwd_q8(d, s["x"], s["r"], s["gamma"], h, s["y"], s["scale"], c["group"], s["rstd"])
        return out | {"y": s["y"].view(torch.float8_e4m3fn), "scale": s["scale"]}
    lc.rmsnorm_fwd(d, s["x"], s["r"], s["gamma"], h, s["y"], s["rstd"])
    out["y"] = s["y"]
    if c["mode"] == "train":
        lc.rmsnorm_bwd(d, s["x"] if h is None else h, s["dy"], s["dh"], s["gamma"], s["rstd"], s["dx"], s["dgamma"], s["ws"],
                       h_ld=0 if h is not None else s["x"].stride(0))
        out |= {"dx": s["dx"], "dgamma": s["dgamma"]}
    return out


def _own_token(s):
    from paper_1709_05011_amd import larsconv as lc
    c = s["case"]
    if "desc" not in s:
        s["desc"] = lc.TokenDesc(c["rows"], c["vocab"], ld=s["z"].stride(0), dtype=lc.LC_BF16 if c["dtype"] == "bf16" else lc.LC_F32, top=c["top"])
        nb = lc.token_logprob_workspace_bytes(s["desc"])
        s["ws"] = torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None
    d = s["desc"]
    lc.token_logprob_fwd(d, s["z"], s["tokens"], s["lp"], s["ent"], s["lse"], s.get("top_ids"), s.get("top_lp"), s["ws"])
    out = {"lp": s["lp"], "ent": s["ent"], "lse": s["lse"]}
    if c["top"]:
        out |= {"top_ids": s["top_ids"], "top_lp": s["top_lp"]}
    if c["mode"] == "train":
        lc.token_logprob_bwd(d, s["z"], s["tokens"], s["lse"], s["ent"], s["dlp"], s["dent"], s["dz"])
        out["dz"] = s["dz"]
    return out


def _own_adamw(s):
    from paper_1709_05011_amd import larsconv as lc
    c = s["case"]
    s["t"] += 1
    if "args" not in s:
        more = dict(w_lowp=s["lowp_views"], g_dtype=lc.LC_BF16 if c["grad"] == "bf16" else lc.LC_F32)
        if c["q8"]:
            s["args"] = lc.AdamWQ8Args(s["w_views"], s["g_views"], s["m_views"], s["m_scale_views"], s["v_views"], s["v_scale_views"], **more)
        else:
            s["args"] = lc.AdamWArgs(s["w_views"], s["g_views"], s["m_views"], s["v_views"], **more)
    if c["q8"]:
        lc.adamw_step_q8(s["args"], LR, BETA1, BETA2, ADAM_EPS, DECAY, s["t"], seed=s["t"], grad_scale=s["scale"])
    else:
        lc.adamw_step(s["args"], LR, BETA1, BETA2, ADAM_EPS, DECAY, s["t"], grad_scale=s["scale"])
    return _adamw_out(s)


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "token": _own_token, "adamw": _own_adamw}[kind](state)
    return {"norm": _norm, "token": _token, "adamw": _adamw}[kind](state)


# ---------------------------------------------------------------------------------------------- costs

def work(case):
    if case["kind"] == "norm":
        e, n, rows, c = (2 if case["dtype"] == "bf16" else 4), case["rows"] * case["c"], case["rows"], case["c"]
        r = 1 if case["residual"] else 0
        groups = -(-c // case["group"]) if case["group"] else 1
        out = n + 4 * rows * groups if case["mode"] == "q8" else n * e
        b = n * e * (1 + 2 * r) + out + 4 * c + 4 * rows
        f = 6 * n
        if case["mode"] == "train":
            b += n * e * (3 + r) + 8 * c + 4 * rows
            f += 10 * n
        return {"bytes": b, "flops": f}
    if case["kind"] == "token":
        e, n = (2 if case["dtype"] == "bf16" else 4), case["rows"] * case["vocab"]
        b, f = n * e + case["rows"] * (16 + 8 * case["top"]), 6 * n
        if case["mode"] == "train":
            b, f = b + 2 * n * e + case["rows"] * 20, f + 8 * n
        return {"bytes": b, "flops": f}
    n = sum(_sizes(case))
    b = 8 + (2 if case["grad"] == "bf16" else 4) + (2 if case["lowp"] else 0) + (4 + 16 / BLOCK if case["q8"] else 16)
    return {"bytes": b * n, "flops": 14 * n}


# ------------------------------------------------------------------------------- the definitions in 64 bits

def _nearest(x, mantissa, least):
    """x on the grid of `mantissa` bits, spaced as at 2^least below that: to nearest, ties to even."""
    e = (torch.frexp(x).exponent - 1).clamp(min=least).double()
    step = torch.exp2(e - mantissa)
    return torch.round(x / step) * step


def _exact_norm(s):
    c, gamma = s["case"], s["gamma"].double()
    h = s["x"].double()
    out = {}
    if s["r"] is not None:
        out["h"] = h + s["r"].double()
        h = out["h"].float().to(s["x"].dtype).double()                       # the norm is that of the values as stored
    rstd = 1.0 / torch.sqrt(torch.sum(h ** 2, 1) / c["c"] + EPS)
    n = h * rstd.unsqueeze(1)
    y = n * gamma
    out["rstd"] = rstd
    if c["mode"] == "q8":
        columns = list(range(0, c["c"], c["group"] or c["c"]))
        width = c["group"] or c["c"]
        scale = torch.stack([y[:, i:i + width].abs().amax(1) for i in columns], 1) / 448.0
        out["scale"] = scale
        out["y"] = torch.cat([_nearest(y[:, i:i + width] / scale[:, j:j + 1], 3, -6) for j, i in enumerate(columns)], 1)
        return out
    out["y"] = y
    if c["mode"] == "train":
        dn = s["dy"].double() * gamma
        through = dn - n * (torch.sum(dn * n, 1, keepdim=True) / c["c"])
        out["dx"] = through * rstd.unsqueeze(1) + (0.0 if s["dh"] is None else s["dh"].double())
        out["dgamma"] = torch.sum(s["dy"].double() * n, 0)
    return out


def _exact_token(s):
    c, parts = s["case"], []
    for at in range(0, c["rows"], 512):
        z, t = s["z"][at:at + 512].double(), s["tokens"][at:at + 512].long()
        lse = torch.logsumexp(z, 1)
        empty = lse == MASKED
        logp = z - torch.where(empty, 0.0, lse)[:, None]
        p = torch.exp(logp)
        finite = torch.where(p > 0, logp, 0.0)
        ent = -torch.sum(p * finite, 1)
        got = torch.take_along_dim(logp, t.clamp(min=0)[:, None], 1)[:, 0]
        part = {"lp": torch.where(t >= 0, got, 0.0), "ent": ent, "lse": lse}
        if c["top"]:
            order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :c["top"]]
            top = torch.take_along_dim(logp, order, 1)
            part["top_lp"] = torch.cat([top, torch.full((top.shape[0], c["top"] - top.shape[1]), MASKED, dtype=top.dtype, device=DEV)], 1)
        if c["mode"] == "train":
            a, b = s["dlp"][at:at + 512].double() * (t >= 0) * ~empty, s["dent"][at:at + 512].double()
            hot = torch.zeros_like(z)
            hot[torch.arange(len(t), device=DEV), t.clamp(min=0)] = 1.0
            part["dz"] = a[:, None] * (hot - p) + b[:, None] * (-p * (finite + ent[:, None]))
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return out | {"top_ids": None} if c["top"] else out


def _exact_adamw(s):
    c, t = s["case"], s["t"] + 1
    g = s["g"].double() * (1.0 if s["scale"] is None else s["scale"].double())
    if c["q8"]:
        m = s["m"].view(torch.float8_e4m3fn).double() * s["m_scale"].double().repeat_interleave(BLOCK)
        v = s["v"].view(torch.float8_e5m2).double() * s["v_scale"].double().repeat_interleave(BLOCK)
    else:
        m, v = s["m"].double(), s["v"].double()
    m += (1 - BETA1) * (g - m)
    v += (1 - BETA2) * (g ** 2 - v)
    w = s["w"].double()
    w = w * (1 - LR * DECAY) - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
    out = {"w": w}
    if c["lowp"]:
        out["lowp"] = w
    if not c["q8"]:
        return out | {"m": m, "v": v}
    for key, x, most in (("m", m, 448.0), ("v", v, 57344.0)):
        scale = torch.exp2(torch.ceil(torch.log2(x.view(-1, BLOCK).abs().amax(1) / most)).clamp(min=-126))
        live = x.view(-1, BLOCK).abs().amax(1) > 0
        out[key + "_scale"] = torch.where(live, scale, 1.0)
        x = x / out[key + "_scale"].repeat_interleave(BLOCK)
        if key == "m":
            out[key] = _nearest(x, 3, -6)
        else:
            u = (s["index"].long() + t * 0x9E3779B1 + 0x7F4A7C15) & 0xFFFFFFFF
            u = ((u ^ (u >> 16)) * 0x9E3779B1) & 0xFFFFFFFF
            u = ((u ^ (u >> 15)) * 0x6A09E667) & 0xFFFFFFFF
            step = torch.exp2((torch.frexp(x).exponent - 1).clamp(min=-14).double() - 2)
            q = torch.floor(x / step + (u >> 11).double() * 2.0 ** -21) * step
            out[key] = torch.where(x > 0, q.clamp(min=2.0 ** -16), 0.0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "token": _exact_token, "adamw": _exact_adamw}[case["kind"]](s)
