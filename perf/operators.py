"""The operators around the vocabulary layers, as cases that can be measured: the norms before and after a block with its
gate and residual scale (forward and backward), and the global gradient norm over many tensors with clipping.

``run`` computes a case in its plain form, elementary torch operations in 32 bits rounded once at the end, or, where ``own``
is true, through the framework's entry points.  ``exact`` gives the same outputs from the definitions in 64 bits.

With m the mean of a row (0 without ``center``) and rho = 1 / sqrt(mean((v - m)^2) + eps):

    u = (y - m1) rho1 w_post + b_post   (with ``post``; else u = y)
    r = x + scale * gate * u            (gate [G, h]: each of its rows serves N / G consecutive tokens)
    H = (r - m2) rho2 w + b

and for gradients g of a list of tensors: norm = sqrt(sum g^2), clipped = g * max_norm / norm where norm exceeds max_norm.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-5


def _norm(name, op, N, h, dtype, post, center, gate, bias, grad_in="f32"):
    # gate: rows of the gate (0: none); grad_in: type of the gradient that comes in (the output layer's dH is fp32)
    return {"name": name, "op": op, "N": N, "h": h, "dtype": dtype, "post": post, "center": center, "gate": gate,
            "bias": bias, "grad_in": grad_in, "scale": 0.5 if gate else 1.0}


def _shards(name, op, p, rows, h, max_norm=1.0):
    # the fp32 gradients of p shards of the vocabulary, of equal size
    return {"name": name, "op": op, "layout": "shards", "p": p, "rows": rows, "h": h, "max_norm": max_norm}


def _model(name, op, n, most, bf16_every, max_norm=1.0):
    # n tensors of a model, of 0 to `most` elements, every bf16_every-th of them bf16 (0: none)
    return {"name": name, "op": op, "layout": "model", "n": n, "most": most, "bf16_every": bf16_every, "max_norm": max_norm}


def listed():
    return [
        # one new token of a model with norms on both sides of a block, before the output layer: latency
        _norm("norm_token", "norm_fwd", 1, 4096, "bf16", True, False, 0, False),
        # the tokens of the Llama-like and the large-vocabulary configuration
        _norm("norm_seq", "norm_fwd", 4096, 4096, "bf16", True, False, 0, False),
        # a model in full precision, sizes that are no multiple of anything, layer norms with biases, a gate per channel
        _norm("norm_f32_odd", "norm_fwd", 509, 1001, "f32", True, True, 1, True),
        # the wide model of the very-large-vocabulary configuration, an element-wise gate
        _norm("norm_wide_gated", "norm_fwd", 4096, 8192, "bf16", False, False, 4096, False),
        # the tiny fp32 configuration: launches and latency
        _norm("norm_bwd_tiny", "norm_bwd", 128, 256, "f32", True, False, 0, False),
        # the tokens of the Llama-like configuration, behind the output layer's fp32 dH
        _norm("norm_bwd_seq", "norm_bwd", 4096, 4096, "bf16", True, False, 0, False),
        # 17 sequences with a gate each, layer norms with biases, inside a model (gradients in bf16)
        _norm("norm_bwd_ragged", "norm_bwd", 17 * 59, 2050, "bf16", True, True, 17, True, grad_in="bf16"),
        # norm over the gradients of the Llama-like configuration's eight shards
        _shards("grad_norm_shards", "grad_norm", 8, 4000, 4096),
        # norm over the tensors of a small model held in bf16 throughout
        _model("grad_norm_bf16", "grad_norm", 60, 2000003, 1),
        # clipping of the tiny configuration's two shards
        _shards("clip_tiny", "clip", 2, 4096, 256),
        # the tensors of a model of mixed types, clipped into the buckets that go to the other devices
        _model("clip_buckets", "clip", 150, 1000003, 3),
        # the gradients of the large-vocabulary configuration's eight shards
        _shards("clip_large", "clip", 8, 16032, 4096),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "norm_fwd", "norm_bwd", "grad_norm", "clip"])
    if op.startswith("norm"):
        h = _log(rng, 64, 16384)
        h = h if rng.random() < 0.4 else (h + 63) // 64 * 64
        most = min(8192, 4096 * 8192 // h)
        N = 1 if op == "norm_fwd" and rng.random() < 0.15 else _log(rng, 2, most)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        gate = rng.choice([0, 1, N, -1])
        if gate < 0:      # a gate per sequence: of all numbers of sequences that split the tokens evenly
            gate = rng.choice([g for g in range(1, min(N, 64) + 1) if N % g == 0])
        case = _norm("", op, N, h, dtype, rng.random() < 0.6, rng.random() < 0.4, gate, rng.random() < 0.4,
                     rng.choice(["f32", dtype]))
    elif rng.random() < 0.4:
        h = _log(rng, 64, 8192)
        p = rng.choice([1, 2, 4, 8, 16])
        case = _shards("", op, p, _log(rng, 16, max(17, 200000000 // (p * h))), h, rng.choice([1.0, 0.1, 1e6]))
    else:
        most = _log(rng, 1000, 4000000)
        case = _model("", op, _log(rng, 2, 400), most, rng.choice([0, 1, 2, 3, 7]), rng.choice([1.0, 0.1, 1e6]))
    del case["name"]
    return case


def _counts(case):
    """(elements, type) of every gradient of a case."""
    if case["layout"] == "shards":
        return [(case["rows"] * case["h"], "f32")] * case["p"]
    every, most = case["bf16_every"], case["most"]
    # sizes spread over their logarithm, one tensor of fifty without elements
    return [(0 if k % 50 == 49 else int(most ** ((k * 0.6180339887) % 1.0)), "bf16" if every and k % every == every - 1 else "f32")
            for k in range(case["n"])]


def _norm_inputs(case, seed):
    N, h, G, dt = case["N"], case["h"], case["gate"], DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std + mean

    # channels of a residual stream differ in size, some by a lot, and its rows have a mean
    spread = torch.exp(normal(h, std=0.7))
    s = {"x": (normal(N, h, mean=0.2) * spread).to(dt), "y": normal(N, h, std=0.5, mean=-0.1).to(dt)}
    s["gate"] = normal(G, h, std=0.5, mean=0.3).to(dt) if G else None
    s["w"] = normal(h, std=0.1, mean=1.0).to(dt)
    s["b"] = normal(h, std=0.1).to(dt) if case["bias"] else None
    s["w_post"] = normal(h, std=0.1, mean=1.0).to(dt) if case["post"] else None
    s["b_post"] = normal(h, std=0.1).to(dt) if case["bias"] and case["post"] else None
    if case["op"] == "norm_bwd":
        # what the forward pass kept: the sum that was normalised (in place of x) and its statistics
        r, _, stats = _plain_norm_fwd(case, s)
        s["r"], s["stats"] = r, stats
        del s["x"]
        s["dH"] = normal(N, h, std=1e-4).to(DTYPES[case["grad_in"]])
        s["dr"] = normal(N, h, std=1e-4).to(dt)
    return s


def _grad_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    # gradients of different parameters differ in size
    return [torch.randn(n, generator=gen, device="cuda").mul_(10.0 ** (-3 + k % 5 * 0.25)).to(DTYPES[t])
            for k, (n, t) in enumerate(_counts(case))]


def prepare(case, seed):
    s = {"case": case}
    if case["op"] == "norm_fwd":
        s.update(_norm_inputs(case, seed))
        s["out"] = {"r": torch.empty_like(s["x"]), "H": torch.empty_like(s["x"]),
                    "stats": torch.empty(4, case["N"], device="cuda")}
    elif case["op"] == "norm_bwd":
        s.update(_norm_inputs(case, seed))

        def vector(t, *shape):
            return None if t is None else torch.empty(*(shape or (case["h"],)), device="cuda")
        s["out"] = {"dx": torch.empty_like(s["dr"]), "dy": torch.empty_like(s["dr"]),
                    "dgate": vector(s["gate"], case["gate"], case["h"]), "dw": vector(s["w"]), "db": vector(s["b"]),
                    "dw_post": vector(s["w_post"]), "db_post": vector(s["b_post"])}
    else:
        s["grads"] = _grad_inputs(case, seed)
        if case["op"] == "clip":
            s["outs"], s["whole"] = _buckets(s["grads"], case["layout"])
    return s


def _buckets(grads, layout):
    """Where the clipped gradients go: tensors of their own, or views of one flat buffer per type."""
    if layout == "shards":
        outs = [torch.empty_like(g) for g in grads]
        return outs, outs
    flat = {t: torch.empty(sum(g.numel() for g in grads if g.dtype == t), dtype=t, device="cuda")
            for t in DTYPES.values()}
    at, outs = dict.fromkeys(flat, 0), []
    for g in grads:
        outs.append(flat[g.dtype][at[g.dtype]:at[g.dtype] + g.numel()])
        at[g.dtype] += g.numel()
    return outs, [f for f in flat.values() if f.numel()]


# ----------------------------------------------------------------------------------------------- plain forms
def _plain_normed(v, center):
    m = v.mean(1, keepdim=True) if center else torch.zeros_like(v[:, :1])
    rho = 1 / torch.sqrt(((v - m) * (v - m)).mean(1, keepdim=True) + EPS)
    return (v - m) * rho, m, rho


def _plain_affine(v, w, b):
    v = v if w is None else v * w.float()
    return v if b is None else v + b.float()


def _plain_spread(gate, N):
    """The gate's row of every token."""
    return 1.0 if gate is None else gate.float().repeat_interleave(N // gate.shape[0], 0)


def _plain_norm_fwd(case, s):
    x, u = s["x"].float(), s["y"].float()
    m1, rho1 = torch.zeros_like(x[:, :1]), torch.ones_like(x[:, :1])
    if case["post"]:
        u, m1, rho1 = _plain_normed(u, case["center"])
        u = _plain_affine(u, s["w_post"], s["b_post"])
    r = x + case["scale"] * _plain_spread(s["gate"], case["N"]) * u
    H, m2, rho2 = _plain_normed(r, case["center"])
    H = _plain_affine(H, s["w"], s["b"])
    return r.to(s["x"].dtype), H.to(s["x"].dtype), torch.cat([m1, rho1, m2, rho2], 1).t().contiguous()


def _plain_back(a, vh, rho, center):
    a = a - a.mean(1, keepdim=True) - vh * (a * vh).mean(1, keepdim=True) if center else a - vh * (a * vh).mean(1, keepdim=True)
    return rho * a


def _plain_norm_bwd(case, s):
    N, h, G = case["N"], case["h"], case["gate"]
    m1, rho1, m2, rho2 = s["stats"].reshape(4, N, 1)
    dH, gate = s["dH"].float(), _plain_spread(s["gate"], N)
    rh, yh = (s["r"].float() - m2) * rho2, (s["y"].float() - m1) * rho1
    g = s["dr"].float() + _plain_back(dH * s["w"].float(), rh, rho2, case["center"])
    d = case["scale"] * gate * g
    out = {"dx": g.to(s["dr"].dtype), "dw": (dH * rh).sum(0), "db": dH.sum(0) if case["bias"] else None, "dgate": None,
           "dw_post": None, "db_post": None}
    if G:
        u = _plain_affine(yh, s["w_post"], s["b_post"])
        out["dgate"] = (case["scale"] * u * g).reshape(G, N // G, h).sum(1)
    if case["post"]:
        out["dw_post"] = (d * yh).sum(0)
        out["db_post"] = d.sum(0) if case["bias"] else None
        d = _plain_back(d * s["w_post"].float(), yh, rho1, case["center"])
    out["dy"] = d.to(s["dr"].dtype)
    return out


def _plain_grad_norm(grads):
    # long sums of squares: in 64 bits
    return torch.sqrt(torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads]).sum()).float().reshape(1)


def _plain_clip(grads, max_norm, outs):
    norm = _plain_grad_norm(grads)
    factor = torch.where((norm > max_norm) & torch.isfinite(norm), max_norm / norm, torch.ones_like(norm))
    [out.copy_(g.float() * factor) for g, out in zip(grads, outs)]
    return norm


# ----------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return _own(case, s)
    if case["op"] == "norm_fwd":
        return dict(zip(("r", "H", "stats"), _plain_norm_fwd(case, s)))
    if case["op"] == "norm_bwd":
        return _plain_norm_bwd(case, s)
    if case["op"] == "grad_norm":
        return {"norm": _plain_grad_norm(s["grads"])}
    return {"norm": _plain_clip(s["grads"], case["max_norm"], s["outs"]), "clipped": s["whole"]}


def _own(case, s):
    import paper_2411_05288_amd as vp
    if case["op"] == "norm_fwd":
        out = s["out"]
        vp.vp_block_norm_fwd(s["x"], s["y"], out["H"], r=out["r"], stats=out["stats"], gate=s["gate"], w=s["w"], b=s["b"],
                             w_post=s["w_post"], b_post=s["b_post"], scale=case["scale"], eps=EPS, post=case["post"],
                             center=case["center"])
        return out
    if case["op"] == "norm_bwd":
        if "workspace" not in s:      # once for these sizes
            n = vp.vp_block_norm_bwd_workspace_bytes(case["N"], case["h"], case["gate"], post=case["post"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        out = s["out"]
        vp.vp_block_norm_bwd(s["dH"], s["r"], s["y"], s["stats"], dr=s["dr"], gate=s["gate"], w=s["w"], w_post=s["w_post"],
                             b_post=s["b_post"], scale=case["scale"], post=case["post"], center=case["center"],
                             workspace=s["workspace"], **out)
        return out
    if "plan" not in s:               # once for these gradients
        s["plan"] = vp.GradientClipPlan(s["grads"], s.get("outs"))
    plan = s["plan"]
    if case["op"] == "grad_norm":
        plan.compute_norm()
        return {"norm": plan.norm}
    plan.clip(case["max_norm"])
    return {"norm": plan.norm, "clipped": s["whole"]}


# ----------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    if not case["op"].startswith("norm"):
        counts = _counts(case)
        size = sum(n * BYTES[t] for n, t in counts)
        n = sum(n for n, _ in counts)
        if case["op"] == "grad_norm":
            return {"bytes": size + 4, "flops": 2 * n}
        return {"bytes": 2 * size + 4, "flops": 3 * n}
    N, h, G, e = case["N"], case["h"], case["gate"], BYTES[case["dtype"]]
    vectors = h * (1 + case["post"]) * (1 + case["bias"])
    if case["op"] == "norm_fwd":
        return {"bytes": 4 * N * h * e + G * h * e + vectors * e + 16 * N, "flops": N * h * (9 + 8 * case["post"] + bool(G))}
    return {"bytes": N * h * (BYTES[case["grad_in"]] + 5 * e) + G * h * (e + 4) + vectors * (e + 4) + 16 * N,
            "flops": N * h * (13 + 12 * case["post"] + 4 * bool(G))}


# ----------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    if not case["op"].startswith("norm"):
        grads = [g.double() for g in _grad_inputs(case, seed)]
        total = math.sqrt(math.fsum(float(torch.dot(g, g)) for g in grads))
        norm = torch.tensor([total], dtype=torch.float64)
        if case["op"] == "grad_norm":
            return {"norm": norm}
        for g in grads:
            if total > case["max_norm"]:
                g.mul_(case["max_norm"] / total)
        if case["layout"] == "shards":
            return {"norm": norm, "clipped": grads}
        kinds = [t for _, t in _counts(case)]
        flat = [torch.cat([g for g, t in zip(grads, kinds) if t == k]) for k in DTYPES if k in kinds]
        return {"norm": norm, "clipped": [f for f in flat if f.numel()]}
    s = {k: None if v is None else v.double() for k, v in _norm_inputs(case, seed).items()}
    N, h, G, scale, center = case["N"], case["h"], case["gate"], case["scale"], case["center"]
    gate = torch.ones(1, 1, 1, dtype=torch.float64, device="cuda") if s["gate"] is None else s["gate"].reshape(G, 1, h)
    one, none = torch.ones(h, dtype=torch.float64, device="cuda"), torch.zeros(h, dtype=torch.float64, device="cuda")
    w_post = one if s["w_post"] is None else s["w_post"]
    b_post = none if s["b_post"] is None else s["b_post"]

    def gated(v):      # scale * gate * v, the tokens of one row of the gate together
        return scale * (v.reshape(gate.shape[0], -1, h) * gate).reshape(N, h)

    if case["op"] == "norm_fwd":
        def statistics(v):
            m = v.sum(1) / h * (1.0 if center else 0.0)
            return m, ((v - m[:, None]).pow(2).sum(1) / h + EPS).pow(-0.5)
        m1, rho1 = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.ones(N, dtype=torch.float64, device="cuda")
        if case["post"]:
            m1, rho1 = statistics(s["y"])
        r = s["x"] + gated((s["y"] - m1[:, None]) * rho1[:, None] * w_post + b_post)
        m2, rho2 = statistics(r)
        H = (r - m2[:, None]) * rho2[:, None] * s["w"] + (none if s["b"] is None else s["b"])
        return {"r": r, "H": H, "stats": torch.stack([m1, rho1, m2, rho2])}
    m1, rho1, m2, rho2 = (t[:, None] for t in s["stats"])

    def through(a, vh, rho):      # the gradient before a norm from the one behind it
        a = a - vh * ((a * vh).sum(1, keepdim=True) / h) - (a.sum(1, keepdim=True) / h if center else 0)
        return a * rho
    rh, yh = (s["r"] - m2) * rho2, (s["y"] - m1) * rho1
    dx = s["dr"] + through(s["dH"] * s["w"], rh, rho2)
    d = gated(dx)
    return {"dx": dx, "dy": through(d * w_post, yh, rho1) if case["post"] else d,
            "dgate": (scale * (yh * w_post + b_post) * dx).reshape(G, -1, h).sum(1) if G else None,
            "dw": (s["dH"] * rh).sum(0), "db": s["dH"].sum(0) if case["bias"] else None,
            "dw_post": (d * yh).sum(0) if case["post"] else None,
            "db_post": d.sum(0) if case["bias"] and case["post"] else None}
