"""The passes around the optimizer step whose time is measured: a linear layer's three products with what is fused into
them, an activation's gradient, and layer norm, forward and backward.

A case is one call of a training loop (or of a model that answers token by token) on t tokens: `forward` is
Y = act(X W^T + b) + R, `input` is dX = (dY W) act'(Z), `weight` is G = dY^T X with the bias gradient, `activation` is
dZ = dY act'(Z), `norm` and `norm_backward` are layer norm's passes. W and G have the step's layout, [rows][cols] =
fan-out x fan-in. `own` says whether a pass computes the plain form or calls the library.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # a model that answers: one token through the 1B model's first MLP matrix; W is read once, everything else is latency
        {"name": "forward-one-token", "op": "forward", "tokens": 1, "rows": 8192, "cols": 2048, "type": "bf16", "act": "gelu", "bias": True},
        # the smallest training pass: one 256 x 256 fp32 layer, an odd number of tokens
        {"name": "forward-256-fp32", "op": "forward", "tokens": 301, "rows": 256, "cols": 256, "type": "f32", "act": "relu", "bias": True, "keep": True},
        # the 1B model's second MLP matrix over a micro-batch of eight sequences of 2048, added to the residual stream
        {"name": "forward-mlp-down", "op": "forward", "tokens": 16384, "rows": 2048, "cols": 8192, "type": "bf16", "act": "none", "bias": True, "residual": True},
        # its input gradient, through the GELU that the first MLP matrix kept its inputs for
        {"name": "input-mlp-down", "op": "input", "tokens": 8192, "rows": 2048, "cols": 8192, "type": "bf16", "act": "gelu"},
        # nothing is a multiple of a tile or of a vector; the rows of dY are part of a wider buffer
        {"name": "input-odd", "op": "input", "tokens": 1531, "rows": 1000, "cols": 517, "type": "bf16", "act": "silu", "pitch": 24},
        # the gradient that the step takes of the 1B model's first MLP matrix, over the micro-batch, with the bias gradient
        {"name": "weight-mlp-up", "op": "weight", "tokens": 16384, "rows": 8192, "cols": 2048, "type": "bf16", "g": "bf16", "bias": True},
        # an attention matrix of the 304M model over one sequence: a small matrix, so the tokens are what can be split; fp32 G
        {"name": "weight-304m-attn", "op": "weight", "tokens": 2048, "rows": 1024, "cols": 1024, "type": "bf16", "g": "f32"},
        # a GELU whose output no product follows, over one sequence of the 7B model's MLP width
        {"name": "activation-gelu", "op": "activation", "tokens": 2048, "rows": 11008, "cols": 0, "type": "bf16", "act": "gelu"},
        # the residual stream's norm: one token, and the 1B model's micro-batch
        {"name": "norm-one-token", "op": "norm", "tokens": 1, "rows": 0, "cols": 2048, "type": "bf16"},
        {"name": "norm-1b", "op": "norm", "tokens": 16384, "rows": 0, "cols": 2048, "type": "bf16", "keep": True},
        # its backward pass, the residual's own gradient added; and an odd fp32 one
        {"name": "norm-backward-1b", "op": "norm_backward", "tokens": 16384, "rows": 0, "cols": 2048, "type": "bf16", "g": "bf16", "residual": True},
        {"name": "norm-backward-odd-fp32", "op": "norm_backward", "tokens": 777, "rows": 0, "cols": 1001, "type": "f32", "g": "f32"},
    ]


def _most():
    w = [work(c) for c in listed()]
    return max(x["bytes"] for x in w), max(x["flops"] for x in w)


def draw(rng):
    """A pass of any of the six kinds: 1 to 16384 tokens, matrix sides of 48 to 11008, odd ones as often as whole tiles."""
    most_b, most_f = _most()

    def size(lo, hi, step):
        n = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return max(lo, n // step * step) if rng.random() < 0.5 and n >= step else n

    while True:
        op = rng.choice(("forward", "forward", "input", "input", "weight", "weight", "activation", "norm", "norm_backward"))
        case = {"op": op, "tokens": size(1, 16384, 64), "rows": size(48, 11008, 64), "cols": size(48, 11008, 64),
                "type": rng.choice(("bf16", "bf16", "bf16", "f32"))}
        if op in ("norm", "norm_backward"):
            case["rows"] = 0
        if op == "activation":
            case["cols"] = 0
        if op in ("forward", "input", "activation"):
            case["act"] = rng.choice(("relu", "gelu", "gelu_tanh", "silu") + ("none",) * (op != "activation"))
        if op in ("forward", "weight"):
            case["bias"] = rng.random() < 0.5
        if op in ("forward", "norm"):
            case["keep"] = rng.random() < 0.5
        if op in ("forward", "norm_backward"):
            case["residual"] = rng.random() < 0.5
        if op in ("weight", "norm_backward"):
            case["g"] = rng.choice(("bf16", "f32"))
        if rng.random() < 0.25:
            case["pitch"] = rng.choice((8, 64, 13, 512))
        w = work(case)
        if w["bytes"] <= most_b and w["flops"] <= (most_f if case["type"] == "bf16" else most_f / 16):
            return case


def _item(kind):
    return 2 if kind == "bf16" else 4


def work(case):
    t, r, c, e = case["tokens"], case["rows"], case["cols"], _item(case["type"])
    g, op = _item(case.get("g", "bf16")), case["op"]
    if op == "forward":
        held = 1 + bool(case.get("residual")) + bool(case.get("keep"))
        return {"bytes": e * (t * c + r * c + t * r * held), "flops": 2 * t * r * c}
    if op == "input":
        held = 1 + (case["act"] != "none")
        return {"bytes": e * (t * r + r * c + t * c * held), "flops": 2 * t * r * c}
    if op == "weight":
        return {"bytes": e * t * (r + c) + g * r * c, "flops": 2 * t * r * c}
    if op == "activation":
        return {"bytes": 3 * e * t * r, "flops": 12 * t * r}
    if op == "norm":
        return {"bytes": 2 * e * t * c, "flops": 8 * t * c}
    return {"bytes": e * t * c * (3 + bool(case.get("residual"))) + 2 * g * c, "flops": 14 * t * c}


def _inputs(case, seed, device="cuda"):
    """Activations of std 1 (a residual stream: tokens of different size, an offset, some channels twenty times the
    others), weights N(0, 0.02^2) and gradients of std 1e-3 with a log-normal scale per token."""
    gen = torch.Generator(device=device)
    gen.manual_seed(int(seed) * 1000003 + 29)
    t, r, c, dt, op = case["tokens"], case["rows"], case["cols"], _TYPES[case["type"]], case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=device)

    def rows(x):   # in the type of the activations; with a pitch, as part of a wider buffer
        out = torch.zeros((x.shape[0], x.shape[1] + case.get("pitch", 0)), dtype=dt, device=device)[:, :x.shape[1]]
        return out.copy_(x)

    def gradient(n):
        return rows(normal(t, n).mul_(1e-3 * torch.exp(normal(t, 1))))

    d = {}
    if op == "forward":
        d["X"], d["W"] = rows(normal(t, c)), normal(r, c).mul_(0.02).to(dt)
        d["bias"] = normal(r).mul_(0.1).to(dt) if case.get("bias") else None
        d["R"] = rows(normal(t, r)) if case.get("residual") else None
    elif op == "input":
        d["dY"], d["W"] = gradient(r), normal(r, c).mul_(0.02).to(dt)
        d["Z"] = rows(normal(t, c)) if case["act"] != "none" else None
    elif op == "weight":
        d["dY"], d["X"] = gradient(r), rows(normal(t, c))
    elif op == "activation":
        d["dY"], d["Z"] = gradient(r), rows(normal(t, r))
    else:
        loud = 1.0 + 19.0 * (torch.rand(c, generator=gen, device=device) < 0.01)
        d["X"] = rows((normal(t, c) * loud + 0.5 * normal(1, c)) * torch.exp(0.5 * normal(t, 1)))
        d["gamma"] = (1.0 + 0.1 * normal(c)).to(dt)
        d["beta"] = normal(c).mul_(0.1).to(dt)
        if op == "norm_backward":
            d["dY"] = gradient(c)
            d["dR"] = gradient(c) if case.get("residual") else None
            x = d["X"].double()
            mean = x.mean(1)
            d["mean"] = mean.float()
            d["rstd"] = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
    return d


def prepare(case, seed):
    """The inputs, and the buffers that a training loop keeps for the outputs."""
    d = _inputs(case, seed)
    t, r, c, dt, op = case["tokens"], case["rows"], case["cols"], _TYPES[case["type"]], case["op"]
    g = _TYPES[case.get("g", "bf16")]

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if op == "forward":
        out = {"Y": empty(t, r), "Z": empty(t, r) if case.get("keep") else None}
    elif op == "input":
        out = {"dX": empty(t, c)}
    elif op == "weight":
        out = {"G": empty(r, c, dtype=g), "dbias": empty(r, dtype=g) if case.get("bias") else None}
    elif op == "activation":
        out = {"dZ": empty(t, r)}
    elif op == "norm":
        keep = case.get("keep")
        out = {"Y": empty(t, c), "mean": empty(t, dtype=torch.float32) if keep else None,
               "rstd": empty(t, dtype=torch.float32) if keep else None}
    else:
        out = {"dX": empty(t, c), "dgamma": empty(c, dtype=g), "dbeta": empty(c, dtype=g)}
    return {"case": dict(case), "in": d, "out": out}


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        k = 2.0 * math.sqrt(2.0 / math.pi)
        s = torch.sigmoid(k * (z + 0.044715 * z * z * z))
        return s + z * s * (1.0 - s) * k * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _plain(case, d, out):
    op, dt, act = case["op"], _TYPES[case["type"]], case.get("act", "none")
    if op == "forward":
        z = d["X"].float() @ d["W"].float().T
        if d["bias"] is not None:
            z = z + d["bias"].float()
        y = _act(z, act)
        if d["R"] is not None:
            y = y + d["R"].float()
        return {"Y": y.to(dt), "Z": z.to(dt) if case.get("keep") else None}
    if op == "input":
        x = d["dY"].float() @ d["W"].float()
        if act != "none":
            x = x * _act_slope(d["Z"].float(), act)
        return {"dX": x.to(dt)}
    if op == "weight":
        g = _TYPES[case["g"]]
        dy = d["dY"].float()
        return {"G": (dy.T @ d["X"].float()).to(g), "dbias": dy.sum(0).to(g) if case.get("bias") else None}
    if op == "activation":
        return {"dZ": (d["dY"].float() * _act_slope(d["Z"].float(), act)).to(dt)}
    x = d["X"].float()
    if op == "norm":
        mean = x.mean(1, keepdim=True)
        x = x - mean
        rstd = (x.square().mean(1, keepdim=True) + EPS).rsqrt()
        y = x * rstd * d["gamma"].float() + d["beta"].float()
        keep = case.get("keep")
        return {"Y": y.to(dt), "mean": mean[:, 0] if keep else None, "rstd": rstd[:, 0] if keep else None}
    g = _TYPES[case["g"]]
    dy, rstd = d["dY"].float(), d["rstd"][:, None]
    xh = (x - d["mean"][:, None]) * rstd
    h = dy * d["gamma"].float()
    dx = rstd * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    if d["dR"] is not None:
        dx = dx + d["dR"].float()
    return {"dX": dx.to(dt), "dgamma": (dy * xh).sum(0).to(g), "dbeta": dy.sum(0).to(g)}


def run(state):
    case, d, out = state["case"], state["in"], state["out"]
    if own:
        from paper_2512_16928_amd import binding
        op, act = case["op"], binding.ACTIVATIONS[case.get("act", "none")]
        if op == "forward":
            binding.dion2_linear_forward(out["Y"], d["X"], d["W"], bias=d["bias"], residual=d["R"], Z=out["Z"], act=act)
        elif op == "input":
            binding.dion2_linear_backward_input(out["dX"], d["dY"], d["W"], Z=d["Z"], act=act)
        elif op == "weight":
            binding.dion2_linear_backward_weight(out["G"], d["dY"], d["X"], dbias=out["dbias"])
        elif op == "activation":
            binding.dion2_activation_backward(out["dZ"], d["dY"], d["Z"], act)
        elif op == "norm":
            binding.dion2_layernorm_forward(out["Y"], d["X"], d["gamma"], d["beta"], eps=EPS, mean=out["mean"], rstd=out["rstd"])
        else:
            binding.dion2_layernorm_backward(out["dX"], d["dY"], d["X"], d["mean"], d["rstd"], gamma=d["gamma"],
                                             residual_grad=d["dR"], dgamma=out["dgamma"], dbeta=out["dbeta"])
        return out
    return _plain(case, d, out)


def exact(case, seed):
    """The definitions in 64 bits; gradients of activations and of the norm by differentiating those."""
    d = {k: None if v is None else v.double() for k, v in _inputs(case, seed).items()}
    op, act = case["op"], case.get("act", "none")

    def apply(z):
        if act == "relu":
            return torch.clamp(z, min=0.0)
        if act == "gelu":
            return z * torch.special.ndtr(z)
        if act == "gelu_tanh":
            return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
        if act == "silu":
            return z / (1.0 + torch.exp(-z))
        return z * 1.0

    def through(z, dy):
        z = z.detach().requires_grad_(True)
        return torch.autograd.grad(apply(z), z, dy)[0]

    if op == "forward":
        z = torch.mm(d["X"], d["W"].t())
        if d["bias"] is not None:
            z += d["bias"]
        y = apply(z)
        if d["R"] is not None:
            y = y + d["R"]
        return {"Y": y, "Z": z if case.get("keep") else None}
    if op == "input":
        x = torch.mm(d["dY"], d["W"])
        return {"dX": x if act == "none" else through(d["Z"], x)}
    if op == "weight":
        return {"G": torch.mm(d["dY"].t(), d["X"]), "dbias": d["dY"].sum(0) if case.get("bias") else None}
    if op == "activation":
        return {"dZ": through(d["Z"], d["dY"])}
    if op == "norm":
        var, mean = torch.var_mean(d["X"], 1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = (d["X"] - mean[:, None]) * rstd[:, None] * d["gamma"] + d["beta"]
        keep = case.get("keep")
        return {"Y": y, "mean": mean if keep else None, "rstd": rstd if keep else None}
    # The statistics given are the forward pass's in fp32: the same function of x to 32 bits.
    x, gamma, beta = (v.detach().requires_grad_(True) for v in (d["X"], d["gamma"], d["beta"]))
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    y = (x - mean) / torch.sqrt(var + EPS) * gamma + beta
    dx, dg, db = torch.autograd.grad(y, (x, gamma, beta), d["dY"])
    return {"dX": dx if d["dR"] is None else dx + d["dR"], "dgamma": dg, "dbeta": db}
