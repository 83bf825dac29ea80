"""The network operators whose speed is measured, through the package's public entry points:
the parts of a residual block that proposes programs' parameters and trains through their
replay.

A case is one operator, its sizes, its type and whether the pass is a forward one (scoring,
no gradient) or a training step (forward and backward, all gradients returned):

  layer_norm  nd.layer_norm(x, weight, bias, eps)          rows x cols
  gated       nd.gated(x, w_gate, w_up, activation)        rows x cols -> rows x width
  dropout     nd.dropout(x, p, seed, offset, residual)     rows x cols

Rows are lanes (one row a lane, or a lane and a data point), so they range from one lane to
wide populations.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


# ------------------------------------------------------------------------------ the cases
def listed():
    return [
        # a small population's first layer in a scoring loop: latency counts
        _c("norm_64", "layer_norm", 64, 256, "bf16", train=False),
        # a training step at the usual width, weights kept in 32 bits beside 16-bit activations
        _c("norm_step", "layer_norm", 16384, 1024, "bf16", wtype="f32"),
        # single precision, odd row count and an odd width (nothing is 16-byte aligned)
        _c("norm_odd_f32", "layer_norm", 5001, 1537, "f32"),
        # the largest norm: a lane and a data point a row
        _c("norm_large", "layer_norm", 65536, 2048, "bf16"),
        # dropout on a small population's step
        _c("drop_64", "dropout", 64, 256, "f32", p=0.1),
        # odd sizes, half precision, no residual
        _c("drop_odd_f16", "dropout", 50001, 333, "f16", p=0.5, residual=False),
        # the residual sum of a wide population's training step
        _c("drop_large", "dropout", 65536, 2048, "bf16", p=0.1),
        # one lane's proposal: the weights are read once for one row
        _c("gated_one", "gated", 1, 2048, "bf16", width=8192, train=False),
        # a small population scored
        _c("gated_64", "gated", 64, 1024, "bf16", width=4096, train=False),
        # odd sizes in half precision, another activation
        _c("gated_odd_f16", "gated", 1501, 333, "f16", width=777, activation="gelu"),
        # a training step over a population of 4096 lanes
        _c("gated_step", "gated", 4096, 1024, "bf16", width=4096),
        # the largest training step
        _c("gated_large", "gated", 16384, 2048, "bf16", width=8192),
    ]


def _c(name, op, rows, cols, dtype, train=True, width=0, wtype="", activation="silu", p=0.0, residual=True):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "train": train, "width": width,
            "wtype": wtype or dtype, "activation": activation, "p": p, "residual": residual}


def draw(rng):
    """One more case of the listed ones' ranges: every operator, type and direction, from one
    row up, odd sizes among them; no more work than the largest listed case of its operator."""
    op = rng.choice(["layer_norm", "dropout", "gated"])
    most = [work(c) for c in listed() if c["op"] == op]
    train = rng.random() < 0.6
    while True:
        rows, cols, width, wtype, activation, p, residual = _log(rng, 1, 65536), _size(rng, 16, 8192), 0, "", "silu", 0.0, True
        if op == "gated":
            dtype = rng.choice(["bf16", "bf16", "f16"])
            rows, cols, width = _log(rng, 1, 32768), _size(rng, 16, 4096), _size(rng, 16, 8192)
            activation = rng.choice(["silu", "silu", "gelu", "relu", "sigmoid"])
        else:
            dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
            if op == "layer_norm":
                wtype = rng.choice([dtype, "f32"])
            else:
                p, residual = rng.choice([0.05, 0.1, 0.2, 0.5]), rng.random() < 0.7
        case = _c("", op, rows, cols, dtype, train, width, wtype, activation, p, residual)
        del case["name"]
        w = work(case)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most) and w["bytes"] >= 1000:
            return case


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: a multiple of 64 half of the time, any number otherwise."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


# ------------------------------------------------------------------------------- the work
def work(case):
    r, c, n, b = case["rows"], case["cols"], case["width"], 4 if case["dtype"] == "f32" else 2
    wb = 4 if case["wtype"] == "f32" else 2
    if case["op"] == "layer_norm":
        if case["train"]:  # x, dy, y, dx; weight, bias and their gradients
            return {"bytes": 4 * r * c * b + 4 * c * wb, "flops": 20 * r * c}
        return {"bytes": 2 * r * c * b + 2 * c * wb, "flops": 8 * r * c}
    if case["op"] == "dropout":
        arrays = 2 + (1 if case["residual"] else 0) + (2 if case["train"] else 0)
        return {"bytes": arrays * r * c * b, "flops": (4 if case["train"] else 2) * r * c}
    if case["train"]:  # x, dx; both weights and their gradients; h, dh
        return {"bytes": (2 * r * c + 4 * n * c + 2 * r * n) * b, "flops": 12 * r * n * c}
    return {"bytes": (r * c + 2 * n * c + r * n) * b, "flops": 4 * r * n * c}


# ----------------------------------------------------------------------------- the inputs
def prepare(case, seed):
    """Activations as a residual stream has them (each column its own level and spread), weights
    as a trained layer's, cotangents of unit scale (a scaled loss)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    r, c, n, t = case["rows"], case["cols"], case["width"], TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    s = {"case": case}
    if case["op"] == "layer_norm":
        x = normal(r, c).mul_(1.0 + 0.5 * torch.rand(c, generator=g, device="cuda")).add_(0.5 * normal(c))
        s["x"] = x.to(t)
        s["weight"] = (1.0 + 0.2 * normal(c)).to(TYPES[case["wtype"]])
        s["bias"] = (0.2 * normal(c)).to(TYPES[case["wtype"]])
        leaves = ("x", "weight", "bias")
    elif case["op"] == "dropout":
        s["x"] = normal(r, c).to(t)
        s["residual"] = normal(r, c).to(t) if case["residual"] else None
        s["seed"] = int(seed) * 0x9E3779B97F4A7C15 % (1 << 64)
        s["offset"] = 4 * (int(seed) % 1000003)
        leaves = ("x", "residual")
    else:
        s["x"] = normal(r, c).to(t)
        s["w_gate"] = normal(n, c).mul_(c ** -0.5).to(t)
        s["w_up"] = normal(n, c).mul_(c ** -0.5).to(t)
        leaves = ("x", "w_gate", "w_up")
    if case["train"]:
        s["dy"] = normal(r, n if case["op"] == "gated" else c).to(t)
        for k in leaves:
            if s[k] is not None:
                s[k].requires_grad_(True)
    return s


# ----------------------------------------------------------------------------- the passes
def run(state):
    return (_own if own else _plain)(state)


def _own(s):
    import paper_2607_03574_gb300 as nd
    case = s["case"]
    with torch.set_grad_enabled(case["train"]):
        if case["op"] == "layer_norm":
            y, inputs = nd.layer_norm(s["x"], s["weight"], s["bias"], EPS), {k: s[k] for k in ("x", "weight", "bias")}
        elif case["op"] == "dropout":
            y, inputs = nd.dropout(s["x"], case["p"], s["seed"], s["offset"], s["residual"]), {"x": s["x"]}
        else:
            y = nd.gated(s["x"], s["w_gate"], s["w_up"], case["activation"])
            inputs = {k: s[k] for k in ("x", "w_gate", "w_up")}
    if not case["train"]:
        return {"y": y}
    grads = torch.autograd.grad(y, list(inputs.values()), s["dy"])
    return {"y": y.detach(), **{"d" + k: v for k, v in zip(inputs, grads)}}


@torch.no_grad()
def _plain(s):
    case = s["case"]
    return {"layer_norm": _plain_norm, "dropout": _plain_dropout, "gated": _plain_gated}[case["op"]](s, case["train"])


def _plain_norm(s, train):
    x, w, b = s["x"].float(), s["weight"].float(), s["bias"].float()
    xc = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    xh = xc * r
    out = {"y": (xh * w + b).to(s["x"].dtype)}
    if train:
        dy = s["dy"].float()
        g = dy * w
        out["dx"] = (r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))).to(s["x"].dtype)
        out["dweight"] = (dy * xh).sum(0).to(s["weight"].dtype)
        out["dbias"] = dy.sum(0).to(s["bias"].dtype)
    return out


def _plain_gated(s, train):
    x, wg, wu, t, act = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["x"].dtype, s["case"]["activation"]
    g, u = x @ wg.t(), x @ wu.t()
    if act == "relu":
        a, da = g.clamp_min(0.0), (g > 0).float()
    elif act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        a, da = g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    else:
        sg = 1.0 / (1.0 + torch.exp(-g))
        a, da = (g * sg, sg * (1.0 + g * (1.0 - sg))) if act == "silu" else (sg, sg * (1.0 - sg))
    out = {"y": (a * u).to(t)}
    if train:
        dy = s["dy"].float()
        du, dg = dy * a, dy * u * da
        out["dx"] = (dg @ wg + du @ wu).to(t)
        out["dw_gate"], out["dw_up"] = (dg.t() @ x).to(t), (du.t() @ x).to(t)
    return out


def _plain_dropout(s, train):
    x, case, n = s["x"], s["case"], s["x"].numel()
    keep = _words(s["seed"], s["offset"], n, x.device) >= round(case["p"] * 2.0 ** 32)
    keep, scale = keep.view(x.shape), 1.0 / (1.0 - case["p"])
    y = torch.where(keep, x.float() * scale, 0.0)
    if s["residual"] is not None:
        y += s["residual"].float()
    out = {"y": y.to(x.dtype)}
    if train:
        out["dx"] = torch.where(keep, s["dy"].float() * scale, 0.0).to(x.dtype)
    return out


def _words(seed, offset, n, device):
    """Words offset .. offset + n - 1 of the sequence: counter-based generator of four 32-bit words a
    block (Philox with 10 rounds; Salmon, Moraes, Dror, Shaw, 2011).  Block q has the counter
    (q mod 2^32, q / 2^32, 0, 0); the key is the seed.  A product's 64 bits are an int64's, whatever its
    sign, so its high half is a shift and a mask.  (The loop is over the generator's rounds.)"""
    low = 0xFFFFFFFF
    q = torch.arange(offset // 4, offset // 4 + (n + 3) // 4, device=device, dtype=torch.int64)
    a, b = q & low, q >> 32
    c = d = torch.zeros_like(q)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p, r = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = (r >> 32 & low) ^ b ^ k0, r & low, (p >> 32 & low) ^ d ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((a, b, c, d), 1).view(-1)[:n]


# --------------------------------------------------------------------- answers in 64 bits
def exact(case, seed):
    """The definition in 64 bits; gradients are torch's derivative of that definition."""
    if work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    x = s["x"].detach().double().requires_grad_(True)
    if case["op"] == "layer_norm":
        inputs = {"x": x, **{k: s[k].detach().double().requires_grad_(True) for k in ("weight", "bias")}}
        y = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + EPS).sqrt() * inputs["weight"] + inputs["bias"]
    elif case["op"] == "dropout":
        inputs = {"x": x}
        y = x * torch.from_numpy(_factors(case, s["seed"], s["offset"])).to(x.device)
        if case["residual"]:
            y = y + s["residual"].detach().double()
    else:
        inputs = {"x": x, **{k: s[k].detach().double().requires_grad_(True) for k in ("w_gate", "w_up")}}
        g = torch.nn.functional.linear(x, inputs["w_gate"])
        act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu, "sigmoid": torch.sigmoid}
        y = act[case["activation"]](g) * torch.nn.functional.linear(x, inputs["w_up"])
    if not case["train"]:
        return {"y": y.detach()}
    grads = torch.autograd.grad(y, list(inputs.values()), s["dy"].double())
    return {"y": y.detach(), **{"d" + k: v for k, v in zip(inputs, grads)}}


def _factors(case, seed, offset):
    """What each element is multiplied by: 0 or 1 / (1 - p), in unsigned 64-bit arithmetic."""
    n, low, u = case["rows"] * case["cols"], np.uint64(0xFFFFFFFF), np.uint64
    block = np.arange((n + 3) // 4, dtype=np.uint64) + u(offset // 4)
    words = [block & low, block >> u(32), np.zeros_like(block), np.zeros_like(block)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        first, second = words[0] * u(0xD2511F53), words[2] * u(0xCD9E8D57)
        words = [second >> u(32) ^ words[1] ^ u(key[0]), second & low, first >> u(32) ^ words[3] ^ u(key[1]), first & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    kept = np.stack(words, 1).reshape(-1)[:n] >= u(round(case["p"] * 2 ** 32))
    return np.where(kept, 1.0 / (1.0 - case["p"]), 0.0).reshape(case["rows"], case["cols"])
