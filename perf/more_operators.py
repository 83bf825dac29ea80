"""The operators of a pre-norm residual block whose speed is measured, through the package's public entry points:
the root-mean-square norm that also adds up the residual stream, dense layers with all of their epilogue, dense layers
that hold what their backward pass needs in 8 bits, and the 8-bit path on which a trained network is scored.

  rms_norm  nd.rms_norm(x, weight, eps, residual)                          rows x cols
  linear    nd.linear(x, w, bias, activation, residual)                    rows x cols -> rows x width
  kept      the same with keep="8bit": what the backward pass reads of x and of the pre-activations is held as 8-bit blocks
  scored    nd.linear_quantized(nd.rms_norm_quantized(x, weight, eps, residual), w, bias, activation), or without a norm
            nd.linear_quantized(nd.quantize(x), w, bias, activation, residual); w in 8-bit blocks

8-bit blocks: 32 consecutive elements of a row share a scale 2^e, the least (from e = -127 on) with which none is over
448 in size; an element is the nearest e4m3 value to v / 2^e (even ones at ties).

Rows are lanes (one row a lane, or a lane and a data point).  A forward pass alone is scoring; a training step returns
the outputs and all gradients.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# ------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the norm of a small population's first block in a scoring loop: latency counts
        _c("rms_64", "rms_norm", 64, 256, "bf16", train=False),
        # a training step at the usual width, weights kept in 32 bits beside 16-bit activations
        _c("rms_step", "rms_norm", 16384, 1024, "bf16", wtype="f32"),
        # single precision, odd sizes (nothing is 16-byte aligned), the first norm (no residual yet)
        _c("rms_odd_f32", "rms_norm", 5001, 1537, "f32", residual=False),
        # a lane and a data point a row
        _c("rms_large", "rms_norm", 65536, 2048, "bf16"),
        # one lane's proposal: the weights are read once for one row
        _c("linear_one", "linear", 1, 2048, "bf16", width=8192, activation="silu", residual=False, train=False),
        # odd sizes in half precision, another activation
        _c("linear_odd_f16", "linear", 1501, 777, "f16", width=333, activation="gelu", residual=False),
        # a training step's projection back into the residual stream, bias kept in 32 bits
        _c("linear_step", "linear", 4096, 4096, "bf16", width=1024, wtype="f32"),
        # the largest training step
        _c("linear_large", "linear", 16384, 2048, "bf16", width=8192, activation="gelu", residual=False),
        # a small population's training step with its activations held in 8 bits, ragged sizes
        _c("kept_small", "kept", 250, 200, "bf16", width=616, activation="silu", residual=False),
        # the same of a wide population, into the residual stream
        _c("kept_step", "kept", 16384, 1024, "bf16", width=1024, activation="silu"),
        # a small population scored
        _c("scored_64", "scored", 64, 1024, "bf16", width=4096, activation="silu", residual=False),
        # the largest scoring pass: the stream's sum, its norm and the layer that reads it
        _c("scored_large", "scored", 16384, 2048, "bf16", width=8192, activation="gelu", norm=True),
    ]


def _c(name, op, rows, cols, dtype, train=True, width=0, wtype="", activation="", residual=True, norm=False):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "train": train and op != "scored", "width": width,
            "wtype": wtype or dtype, "activation": activation, "residual": residual, "norm": norm}


def draw(rng):
    """One more case of the listed ones' ranges: every operator, type, activation and direction, from one row up, odd
    sizes among them; no more work than the largest listed case of its operator."""
    op = rng.choice(["rms_norm", "rms_norm", "linear", "linear", "kept", "scored"])
    most = [work(c) for c in listed() if c["op"] == op]
    while True:
        rows, cols, width, activation, norm = _log(rng, 1, 65536), _size(rng, 16, 8192), 0, "", False
        residual, train = rng.random() < 0.6, op == "kept" or rng.random() < 0.6
        if op == "rms_norm":
            dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
            wtype = rng.choice([dtype, "f32"])
        else:
            dtype = rng.choice(["bf16", "bf16", "f16"])
            rows, width = _log(rng, 1, 32768), _size(rng, 16, 8192)
            # a binary32 bias beside smooth pre-activations: what lies at a border (relu's 0, an 8-bit step's) decides
            # about whole terms of its gradient, which 32 bits then say too exactly
            activation = rng.choice(["", "silu", "gelu", "relu", "sigmoid"])
            wtype = rng.choice([dtype, "f32"]) if op == "linear" and activation != "relu" else dtype
            norm = op == "scored" and rng.random() < 0.5
        case = _c("", op, rows, cols, dtype, train, width, wtype, activation, residual, norm)
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
    wb, res = 4 if case["wtype"] == "f32" else 2, 1 if case["residual"] else 0
    if case["op"] == "rms_norm":
        if case["train"]:  # x, dy, y, dx; the residual, the sum and its cotangent; weight and its gradient
            return {"bytes": (4 + 3 * res) * r * c * b + 2 * c * wb, "flops": 16 * r * c}
        return {"bytes": (2 + 2 * res) * r * c * b + c * wb, "flops": 5 * r * c}
    if case["op"] == "scored":
        stream = 1 + (2 if case["norm"] and res else 0)  # x; the residual and the sum
        rest = 1 + (1 if res and not case["norm"] else 0)  # y; the residual
        return {"bytes": stream * r * c * b + n * c * 33 // 32 + rest * r * n * b + n * wb, "flops": 2 * r * n * c}
    if case["train"]:  # x, dx; w and its gradient; y, dy, the residual; bias and its gradient
        return {"bytes": (2 * r * c + 2 * n * c + (2 + res) * r * n) * b + 2 * n * wb, "flops": 6 * r * n * c}
    return {"bytes": (r * c + n * c + (1 + res) * r * n) * b + n * wb, "flops": 2 * r * n * c}


# ----------------------------------------------------------------------------- the inputs
def prepare(case, seed):
    """Activations as a residual stream has them (each column its own spread, some columns far wider than the rest),
    weights as a trained layer's, cotangents of unit scale (a scaled loss)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    r, c, n, t, wt = case["rows"], case["cols"], case["width"], TYPES[case["dtype"]], TYPES[case["wtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    def stream():
        spread = 0.5 + torch.rand(c, generator=g, device="cuda")
        spread[torch.rand(c, generator=g, device="cuda") < 0.01] *= 20.0
        return normal(r, c).mul_(spread).to(t)

    s = {"case": case, "residual": None}
    leaves = []
    if case["op"] == "rms_norm":
        s["x"], s["weight"] = stream(), (1.0 + 0.2 * normal(c)).to(wt)
        leaves += ["x", "weight"]
        if case["residual"]:
            s["residual"] = stream()
            leaves.append("residual")
        if case["train"]:
            s["dy"] = normal(r, c).to(t)
            s["dsum"] = normal(r, c).to(t) if case["residual"] else None
    else:
        s["x"] = stream() if case["op"] == "scored" else normal(r, c).to(t)
        w = normal(n, c).mul_(c ** -0.5)
        s["bias"] = (0.2 * normal(n)).to(wt)
        s["weight"] = (1.0 + 0.2 * normal(c)).to(t) if case["norm"] else None
        if case["residual"]:
            s["residual"] = stream() if case["norm"] else normal(r, n).to(t)
        if case["op"] == "scored":
            s["w"], s["w_scales"] = _encode(w)
        else:
            s["w"] = w.to(t)
        leaves += ["x", "w", "bias"] + (["residual"] if case["residual"] else [])
        if case["train"]:
            s["dy"] = normal(r, n).to(t)
    if case["train"]:
        for k in leaves:
            s[k].requires_grad_(True)
    return s


def _encode(w):
    """A weight matrix in 8-bit blocks as nd.Quantized holds it: e4m3 values in rows of whole 16 bytes, and the exponents
    + 127 as bytes [row / 128][column / 128][row % 32][row / 32 % 4][column / 32 % 4]."""
    n, c = w.shape
    q, e = _blocks(w)
    values = torch.zeros(n, -(-c // 16) * 16, dtype=torch.float8_e4m3fn, device=w.device)
    values.view(torch.uint8)[:, :c] = q.to(torch.float8_e4m3fn).view(torch.uint8)
    codes = torch.zeros(-(-n // 128) * 128, -(-c // 128) * 4, dtype=torch.uint8, device=w.device)
    codes[:n, :e.shape[1]] = (e + 127).to(torch.uint8)
    codes = codes.view(-1, 4, 32, codes.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()
    return values[:, :c], codes


# ----------------------------------------------------------------------------- the passes
def run(state):
    return (_own if own else _plain)(state)


def _own(s):
    import paper_2607_03574_gb300 as nd
    case = s["case"]
    act, outputs, cotangents = case["activation"] or None, {}, []
    with torch.set_grad_enabled(case["train"]):
        if case["op"] == "rms_norm":
            inputs = {k: s[k] for k in ("x", "weight")}
            y = nd.rms_norm(s["x"], s["weight"], EPS, s["residual"])
            if case["residual"]:
                inputs["residual"] = s["residual"]
                outputs["y"], outputs["sum"] = y
                cotangents = [s.get("dy"), s.get("dsum")]
            else:
                outputs["y"], cotangents = y, [s.get("dy")]
        elif case["op"] == "scored":
            w = nd.Quantized(s["w"], s["w_scales"])
            if case["norm"] and case["residual"]:
                x, outputs["sum"] = nd.rms_norm_quantized(s["x"], s["weight"], EPS, s["residual"])
            elif case["norm"]:
                x = nd.rms_norm_quantized(s["x"], s["weight"], EPS)
            else:
                x = nd.quantize(s["x"])
            outputs["y"] = nd.linear_quantized(x, w, s["bias"], act, None if case["norm"] else s["residual"], s["x"].dtype)
        else:
            inputs = {k: s[k] for k in ("x", "w", "bias", "residual") if s[k] is not None}
            outputs["y"] = nd.linear(s["x"], s["w"], s["bias"], act, s["residual"], keep="8bit" if case["op"] == "kept" else None)
            cotangents = [s.get("dy")]
    if not case["train"]:
        return outputs
    grads = torch.autograd.grad(list(outputs.values()), list(inputs.values()), cotangents)
    return {**{k: v.detach() for k, v in outputs.items()}, **{"d" + k: v for k, v in zip(inputs, grads)}}


@torch.no_grad()
def _plain(s):
    return {"rms_norm": _plain_norm, "linear": _plain_linear, "kept": _plain_linear, "scored": _plain_scored}[s["case"]["op"]](s)


def _plain_norm(s):
    t, out = s["x"].dtype, {}
    x, w = s["x"].float(), s["weight"].float()
    if s["residual"] is not None:  # the stream goes on in its own type, and the norm is that of the stream
        out["sum"] = (x + s["residual"].float()).to(t)
        x = out["sum"].float()
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    xh = x * r
    out["y"] = (xh * w).to(t)
    if s["case"]["train"]:
        dy = s["dy"].float()
        g = dy * w
        dx = r * (g - xh * (g * xh).mean(1, keepdim=True))
        if s["residual"] is not None:
            dx = dx + s["dsum"].float()
        out["dx"], out["dweight"] = dx.to(t), (dy * xh).sum(0).to(s["weight"].dtype)
        if s["residual"] is not None:
            out["dresidual"] = out["dx"]
    return out


def _activate(z, act):
    """(act(z), act'(z))"""
    if act == "":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp_min(0.0), (z > 0).float()
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sg = 1.0 / (1.0 + torch.exp(-z))
    return (z * sg, sg * (1.0 + z * (1.0 - sg))) if act == "silu" else (sg, sg * (1.0 - sg))


def _plain_linear(s):
    case, t = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t() + s["bias"].float()
    y = _activate(z, case["activation"])[0]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(t)}
    if case["train"]:
        if case["op"] == "kept":
            x, z = _held(x).to(t).float(), _held(z)
        dy = s["dy"].float()
        dz = dy * _activate(z, case["activation"])[1]
        out["dx"], out["dw"], out["dbias"] = (dz @ w).to(t), (dz.t() @ x).to(t), dz.sum(0).to(s["bias"].dtype)
        if s["residual"] is not None:
            out["dresidual"] = s["dy"]
    return out


def _plain_scored(s):
    case, t, out = s["case"], s["x"].dtype, {}
    x, n, c = s["x"].float(), case["width"], case["cols"]
    if case["norm"]:
        if s["residual"] is not None:
            out["sum"] = (x + s["residual"].float()).to(t)
            x = out["sum"].float()
        x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["weight"].float()
    codes = s["w_scales"].permute(0, 3, 2, 1, 4).reshape(s["w_scales"].shape[0] * 128, -1)[:n]
    w = s["w"].float() * torch.exp2(codes.float() - 127.0).repeat_interleave(32, 1)[:, :c]
    y = _activate(_held(x) @ w.t() + s["bias"].float(), case["activation"])[0]
    if s["residual"] is not None and not case["norm"]:
        y = y + s["residual"].float()
    out["y"] = y.to(t)
    return out


def _blocks(v):
    """(values over their block's scale, rounded to e4m3; the exponents of the scales [rows, blocks])"""
    rows, cols = v.shape
    padded = torch.nn.functional.pad(v, (0, -cols % 32)).view(rows, -1, 32)
    mantissa, exponent = torch.frexp(padded.abs().amax(2))
    e = (exponent - 9 + (mantissa > 0.875)).clamp_min(-127)  # 448 is 0.875 * 2^9
    q = (padded * torch.exp2(-e.float())[:, :, None]).to(torch.float8_e4m3fn).float()
    return q.reshape(rows, -1)[:, :cols], e


def _held(v):
    """What 8-bit blocks stand for."""
    q, e = _blocks(v)
    return q * torch.exp2(e.float()).repeat_interleave(32, 1)[:, :v.shape[1]]


# --------------------------------------------------------------------- answers in 64 bits
def exact(case, seed):
    """The definition in 64 bits; gradients are torch's derivative of that definition (8-bit blocks pass them on as
    they come)."""
    if work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    t, act, out = s["x"].dtype, case["activation"], {}
    v = {k: s[k].detach().double() for k in ("x", "w", "weight", "bias", "residual") if s.get(k) is not None}
    leaves = [k for k in v if s[k].requires_grad]
    for k in leaves:
        v[k].requires_grad_(True)
    functions = {"": lambda z: z, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu, "sigmoid": torch.sigmoid}
    x, cotangents = v["x"], []
    if case["op"] == "rms_norm" or case["norm"]:
        if "residual" in v:
            x = x + v.pop("residual")
            x = out["sum"] = x + (x.detach().to(t).double() - x.detach())
        x = x / (x.square().mean(1, keepdim=True) + EPS).sqrt() * v["weight"]
    if case["op"] == "rms_norm":
        out = {"y": x, **out}
    elif case["op"] == "scored":
        out["y"] = functions[act](torch.nn.functional.linear(_stands_for(x), _decoded(s["w"], s["w_scales"]), v["bias"]))
        if "residual" in v:
            out["y"] = out["y"] + v["residual"]
    elif case["op"] == "linear" or not case["train"]:
        out["y"] = functions[act](torch.nn.functional.linear(x, v["w"], v["bias"])) + v.get("residual", 0.0)
    else:
        return _exact_kept(s, v, functions[act], leaves)
    if not case["train"]:
        return {k: u.detach() for k, u in out.items()}
    cotangents = [s["d" + k].double() for k in out]
    inputs = [{**v, "residual": None}.get(k) for k in leaves]
    found = dict(zip([k for k, u in zip(leaves, inputs) if u is not None], torch.autograd.grad(list(out.values()), [u for u in inputs if u is not None], cotangents, retain_graph=True)))
    if "residual" in leaves:
        found["residual"] = found["x"] if case["op"] == "rms_norm" else s["dy"].double()
    return {**{k: u.detach() for k, u in out.items()}, **{"d" + k: found[k] for k in leaves}}


def _exact_kept(s, v, function, leaves):
    """The forward pass as it is, and the gradients at the held x and pre-activations."""
    v = {k: u.detach() for k, u in v.items()}
    z = torch.nn.functional.linear(v["x"], v["w"], v["bias"])
    at, dy = _stands_for(z).requires_grad_(True), s["dy"].double()
    dz, = torch.autograd.grad(function(at), at, dy)
    held = _stands_for(v["x"]).to(s["x"].dtype).double()
    grads = {"x": dz @ v["w"], "w": dz.t() @ held, "bias": dz.sum(0), "residual": dy}
    return {"y": function(z) + v.get("residual", 0.0), **{"d" + k: grads[k] for k in leaves}}


def _decoded(values, codes):
    rows, cols = values.shape
    r, b = torch.arange(rows, device=values.device)[:, None], torch.arange(cols, device=values.device)[None] // 32
    return torch.ldexp(values.double(), codes[r // 128, b // 4, r % 32, r // 32 % 4, b % 4].double() - 127)


def _stands_for(v):
    """8-bit blocks by their definition: the least scale by trial of both candidates, the nearest multiple of an e4m3
    value's step (2^-3 of its power of two, 2^-9 below 2^-6)."""
    rows, cols = v.shape
    b = torch.nn.functional.pad(v.detach(), (0, -cols % 32)).view(rows, -1, 32)
    largest = b.abs().amax(2, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(largest.clamp_min(1e-300))) - 9).clamp_min(2.0 ** -127)
    for _ in range(2):
        scale = torch.where(largest > 448 * scale, 2 * scale, scale)
    u = b / scale
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(u / step) * step * scale).reshape(rows, -1)[:, :cols]
