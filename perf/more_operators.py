"""More operators of the acoustic model whose speed is measured: which calls, at which sizes, on which inputs.

Beside the layers, norm and losses of a feed-forward acoustic model these are
the gated layer (two projections of the same frames, the one's activation times
the other), the layer norm, both with their gradients, and the clipping of a
model's gradients by their norm over all tensors.

Frames and units are those of ``paper_1808_00687_amd/workloads.py``: batches
of 64 utterances of 300 to 1,500 frames (53,274 together), 64, 2,000 or 6,000
units.  The small model whose gradients are clipped is that of
``examples/acoustic_model.py``; the layers' widths are generic.

With ``own`` false ``run`` computes the plain form in 32 bits; with ``own``
true it calls ``paper_1808_00687_amd/acoustic.py``.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "f8": 1}
E4M3_MAX = 448.0       # largest finite e4m3 value
EPS = 1e-5             # the layer norm's default

BATCH_FRAMES = 53274   # frames of the 64-utterance batch
MOST_FLOPS = 2.7e11    # no drawn case costs more than the largest listed one of its operator
MOST_BYTES = 4e8
MOST_CLIP_BYTES = 3.2e9


def listed():
    return [
        # one new frame through a gated layer: a recogniser that answers frame by frame
        {"name": "gated one frame", "op": "gated", "rows": 1, "inner": 1024, "outer": 4096, "type": "bf16",
         "out": "bf16", "activation": "silu"},
        # an utterance's spliced features (40 coefficients, 11 frames) into a gated layer of 1,000
        {"name": "gated odd f16", "op": "gated", "rows": 777, "inner": 440, "outer": 1000, "type": "f16",
         "out": "f16", "activation": "gelu"},
        # a training batch, with what the gradient needs
        {"name": "gated batch bf16", "op": "gated", "rows": 16384, "inner": 1024, "outer": 4096, "type": "bf16",
         "out": "bf16", "activation": "silu", "save_pre": True},
        # the whole batch scored in 8 bits
        {"name": "gated batch f8", "op": "gated", "rows": BATCH_FRAMES, "inner": 1024, "outer": 1280, "type": "f8",
         "out": "bf16", "activation": "silu"},
        # gradients over one utterance: adapting a model to a speaker
        {"name": "gated backward utterance", "op": "gated_backward", "rows": 833, "inner": 512, "outer": 1280,
         "type": "f16", "activation": "gelu"},
        # gradients over a training batch
        {"name": "gated backward batch", "op": "gated_backward", "rows": 16384, "inner": 1024, "outer": 2048,
         "type": "bf16", "activation": "silu"},
        # the norm of one new frame
        {"name": "layer norm one frame", "op": "layer_norm", "rows": 1, "width": 1024, "type": "bf16",
         "out": "bf16", "residual": True},
        # the norm of the whole batch, to 8 bits
        {"name": "layer norm batch", "op": "layer_norm", "rows": BATCH_FRAMES, "width": 1024, "type": "bf16",
         "out": "f8", "residual": True},
        # the norm's gradients in 32 bits over an odd width
        {"name": "layer norm backward odd", "op": "layer_norm_backward", "rows": 833, "width": 1283, "type": "f32",
         "ds": False},
        # the norm's gradients over a training batch
        {"name": "layer norm backward batch", "op": "layer_norm_backward", "rows": 16384, "width": 2048,
         "type": "bf16", "ds": True},
        # the example's model: a few small tensors in two types
        {"name": "clip small model", "op": "clip", "blocks": 2, "width": 128, "features": 40, "units": 64,
         "type": "bf16", "share": 0.5},
        # a large model's gradients, 125 tensors
        {"name": "clip large model", "op": "clip", "blocks": 24, "width": 2048, "features": 440, "units": 6000,
         "type": "bf16", "share": 0.5},
    ]


# --------------------------------------------------------------------------
# drawn cases
# --------------------------------------------------------------------------

# frames of one utterance and of a batch are any number; a layer's width is
# usually a round one
WIDTHS = (64, 128, 256, 320, 512, 640, 1024, 1280, 2048, 2560, 4096)
UNITS = (64, 80, 500, 2000, 6000)


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n if n % 64 else n + 1   # the round sizes come from the lists above


def _width(rng):
    return rng.choice(WIDTHS) if rng.random() < 0.6 else _log(rng, 64, 4096)


def _rows(rng, bytes_per_row, flops_per_row=0):
    most = min(BATCH_FRAMES, MOST_BYTES / bytes_per_row)
    if flops_per_row:
        most = min(most, MOST_FLOPS / flops_per_row)
    return _log(rng, 1, max(1, int(most)))


def draw(rng):
    op = rng.choice(["gated", "gated", "gated_backward", "layer_norm", "layer_norm_backward", "clip"])
    if op in ("gated", "gated_backward"):
        k, n = _width(rng), _width(rng)
        t = rng.choice(["bf16", "f16", "f8"] if op == "gated" else ["bf16", "f16"])
        backward = op == "gated_backward"
        c = {"op": op, "rows": _rows(rng, 4 * k + (14 if backward else 10) * n, (8 if backward else 4) * k * n),
             "inner": k, "outer": n, "type": t, "activation": rng.choice(["none", "relu", "silu", "gelu"])}
        if op == "gated":
            c["out"] = rng.choice(["f32", t] if t != "f8" else ["bf16", "f16"])
            c["save_pre"] = rng.random() < 0.3
            c["pad"] = rng.choice([0, 0, 0, 16, 5])
        return c
    t = rng.choice(["bf16", "f16", "f32"])
    if op == "clip":
        per = 2 * BYTES[t]   # bytes read and written for a weight
        units, features = rng.choice([rng.choice(UNITS), _log(rng, 30, 8000)]), rng.choice([40, 80, 440])
        width = rng.choice(WIDTHS[:9]) if rng.random() < 0.5 else _log(rng, 16, 2048)
        most = int(MOST_CLIP_BYTES / per - (units + features) * width) // (8 * width * width)
        return {"op": "clip", "blocks": _log(rng, 1, max(1, min(32, most))), "width": width, "features": features,
                "units": units, "type": t, "share": rng.choice([0.01, 0.5, 3.0])}
    d = rng.choice([_width(rng), _width(rng), _log(rng, 16, 20000)])
    c = {"op": op, "rows": _rows(rng, 16 * d), "width": d, "type": t}
    if op == "layer_norm":
        c |= {"out": rng.choice(["f8", t, t]), "residual": rng.random() < 0.6}
    else:
        c["ds"] = rng.random() < 0.5
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _quantise(v):
    """Rows of e4m3 values and their scales."""
    scale = v.abs().amax(1) / E4M3_MAX
    return (v / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def _gradient_shapes(c):
    """Shapes and types of a model's parameters: weights in the case's type, biases and gains in 32 bits."""
    d, t = c["width"], c["type"]
    shapes = [((d, c["features"]), t), ((d,), "f32")]
    for _ in range(c["blocks"]):
        shapes += [((4 * d, d), t), ((4 * d,), "f32"), ((d, 4 * d), t), ((d,), "f32"), ((d,), "f32")]
    return shapes + [((c["units"], d), t), ((c["units"],), "f32"), ((d,), "f32")]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device=dev) * std + mean

    op = case["op"]
    dt = DTYPES[case["type"]]
    s = {"case": case}
    if op == "clip":
        s["grads"], count = [], 0
        for shape, t in _gradient_shapes(case):
            s["grads"].append(normal(*shape, std=0.01).to(DTYPES[t]))
            count += math.prod(shape)
        # clipped gradients go into one buffer of each type: what the optimizer, or an exchange with other processes, reads
        s["flat"], s["out"] = {}, []
        for t in dict.fromkeys([case["type"], "f32"]):
            shapes = [shape for shape, u in _gradient_shapes(case) if u == t]
            s["flat"][t] = torch.empty(sum(map(math.prod, shapes)), dtype=DTYPES[t], device=dev)
        at = dict.fromkeys(s["flat"], 0)
        for shape, t in _gradient_shapes(case):
            n = math.prod(shape)
            s["out"].append(s["flat"][t][at[t]:at[t] + n].view(shape))
            at[t] += n
        s["max_norm"] = case["share"] * 0.01 * count ** 0.5 * (0.9 + 0.2 * (seed % 7) / 7)
        return s
    rows = case["rows"]
    if op in ("gated", "gated_backward"):
        k, n = case["inner"], case["outer"]
        # activations after a norm; weights that keep the projections at unit size.  Rows of w: the gate's, then the others
        x, w = normal(rows, k), normal(2 * n, k, std=k ** -0.5)
        if dt == torch.float8_e4m3fn:
            (x, s["x_scale"]), (w, s["w_scale"]) = _quantise(x), _quantise(w)
        else:
            x, w = x.to(dt), w.to(dt)
        pad = case.get("pad", 0)
        if pad:
            wide = torch.zeros(rows, k + pad, dtype=x.dtype, device=dev)
            wide[:, :k] = x
            x = wide[:, :k]
        s["x"], s["w"] = x, w
        if op == "gated":
            out = DTYPES[case["out"]]
            s["bias"] = normal(2 * n, std=0.1)
            s["y"] = torch.empty(rows, n, dtype=out, device=dev)
            s["pre"] = torch.empty(rows, 2 * n, dtype=out, device=dev) if case.get("save_pre") else None
        else:
            s["dy"] = normal(rows, n, std=0.01).to(dt)
            s["pre"] = normal(rows, 2 * n).to(dt)
        return s
    d = case["width"]
    s["gain"] = normal(d, std=0.1, mean=1.0)
    if op == "layer_norm":
        s["bias"] = normal(d, std=0.1)
        s["x"] = normal(rows, d).to(dt)
        s["residual"] = normal(rows, d, std=3.0, mean=0.5).to(dt) if case["residual"] else None
    else:
        s["s"] = normal(rows, d, std=3.0, mean=0.5).to(dt)
        s["dy"] = normal(rows, d, std=0.01).to(dt)
        s["ds"] = normal(rows, d, std=0.01).to(dt) if case["ds"] else None
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    from paper_1808_00687_amd import acoustic as am

    c = s["case"]
    op = c["op"]
    if op == "gated":
        am.wfst_am_gated(s["x"], s["w"], s["bias"], activation=c["activation"], x_scale=s.get("x_scale"),
                         w_scale=s.get("w_scale"), pre=s["pre"], out=s["y"])
        return {"y": s["y"], "pre": s["pre"]}
    if op == "gated_backward":
        dx, dw, db = am.wfst_am_gated_backward(s["dy"], s["pre"], s["x"], s["w"], activation=c["activation"])
        return {"dx": dx, "dw": dw, "dbias": db}
    if op == "layer_norm":
        y, scale, total = am.wfst_am_layer_norm(s["x"], s["gain"], s["bias"], residual=s["residual"],
                                                out_dtype=DTYPES[c["out"]])
        return {"y": y, "scale": scale, "sum": total}
    if op == "layer_norm_backward":
        dx, dg, db = am.wfst_am_layer_norm_backward(s["dy"], s["s"], s["gain"], dsum=s["ds"])
        return {"dx": dx, "dgain": dg, "dbias": db}
    _, norm = am.wfst_am_clip(s["grads"], s["max_norm"], out=s["out"])
    return {"norm": norm, **s["flat"]}


def _activate(z, kind):
    if kind == "relu":
        return torch.clamp(z, min=0)
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "silu":
        e = 1 / (1 + torch.exp(-z))
        return e * (1 + z * (1 - e))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _flat(s, found):
    """The tensors of each type one after the other."""
    return {t: torch.cat([v.reshape(-1) for v, g in zip(found, s["grads"]) if g.dtype == DTYPES[t]]) for t in s["flat"]}


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "gated":
        n, dt = c["outer"], DTYPES[c["out"]]
        z = s["x"].float() @ s["w"].float().t()
        if c["type"] == "f8":
            z = z * s["x_scale"][:, None] * s["w_scale"]
        z = z + s["bias"]
        y = _activate(z[:, :n], c["activation"]) * z[:, n:]
        return {"y": y.to(dt), "pre": z.to(dt) if s["pre"] is not None else None}
    if op == "gated_backward":
        n, dt = c["outer"], DTYPES[c["type"]]
        dy, gate, value = s["dy"].float(), s["pre"][:, :n].float(), s["pre"][:, n:].float()
        dz = torch.cat([dy * value * _slope(gate, c["activation"]), dy * _activate(gate, c["activation"])], 1)
        return {"dx": (dz @ s["w"].float()).to(dt), "dw": (dz.t() @ s["x"].float()).to(dt), "dbias": dz.sum(0)}
    if op == "layer_norm":
        total = s["x"].float()
        if s["residual"] is not None:
            total = total + s["residual"].float()
        mean = total.double().mean(1, keepdim=True)   # a row far from zero loses its differences in 32 bits
        y = (total - mean).float()
        y = y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS) * s["gain"] + s["bias"]
        kept = total.to(DTYPES[c["type"]]) if s["residual"] is not None else None
        if c["out"] != "f8":
            return {"y": y.to(DTYPES[c["out"]]), "scale": None, "sum": kept}
        scale = y.abs().amax(1) / E4M3_MAX
        q = (y / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        return {"y": q, "scale": scale, "sum": kept}
    if op == "layer_norm_backward":
        x, dy = s["s"].float(), s["dy"].float()
        x = (x - x.double().mean(1, keepdim=True)).float()
        r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        x = x * r
        u = dy * s["gain"]
        dx = r * (u - u.mean(1, keepdim=True) - x * (u * x).mean(1, keepdim=True))
        if s["ds"] is not None:
            dx = dx + s["ds"].float()
        return {"dx": dx.to(DTYPES[c["type"]]), "dgain": (dy * x).sum(0), "dbias": dy.sum(0)}
    total = torch.zeros((), dtype=torch.float64, device=s["grads"][0].device)
    for g in s["grads"]:
        total = total + g.double().square().sum()   # a sum over up to a billion values, and a norm next to its limit
    norm = torch.sqrt(total)
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    return {"norm": norm.float().reshape(1), **_flat(s, [(g.float() * scale).to(g.dtype) for g in s["grads"]])}


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    op, b = case["op"], BYTES[case["type"]]
    if op == "clip":
        counts = [(math.prod(shape), BYTES[t]) for shape, t in _gradient_shapes(case)]
        return {"bytes": sum(2 * n * t for n, t in counts), "flops": 3 * sum(n for n, _ in counts)}
    m = case["rows"]
    if op == "gated":
        k, n, o = case["inner"], case["outer"], BYTES[case["out"]]
        outs = 3 if case.get("save_pre") else 1
        return {"bytes": (m + 2 * n) * k * b + 8 * n + m * n * o * outs + (4 * (m + 2 * n) if b == 1 else 0),
                "flops": 4 * m * n * k}
    if op == "gated_backward":
        k, n = case["inner"], case["outer"]
        return {"bytes": b * (2 * (m + 2 * n) * k + 3 * m * n) + 8 * n, "flops": 8 * m * n * k}
    d = case["width"]
    if op == "layer_norm":
        o = BYTES[case["out"]]
        return {"bytes": m * d * (b * (3 if case["residual"] else 1) + o) + 8 * d + (4 * m if o == 1 else 0),
                "flops": 8 * m * d}
    return {"bytes": m * d * b * (4 if case["ds"] else 3) + 12 * d, "flops": 14 * m * d}


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def _e4m3(v):
    """v rounded to the nearest e4m3 value, ties to even: 3 bits after the leading one, spacing 2^-9 below 2^-6."""
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"]))
        factor = min(1.0, s["max_norm"] / norm)
        return {"norm": torch.full((1,), norm, dtype=torch.float64, device="cuda"),
                **_flat(s, [g.double() * factor for g in s["grads"]])}
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op == "gated":
        z = torch.matmul(f["x"], f["w"].transpose(0, 1))
        if "x_scale" in f:
            z = z * torch.outer(f["x_scale"], f["w_scale"])
        z += f["bias"]
        gate, value = z.chunk(2, 1)
        kind = case["activation"]
        a = (torch.nn.functional.relu(gate) if kind == "relu" else gate * torch.sigmoid(gate) if kind == "silu" else
             gate * torch.special.ndtr(gate) if kind == "gelu" else gate)
        return {"y": a * value, "pre": z if s["pre"] is not None else None}
    if op == "gated_backward":
        (gate, value), dy, kind = f["pre"].chunk(2, 1), f["dy"], case["activation"]
        if kind == "relu":
            on = (gate > 0).double()
            a, da = gate * on, on
        elif kind == "silu":
            sig = torch.sigmoid(gate)
            a, da = gate * sig, sig + gate * sig * (1 - sig)
        elif kind == "gelu":
            phi = torch.special.ndtr(gate)
            a, da = gate * phi, phi + gate * torch.exp(-gate.square() / 2) / math.sqrt(2 * math.pi)
        else:
            a, da = gate, torch.ones_like(gate)
        dg, dv = dy * value * da, dy * a
        n = case["outer"]
        return {"dx": torch.matmul(dg, f["w"][:n]) + torch.matmul(dv, f["w"][n:]),
                "dw": torch.cat([torch.matmul(dg.t(), f["x"]), torch.matmul(dv.t(), f["x"])]),
                "dbias": torch.cat([dg.sum(0), dv.sum(0)])}
    if op == "layer_norm":
        a = f["x"] + f["residual"] if "residual" in f else f["x"]
        var, mean = torch.var_mean(a, 1, correction=0, keepdim=True)
        y = f["gain"] * (a - mean) / torch.sqrt(var + EPS) + f["bias"]
        kept = a if "residual" in f else None
        if case["out"] != "f8":
            return {"y": y, "scale": None, "sum": kept}
        scale = y.abs().max(1).values / E4M3_MAX
        return {"y": _e4m3(y / scale[:, None]), "scale": scale, "sum": kept}
    a, dy = f["s"], f["dy"]
    var, mean = torch.var_mean(a, 1, correction=0, keepdim=True)
    std = torch.sqrt(var + EPS)
    unit = (a - mean) / std
    u = dy * f["gain"]
    dx = (u - u.mean(1)[:, None] - unit * (u * unit).mean(1)[:, None]) / std
    return {"dx": dx + f["ds"] if "ds" in f else dx, "dgain": (dy * unit).sum(0), "dbias": dy.sum(0)}
