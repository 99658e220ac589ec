"""The acoustic-model operators whose speed is measured: which calls, at which sizes, on which inputs.

The search reads rows of log-likelihoods.  These operators make them: the
layers of a feed-forward acoustic model (matrix product with bias, activation
and residual; root-mean-square norm with the residual's addition and an 8-bit
output), its training from a teacher's top logits, and the conversion of its
logits to the rows that ``wfst_decode`` reads.

Frames and units are those of ``paper_1808_00687_amd/workloads.py``: batches
of 64 utterances of 300 to 1,500 frames (53,274 together), 64, 80, 2,000 or
6,000 units.  The layers' widths are generic.

With ``own`` false ``run`` computes the plain form in 32 bits; with ``own``
true it calls ``paper_1808_00687_amd/acoustic.py``.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "f8": 1}
E4M3_MAX = 448.0      # largest finite e4m3 value

BATCH_FRAMES = 53274  # frames of the 64-utterance batch
MOST_FLOPS = 4.5e11   # no drawn case costs more than the largest listed ones
MOST_BYTES = 1.9e9


def listed():
    return [
        # one new frame through the output layer: a recogniser that answers frame by frame
        {"name": "linear one frame", "op": "linear", "rows": 1, "inner": 1024, "outer": 6000, "type": "bf16",
         "out": "f32", "activation": "none"},
        # an utterance's spliced features (40 coefficients, 11 frames) into a layer of 2,000, with the residual
        {"name": "linear odd f16", "op": "linear", "rows": 777, "inner": 440, "outer": 2000, "type": "f16",
         "out": "f16", "activation": "silu", "residual": True},
        # the batch through a narrowing layer, the residual stream added
        {"name": "linear batch bf16", "op": "linear", "rows": 16384, "inner": 4096, "outer": 1024, "type": "bf16",
         "out": "bf16", "activation": "none", "residual": True},
        # the whole batch through a widening layer in 8 bits
        {"name": "linear batch f8", "op": "linear", "rows": BATCH_FRAMES, "inner": 1024, "outer": 4096, "type": "f8",
         "out": "bf16", "activation": "gelu"},
        # gradients of a widening layer over the frames of one training batch
        {"name": "linear backward", "op": "linear_backward", "rows": 16384, "inner": 1024, "outer": 4096,
         "type": "bf16", "activation": "silu"},
        # the norm of one new frame, to 8 bits
        {"name": "norm one frame", "op": "norm", "rows": 1, "width": 1024, "type": "bf16", "out": "f8",
         "residual": True},
        # the norm of the whole batch, to 8 bits
        {"name": "norm batch", "op": "norm", "rows": BATCH_FRAMES, "width": 1024, "type": "bf16", "out": "f8",
         "residual": True},
        # the norm's gradients over a training batch
        {"name": "norm backward", "op": "norm_backward", "rows": 16384, "width": 2048, "type": "bf16", "ds": True},
        # gradient of the loss against a small CTC model's units, one utterance
        {"name": "distill utterance", "op": "distill", "rows": 833, "units": 80, "top": 8, "type": "f32",
         "temperature": 2.0},
        # loss and gradient over a training batch of an LVCSR model
        {"name": "distill batch", "op": "distill", "rows": 16384, "units": 6000, "top": 20, "type": "bf16",
         "temperature": 1.0},
        # one utterance's rows for the search, medium unit set
        {"name": "loglikes utterance", "op": "loglikes", "rows": 833, "units": 2000, "type": "f16"},
        # the whole batch's rows for the search
        {"name": "loglikes batch", "op": "loglikes", "rows": BATCH_FRAMES, "units": 6000, "type": "bf16"},
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
    op = rng.choice(["linear", "linear", "linear_backward", "norm", "norm_backward", "distill", "distill_backward",
                     "loglikes"])
    if op in ("linear", "linear_backward"):
        k, n = _width(rng), rng.choice([_width(rng), _width(rng), rng.choice(UNITS)])
        t = rng.choice(["bf16", "f16", "f8"] if op == "linear" else ["bf16", "f16"])
        c = {"op": op, "rows": _rows(rng, 8 * (k + n), (4 if op == "linear_backward" else 2) * k * n), "inner": k,
             "outer": n, "type": t, "activation": rng.choice(["none", "relu", "silu", "gelu"])}
        if op == "linear":
            c["out"] = rng.choice(["f32", t] if t != "f8" else ["bf16", "f16"])
            c["residual"] = rng.random() < 0.4
            c["save_pre"] = rng.random() < 0.3
            c["pad"] = rng.choice([0, 0, 0, 16, 5])
        return c
    t = rng.choice(["bf16", "f16", "f32"])
    if op in ("norm", "norm_backward"):
        d = rng.choice([_width(rng), _width(rng), _log(rng, 16, 20000)])
        c = {"op": op, "rows": _rows(rng, 16 * d), "width": d, "type": t}
        if op == "norm":
            c |= {"out": rng.choice(["f8", "f8", t]), "residual": rng.random() < 0.6}
        else:
            c["ds"] = rng.random() < 0.5
        return c
    n = rng.choice([rng.choice(UNITS), _log(rng, 30, 40000)])
    c = {"op": op, "rows": _rows(rng, 8 * n), "units": n, "type": t}
    if op != "loglikes":
        c |= {"top": min(n, _log(rng, 1, 64)), "temperature": rng.choice([1.0, 2.0, 4.0])}
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _quantise(v):
    """Rows of e4m3 values and their scales."""
    scale = v.abs().amax(1) / E4M3_MAX
    return (v / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device=dev) * std + mean

    op, rows = case["op"], case["rows"]
    dt = DTYPES[case["type"]]
    s = {"case": case}
    if op in ("linear", "linear_backward"):
        k, n = case["inner"], case["outer"]
        # activations after a norm; weights that keep the outputs at unit size
        x, w = normal(rows, k), normal(n, k, std=k ** -0.5)
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
        if op == "linear":
            out = DTYPES[case["out"]]
            s["bias"] = normal(n, std=0.1)
            s["residual"] = normal(rows, n).to(out) if case.get("residual") else None
            s["y"] = torch.empty(rows, n, dtype=out, device=dev)
            s["pre"] = torch.empty(rows, n, dtype=out, device=dev) if case.get("save_pre") else None
        else:
            s["dy"] = normal(rows, n, std=0.01).to(dt)
            s["pre"] = None if case["activation"] == "none" else normal(rows, n).to(dt)
    elif op in ("norm", "norm_backward"):
        d = case["width"]
        s["gain"] = normal(d, std=0.1, mean=1.0)
        if op == "norm":
            s["x"] = normal(rows, d).to(dt)
            s["residual"] = normal(rows, d, std=3.0).to(dt) if case["residual"] else None
        else:
            s["s"] = normal(rows, d, std=3.0).to(dt)
            s["dy"] = normal(rows, d, std=0.01).to(dt)
            s["ds"] = normal(rows, d, std=0.01).to(dt) if case["ds"] else None
    else:
        n = case["units"]
        student = normal(rows, n, std=3.0)
        s["logits"] = student.to(dt)
        if op == "loglikes":
            s["log_prior"] = torch.log_softmax(normal(n), 0)
            s["scale"] = 0.1 + 0.9 * (seed % 7) / 7
            s["ll"] = torch.empty(rows, n, device=dev)
        else:
            # a teacher that mostly agrees; its best units, kept in 16 bits
            teacher = student.add_(normal(rows, n, std=1.5))
            value, index = torch.topk(teacher, case["top"], 1)
            s["top_logit"], s["top_index"] = value.to(torch.float16), index.to(torch.int32)
            s["weight"] = torch.full((rows,), 1.0 / rows, device=dev)
            if op == "distill_backward":
                s["lse"] = torch.logsumexp(s["logits"].float() / case["temperature"], 1)
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
    if op == "linear":
        am.wfst_am_linear(s["x"], s["w"], s["bias"], activation=c["activation"], residual=s["residual"],
                          x_scale=s.get("x_scale"), w_scale=s.get("w_scale"), pre=s["pre"], out=s["y"])
        return {"y": s["y"], "pre": s["pre"]}
    if op == "linear_backward":
        dx, dw, db = am.wfst_am_linear_backward(s["dy"], s["x"], s["w"], activation=c["activation"], pre=s["pre"])
        return {"dx": dx, "dw": dw, "dbias": db}
    if op == "norm":
        y, scale, total = am.wfst_am_norm(s["x"], s["gain"], residual=s["residual"], out_dtype=DTYPES[c["out"]])
        return {"y": y, "scale": scale, "sum": total}
    if op == "norm_backward":
        dx, dg = am.wfst_am_norm_backward(s["dy"], s["s"], s["gain"], dsum=s["ds"])
        return {"dx": dx, "dgain": dg}
    if op == "distill":
        loss, lse, dl = am.wfst_am_distill(s["logits"], s["top_index"], s["top_logit"],
                                           temperature=c["temperature"], weight=s["weight"], gradient=True)
        return {"loss": loss, "lse": lse, "dlogits": dl}
    if op == "distill_backward":
        return {"dlogits": am.wfst_am_distill_backward(s["logits"], s["top_index"], s["top_logit"], s["lse"],
                                                       temperature=c["temperature"], weight=s["weight"])}
    return {"ll": am.wfst_am_loglikes(s["logits"], s["log_prior"], scale=s["scale"], out=s["ll"])}


NORM_EPS = 1e-6   # the operators' default


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
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "linear":
        z = s["x"].float() @ s["w"].float().t()
        if c["type"] == "f8":
            z = z * s["x_scale"][:, None] * s["w_scale"]
        z = z + s["bias"]
        y = _activate(z, c["activation"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(DTYPES[c["out"]]), "pre": z.to(DTYPES[c["out"]]) if s["pre"] is not None else None}
    if op == "linear_backward":
        dz = s["dy"].float()
        if s["pre"] is not None:
            dz = dz * _slope(s["pre"].float(), c["activation"])
        dt = DTYPES[c["type"]]
        return {"dx": (dz @ s["w"].float()).to(dt), "dw": (dz.t() @ s["x"].float()).to(dt), "dbias": dz.sum(0)}
    if op == "norm":
        total = s["x"].float()
        if s["residual"] is not None:
            total = total + s["residual"].float()
        y = total * torch.rsqrt((total * total).mean(1, keepdim=True) + NORM_EPS) * s["gain"]
        kept = total.to(DTYPES[c["type"]]) if s["residual"] is not None else None
        if c["out"] != "f8":
            return {"y": y.to(DTYPES[c["out"]]), "scale": None, "sum": kept}
        scale = y.abs().amax(1) / E4M3_MAX
        q = (y / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        return {"y": q, "scale": scale, "sum": kept}
    if op == "norm_backward":
        x, dy = s["s"].float(), s["dy"].float()
        r = torch.rsqrt((x * x).mean(1, keepdim=True) + NORM_EPS)
        u = dy * s["gain"]
        dx = r * (u - x * (r * r * (u * x).mean(1, keepdim=True)))
        if s["ds"] is not None:
            dx = dx + s["ds"].float()
        return {"dx": dx.to(DTYPES[c["type"]]), "dgain": (dy * x * r).sum(0)}
    if op == "loglikes":
        x = s["logits"].float()
        x = x - x.amax(1, keepdim=True)
        return {"ll": (x - torch.log(torch.exp(x).sum(1, keepdim=True)) - s["log_prior"]) * s["scale"]}
    t, index = c["temperature"], s["top_index"].long()
    x = s["logits"].float() / t
    top = s["top_logit"].float() / t
    log_p = top - torch.logsumexp(top, 1, keepdim=True)
    p = torch.exp(log_p)
    if op == "distill":
        m = x.amax(1)
        lse = m + torch.log(torch.exp(x - m[:, None]).sum(1))
        loss = s["weight"] * t * t * (p * (log_p - (torch.gather(x, 1, index) - lse[:, None]))).sum(1)
    else:
        lse = s["lse"]
    d = torch.exp(x - lse[:, None]).scatter_add_(1, index, -p) * (s["weight"] * t)[:, None]
    d = d.to(DTYPES[c["type"]])
    return {"dlogits": d} if op == "distill_backward" else {"loss": loss, "lse": lse, "dlogits": d}


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    op, m = case["op"], case["rows"]
    b = BYTES[case["type"]]
    if op == "linear":
        k, n, o = case["inner"], case["outer"], BYTES[case["out"]]
        outs = 1 + bool(case.get("residual")) + bool(case.get("save_pre"))
        return {"bytes": (m + n) * k * b + 4 * n + m * n * o * outs + (4 * (m + n) if b == 1 else 0),
                "flops": 2 * m * n * k}
    if op == "linear_backward":
        k, n = case["inner"], case["outer"]
        return {"bytes": b * (2 * (m + n) * k + m * n * (1 + (case["activation"] != "none"))) + 4 * n,
                "flops": 4 * m * n * k}
    if op == "norm":
        d, o = case["width"], BYTES[case["out"]]
        return {"bytes": m * d * (b * (3 if case["residual"] else 1) + o) + 4 * d + (4 * m if o == 1 else 0),
                "flops": 6 * m * d}
    if op == "norm_backward":
        d = case["width"]
        return {"bytes": m * d * b * (4 if case["ds"] else 3) + 8 * d, "flops": 10 * m * d}
    n = case["units"]
    if op == "loglikes":
        return {"bytes": m * n * (b + 4) + 4 * n, "flops": 5 * m * n}
    return {"bytes": 2 * m * n * b + m * case["top"] * 6 + 12 * m, "flops": 6 * m * n}


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
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op == "linear":
        z = torch.matmul(f["x"], f["w"].transpose(0, 1))
        if "x_scale" in f:
            z = z * torch.outer(f["x_scale"], f["w_scale"])
        z += f["bias"]
        kind = case["activation"]
        y = (torch.nn.functional.relu(z) if kind == "relu" else z * torch.sigmoid(z) if kind == "silu" else
             z * torch.special.ndtr(z) if kind == "gelu" else z)
        return {"y": y + f["residual"] if s["residual"] is not None else y, "pre": z if s["pre"] is not None else None}
    if op == "linear_backward":
        dz, kind = f["dy"], case["activation"]
        if kind != "none":
            z = f["pre"]
            if kind == "relu":
                dz = torch.where(z > 0, dz, torch.zeros_like(dz))
            elif kind == "silu":
                sig = torch.sigmoid(z)
                dz = dz * (sig + z * sig * (1 - sig))
            else:
                dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi))
        return {"dx": torch.matmul(dz, f["w"]), "dw": torch.matmul(dz.t(), f["x"]), "dbias": dz.sum(0)}
    if op == "norm":
        a = f["x"] + f["residual"] if "residual" in f else f["x"]
        y = f["gain"] * a / torch.sqrt(a.square().mean(1) + NORM_EPS)[:, None]
        kept = a if "residual" in f else None
        if case["out"] != "f8":
            return {"y": y, "scale": None, "sum": kept}
        scale = y.abs().max(1).values / E4M3_MAX
        return {"y": _e4m3(y / scale[:, None]), "scale": scale, "sum": kept}
    if op == "norm_backward":
        a, dy = f["s"], f["dy"]
        rms = torch.sqrt(a.square().mean(1) + NORM_EPS)[:, None]
        unit = a / rms
        u = dy * f["gain"]
        dx = (u - unit * (u * unit).mean(1)[:, None]) / rms
        return {"dx": dx + f["ds"] if "ds" in f else dx, "dgain": (dy * unit).sum(0)}
    if op == "loglikes":
        return {"ll": s["scale"] * (torch.log_softmax(f["logits"], 1) - f["log_prior"])}
    t = case["temperature"]
    log_q = torch.log_softmax(f["logits"] / t, 1)
    p = torch.softmax(f["top_logit"] / t, 1)
    index = s["top_index"].long()
    d = torch.exp(log_q)
    for j in range(index.shape[1]):   # a unit is at most once among a row's entries
        rows = torch.arange(index.shape[0], device=index.device)
        d[rows, index[:, j]] -= p[:, j]
    d *= t * f["weight"][:, None]
    if op == "distill_backward":
        return {"dlogits": d}
    loss = f["weight"] * t * t * (torch.xlogy(p, p) - p * log_q.gather(1, index)).sum(1)
    return {"loss": loss, "lse": torch.logsumexp(f["logits"] / t, 1), "dlogits": d}
