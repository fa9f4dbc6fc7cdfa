"""What layers whose activations are held in 8 bits cost a training program, and group norm: rows of int8 with an exponent each
(a token's activations, a pixel's channels, an output channel of a weight) written and read back, the linear layer on two such
operands forward and backward, and group norm with an activation on channels-last maps, forward (leaving its input in 8 bits if asked)
and backward (from the 8 bits or from the input itself), each through the calls of include/ppll.h, beside its plain form in torch.

A row of 8 bits is q 2^e: e the least integer in -126 .. 121 with max|x| <= 127 2^e, q = x 2^-e rounded to the nearest (ties to even).

A case is a flat dict; "op" names the entry point.  listed() holds the cases to look at, draw() gives more of the same ranges, prepare()
makes what a program has in hand before the call, run() is one call, exact() the same from the definition in 64 bits, work() what the
call cannot do without.
"""
import math

import torch

own = False
DEV = "cuda"
CHECKPOINT, FORWARD, BACKWARD = "checkpoint", "linear forward", "linear backward"
NORM, NORM_BACKWARD = "group norm forward", "group norm backward"
EPS = 1e-5
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
LEAST, MOST = -126, 121                   # exponents of a row


def _checkpoint(name, rows, cols, dtype):
    return {"name": name, "op": CHECKPOINT, "rows": rows, "cols": cols, "dtype": dtype}


def _linear(name, op, rows, n_in, n_out, dtype, gelu=False, extra=False):
    """extra: a residual that the forward adds, a slope that the input gradient is multiplied by."""
    return {"name": name, "op": op, "rows": rows, "in": n_in, "out": n_out, "dtype": dtype, "gelu": gelu, "extra": extra}


def _norm(name, op, images, height, width, channels, groups, dtype, act, residual=False, kept=False):
    return {"name": name, "op": op, "images": images, "height": height, "width": width, "channels": channels, "groups": groups, "dtype": dtype,
            "act": act, "residual": residual, "kept": kept}


def listed():
    return [
        # the smallest: layer inputs of the narrow fp32 block that an installation is checked with, 8 images of 65 tokens of width 64
        _checkpoint("checkpoint tiny", 520, 64, "fp32"),
        # inputs of the second MLP layer of an ordinary stage twice as wide as usual: 128 images of 197 tokens
        _checkpoint("checkpoint large", 25216, 1536, "bf16"),
        # one token at a time through the first MLP layer of a trained stage: latency, and the weight's bytes
        _linear("linear one token", FORWARD, 1, 384, 1536, "bf16", gelu=True),
        # first MLP layer of an ordinary stage: 128 images of 65 tokens, GELU and its slope
        _linear("linear stage", FORWARD, 8320, 384, 1536, "bf16", gelu=True),
        # sizes that are a multiple of nothing
        _linear("linear ragged", FORWARD, 1003, 333, 517, "fp32", extra=True),
        # the largest: second MLP layer at the widest block there may be
        _linear("linear wide", FORWARD, 25216, 6144, 1536, "bf16", extra=True),
        # gradients of the second MLP layer of the stage, multiplied by the slope of the GELU in front of it
        _linear("linear stage backward", BACKWARD, 8320, 1536, 384, "bf16", extra=True),
        # gradients of an odd layer
        _linear("linear ragged backward", BACKWARD, 777, 201, 333, "bf16"),
        # a norm of the first stage of ResNet-32 in front of a shortcut's end
        _norm("norm stage", NORM, 128, 32, 32, 16, 4, "bf16", "relu", residual=True),
        # wide maps of large images, input kept in 8 bits
        _norm("norm large", NORM, 16, 96, 96, 256, 32, "bf16", "silu", kept=True),
        # gradients of the norm of the stage from its input in 8 bits
        _norm("norm stage backward", NORM_BACKWARD, 128, 32, 32, 16, 4, "bf16", "relu", residual=True, kept=True),
        # gradients over the wide maps from the input itself
        _norm("norm large backward", NORM_BACKWARD, 16, 96, 96, 256, 32, "bf16", "silu"),
    ]


LARGEST_FLOPS = 4.7e11        # of a layer, and
LARGEST_ELEMENTS = 3.8e7      # of a map or a checkpoint: a little under the largest listed ones


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice((CHECKPOINT, FORWARD, FORWARD, BACKWARD, BACKWARD, NORM, NORM_BACKWARD))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    while True:
        if op == CHECKPOINT:
            c = _checkpoint("", _log(rng, 1, 65536), _log(rng, 8, 6144), dtype)
            small = c["rows"] * c["cols"] <= LARGEST_ELEMENTS
        elif op in (FORWARD, BACKWARD):
            c = _linear("", op, _log(rng, 1, 32768), _log(rng, 16, 6144), _log(rng, 16, 6144), dtype, gelu=op == FORWARD and rng.random() < 0.4,
                        extra=rng.random() < 0.5)
            flops = (2.0 if op == FORWARD else 4.0) * c["rows"] * c["in"] * c["out"]
            small = flops * (8 if dtype == "fp32" else 1) <= LARGEST_FLOPS
        else:
            groups = rng.choice((1, 2, 4, 8, 8, 16, 32))
            act = rng.choice(("none", "relu", "relu", "silu", "gelu"))
            c = _norm("", op, _log(rng, 1, 512), _log(rng, 1, 128), _log(rng, 1, 128), groups * _log(rng, 1, 512 // groups), groups, dtype, act,
                      residual=rng.random() < 0.5, kept=rng.random() < 0.5)
            small = _pixels(c) * c["channels"] <= LARGEST_ELEMENTS
            small = small and c["height"] * c["width"] * c["channels"] // groups > 4         # statistics of something
        if small:
            del c["name"]
            return c


def _pixels(c):
    return c["images"] * c["height"] * c["width"]


def work(case):
    c, s = case, DTYPES[case["dtype"]].itemsize
    if c["op"] == CHECKPOINT:
        e = c["rows"] * c["cols"]
        return {"bytes": float(2 * (e * (s + 1) + c["rows"])), "flops": float(4 * e)}
    if c["op"] == FORWARD:
        m, k, n = c["rows"], c["in"], c["out"]
        out = m * n * s * (1 + c["gelu"] + c["extra"])
        return {"bytes": float(m * k * s + n * k + n * 5 + out), "flops": 2.0 * m * k * n}
    if c["op"] == BACKWARD:
        m, k, n = c["rows"], c["in"], c["out"]
        return {"bytes": float(m * k + m + n * k + n + m * n * s + m * k * s * (1 + c["extra"]) + (k + 1) * n * 4), "flops": 4.0 * m * k * n}
    e = _pixels(c) * c["channels"]
    if c["op"] == NORM:
        # the kept input is written, and read back to be looked at
        return {"bytes": float(e * (s * (2 + c["residual"]) + (2 + s) * c["kept"])), "flops": float(10 * e)}
    read = (1 if c["kept"] else s) + s + s * _reads_y(c) + s * _reads_residual(c)
    return {"bytes": float(e * (read + s + s * c["residual"])), "flops": float(20 * e)}


def _reads_y(c):
    return c["act"] == "relu"


def _reads_residual(c):
    return c["residual"] and c["act"] in ("silu", "gelu")


# ------------------------------------------------------------------ rows of 8 bits
def _pow2(e):
    """2^e in 32 bits, exact."""
    return torch.ldexp(torch.ones((), device=DEV), e.to(torch.int32))


def _pack(x):
    """x [rows, cols] -> whole numbers [rows, cols] as floats, exponents [rows]."""
    x = x.float()
    fraction, exponent = torch.frexp(x.abs().amax(1))              # max|x| = fraction 2^exponent, 1/2 <= fraction < 1
    e = torch.where(fraction <= 127 / 128, exponent - 7, exponent - 6)
    e = torch.where(fraction > 0, e, LEAST).clamp(LEAST, MOST)
    return (x * _pow2(-e)[:, None]).round().clamp(-127, 127), e


def _as_bytes(q, e):
    """The format in memory: rows a multiple of 16 bytes apart, zeros behind the last column."""
    rows, cols = q.shape
    out = torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=DEV)
    out[:, :cols] = q.to(torch.int8)
    return out, e.to(torch.int8)


# ------------------------------------------------------------------ inputs
def _activations(rows, cols, gen):
    """Activations of a layer: tokens and channels of different size."""
    x = torch.randn((rows, cols), generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device=DEV))
    return x * torch.exp(0.3 * torch.randn((1, cols), generator=gen, device=DEV))


def _group_view(c, x):
    return x.reshape(c["images"], c["height"] * c["width"], c["groups"], c["channels"] // c["groups"])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    c, dtype, s = case, DTYPES[case["dtype"]], {"case": case}
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEV)  # noqa: E731
    if c["op"] == CHECKPOINT:
        s["x"] = _activations(c["rows"], c["cols"], gen).to(dtype)
        return s
    if c["op"] in (FORWARD, BACKWARD):
        m, k, n = c["rows"], c["in"], c["out"]
        x = _activations(m, k, gen)
        s["w"], s["w_exp"] = _as_bytes(*_pack(normal(n, k) / math.sqrt(k)))          # a trained layer's weight: a row for each output channel
        if c["op"] == FORWARD:
            s["x"], s["bias"] = x.to(dtype), 0.1 * normal(n)
            s["residual"] = normal(m, n).to(dtype) if c["extra"] else None
        else:
            s["x"], s["x_exp"] = _as_bytes(*_pack(x.to(dtype)))
            s["dy"] = (1e-3 * normal(m, n) * torch.exp(0.5 * normal(m, 1))).to(dtype)
            s["gate"] = torch.rand((m, k), generator=gen, device=DEV).to(dtype) if c["extra"] else None
        return s
    p, ch = _pixels(c), c["channels"]
    x = (normal(p, ch) * torch.exp(0.3 * normal(1, ch)) + 0.5 * normal(1, ch)).to(dtype)
    s["scale"], s["shift"] = 1 + 0.1 * normal(ch), 0.1 * normal(ch)
    s["residual"] = normal(p, ch).to(dtype) if c["residual"] else None
    if c["op"] == NORM:
        s["x"] = x
        return s
    y, s["stats"] = _norm_plain(c, x, s["scale"], s["shift"], s["residual"])
    s["y"] = y.to(dtype) if _reads_y(c) else None
    if not _reads_residual(c):
        s["residual"] = None
    s["dy"] = (1e-3 * normal(p, ch)).to(dtype)
    if c["kept"]:
        s["x"], s["x_exp"] = _as_bytes(*_pack(x))
    else:
        s["x"] = x
    return s


# ------------------------------------------------------------------ plain forms
def _activated(c, z):
    if c["act"] == "relu":
        return z.clamp(min=0)
    if c["act"] == "silu":
        return z * torch.sigmoid(z)
    return _gelu(z)[0] if c["act"] == "gelu" else z


def _gelu(h):
    """GELU and its derivative."""
    cdf = 0.5 * (1 + torch.erf(h * 0.7071067811865476))
    return h * cdf, cdf + h * torch.exp(-0.5 * h * h) * 0.3989422804014327


def _slope(c, z):
    if c["act"] == "silu":
        sig = torch.sigmoid(z)
        return sig * (1 + z * (1 - sig))
    return _gelu(z)[1]


def _norm_plain(c, x, scale, shift, residual):
    """y in 32 bits, and mean and 1 / deviation [images, groups, 2]."""
    v = _group_view(c, x.float())
    mean = v.mean((1, 3), keepdim=True)
    r = torch.rsqrt((v - mean).square().mean((1, 3), keepdim=True) + EPS)
    z = ((v - mean) * r).reshape(x.shape) * scale + shift
    if residual is not None:
        z = z + residual.float()
    return _activated(c, z), torch.stack([mean, r], -1).view(c["images"], c["groups"], 2)


def _linear_forward(s):
    c, dtype = s["case"], s["x"].dtype
    q, e = _pack(s["x"])
    h = q @ s["w"][:, :c["in"]].float().t()
    h = h * _pow2(e)[:, None] * _pow2(s["w_exp"]) + s["bias"]
    if c["extra"]:
        h = h + s["residual"].float()
    if not c["gelu"]:
        return {"y": h.to(dtype)}
    y, slope = _gelu(h)
    return {"y": y.to(dtype), "slope": slope.to(dtype)}


def _linear_backward(s):
    c, dtype, k = s["case"], s["dy"].dtype, s["case"]["in"]
    dy = s["dy"].float()
    dx = dy @ (s["w"][:, :k].float() * _pow2(s["w_exp"])[:, None])
    if c["extra"]:
        dx = dx * s["gate"].float()
    dw = (s["x"][:, :k].float() * _pow2(s["x_exp"])[:, None]).t() @ dy
    return {"dx": dx.to(dtype), "dw": dw, "db": dy.sum(0)}


def _norm_backward(s):
    c, dtype, ch = s["case"], s["dy"].dtype, s["case"]["channels"]
    x = s["x"][:, :ch].float()
    if c["kept"]:
        x = x * _pow2(s["x_exp"])[:, None]
    mean, r = (v[:, None, :, None] for v in s["stats"].unbind(-1))
    xhat = ((_group_view(c, x) - mean) * r).reshape(x.shape)
    dz = s["dy"].float()
    if c["act"] == "relu":
        dz = torch.where(s["y"] > 0, dz, 0)
    elif c["act"] != "none":
        z = xhat * s["scale"] + s["shift"]
        dz = dz * _slope(c, z if s["residual"] is None else z + s["residual"].float())
    g, v = _group_view(c, dz * s["scale"]), _group_view(c, xhat)
    dx = r * (g - g.mean((1, 3), keepdim=True) - v * (g * v).mean((1, 3), keepdim=True))
    out = {"dx": dx.reshape(x.shape).to(dtype), "d_scale": (dz * xhat).sum(0), "d_shift": dz.sum(0)}
    return {**out, "d_residual": dz.to(dtype)} if c["residual"] else out


def _run_plain(s):
    c = s["case"]
    if c["op"] == CHECKPOINT:
        q, e = _pack(s["x"])
        return (q * _pow2(e)[:, None]).to(s["x"].dtype)
    if c["op"] == FORWARD:
        return _linear_forward(s)
    if c["op"] == BACKWARD:
        return _linear_backward(s)
    if c["op"] == NORM_BACKWARD:
        return _norm_backward(s)
    y, stats = _norm_plain(c, s["x"], s["scale"], s["shift"], s["residual"])
    out = {"y": y.to(s["x"].dtype), "stats": stats}
    if c["kept"]:
        q, e = _pack(s["x"])
        out["kept"] = (q * _pow2(e)[:, None]).to(s["x"].dtype)
    return out


# ------------------------------------------------------------------ this library's calls
def _new_byte_rows(P, rows, cols):
    q = torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=DEV)
    e = torch.empty(rows, dtype=torch.int8, device=DEV)
    return q, e, P.byte_rows(q, e)


def _workspace(nbytes):
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=DEV)


def _run_own(s):
    from paper_2411_12780_amd import binding as P
    c, stream = s["case"], torch.cuda.current_stream().cuda_stream
    dtype, precision = DTYPES[c["dtype"]], P.BF16 if c["dtype"] == "bf16" else P.FP32
    new = lambda *shape: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    rows = lambda t: None if t is None else P.rows(t)  # noqa: E731
    if c["op"] == CHECKPOINT:
        q, e, x8 = _new_byte_rows(P, c["rows"], c["cols"])
        P.ppll_byte_rows_pack(precision, c["rows"], c["cols"], rows(s["x"]), x8, stream)
        out = new(c["rows"], c["cols"])
        P.ppll_byte_rows_unpack(precision, c["rows"], c["cols"], x8, rows(out), stream)
        return out
    if c["op"] in (FORWARD, BACKWARD):
        m, k, n = c["rows"], c["in"], c["out"]
        cfg = P.byte_linear_config(precision=precision, rows=m, in_dim=k, out_dim=n, activation=P.ACT_GELU if c["gelu"] else P.ACT_NONE)
        w8 = P.byte_rows(s["w"], s["w_exp"])
        if c["op"] == FORWARD:
            q, e, x8 = _new_byte_rows(P, m, k)
            P.ppll_byte_rows_pack(precision, m, k, rows(s["x"]), x8, stream)
            y, slope = new(m, n), new(m, n) if c["gelu"] else None
            P.ppll_byte_linear_forward(cfg, x8, w8, s["bias"], rows(s["residual"]), rows(y), rows(slope), stream)
            return {"y": y, "slope": slope} if c["gelu"] else {"y": y}
        dx, dw, db = new(m, k), torch.empty(k, n, device=DEV), torch.empty(n, device=DEV)
        ws = _workspace(P.ppll_byte_linear_workspace_bytes(cfg))
        P.ppll_byte_linear_backward(cfg, P.byte_rows(s["x"], s["x_exp"]), w8, rows(s["dy"]), rows(s["gate"]), rows(dx), dw, db, ws, ws.numel(), stream)
        return {"dx": dx, "dw": dw, "db": db}
    p, ch = _pixels(c), c["channels"]
    act = {"none": P.ACT_NONE, "relu": P.ACT_RELU, "silu": P.ACT_SILU, "gelu": P.ACT_GELU}[c["act"]]
    cfg = P.group_norm_config(precision=precision, images=c["images"], pixels=c["height"] * c["width"], channels=ch, groups=c["groups"],
                              activation=act, eps=EPS)
    ws = _workspace(P.ppll_group_norm_workspace_bytes(cfg))
    if c["op"] == NORM:
        y, stats = new(p, ch), torch.empty(c["images"], c["groups"], 2, device=DEV)
        q, e, x8 = _new_byte_rows(P, p, ch) if c["kept"] else (None, None, None)
        P.ppll_group_norm_forward(cfg, rows(s["x"]), s["scale"], s["shift"], rows(s["residual"]), rows(y), stats, x8, ws, ws.numel(), stream)
        out = {"y": y, "stats": stats}
        if c["kept"]:
            out["kept"] = new(p, ch)
            P.ppll_byte_rows_unpack(precision, p, ch, x8, rows(out["kept"]), stream)
        return out
    dx, dres = new(p, ch), new(p, ch) if c["residual"] else None
    d_scale, d_shift = torch.empty(ch, device=DEV), torch.empty(ch, device=DEV)
    x, x8 = (None, P.byte_rows(s["x"], s["x_exp"])) if c["kept"] else (rows(s["x"]), None)
    P.ppll_group_norm_backward(cfg, x, x8, s["stats"], s["scale"], s["shift"], rows(s["residual"]), rows(s["y"]), rows(s["dy"]), rows(dx),
                               rows(dres), d_scale, d_shift, ws, ws.numel(), stream)
    out = {"dx": dx, "d_scale": d_scale, "d_shift": d_shift}
    return {**out, "d_residual": dres} if c["residual"] else out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_byte_rows(x):
    """The values that x's rows stand for in 8 bits."""
    x = x.double()
    most = x.abs().max(1).values
    e = torch.arange(LEAST, MOST + 1, dtype=torch.float64, device=x.device)
    fits = most[:, None] <= 127 * torch.exp2(e)                    # the least exponent that fits is the one behind all that do not
    step = torch.exp2(e[(~fits).sum(1).clamp(max=len(e) - 1)])[:, None]
    return torch.round(x / step).clamp(-127, 127) * step


def _exact_values(s, q, e):
    """What rows in memory stand for."""
    return q.double() * torch.exp2(e.double())[:, None]


def _exact_act(name, z):
    """An activation and its slope."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        t = 1 / (1 + torch.exp(-z))
        return z * t, t + z * t * (1 - t)
    if name == "gelu":
        below = torch.special.ndtr(z)
        return z * below, below + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.relu(z), (z > 0).double()


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == CHECKPOINT:
        return _exact_byte_rows(s["x"])
    if c["op"] == FORWARD:
        h = torch.matmul(_exact_byte_rows(s["x"]), _exact_values(s, s["w"], s["w_exp"])[:, :c["in"]].t().contiguous()) + s["bias"].double()
        if c["extra"]:
            h += s["residual"].double()
        y, slope = _exact_act("gelu" if c["gelu"] else "none", h)
        return {"y": y, "slope": slope} if c["gelu"] else {"y": y}
    if c["op"] == BACKWARD:
        dy, x, w = s["dy"].double(), _exact_values(s, s["x"], s["x_exp"])[:, :c["in"]], _exact_values(s, s["w"], s["w_exp"])[:, :c["in"]]
        dx = torch.matmul(dy, w.contiguous())
        return {"dx": dx * s["gate"].double() if c["extra"] else dx, "dw": torch.matmul(x.t().contiguous(), dy), "db": dy.sum(0)}
    ch, per = c["channels"], c["channels"] // c["groups"]
    shape = (c["images"], -1, ch)
    spread = lambda v: v.repeat_interleave(per, -1).unsqueeze(1)  # noqa: E731     [images, groups] -> [images, 1, channels]
    if c["op"] == NORM:
        x = s["x"].double().view(shape)
        count = x.shape[1] * per
        mean = x.sum(1).view(-1, c["groups"], per).sum(2) / count
        var = (x - spread(mean)).pow(2).sum(1).view(-1, c["groups"], per).sum(2) / count
        r = 1 / torch.sqrt(var + EPS)
        z = (x - spread(mean)) * spread(r) * s["scale"].double() + s["shift"].double()
        z = z.view(-1, ch) if s["residual"] is None else z.view(-1, ch) + s["residual"].double()
        out = {"y": _exact_act(c["act"], z)[0], "stats": torch.stack([mean, r], 2)}
        return {**out, "kept": _exact_byte_rows(s["x"])} if c["kept"] else out
    x = (_exact_values(s, s["x"], s["x_exp"])[:, :ch] if c["kept"] else s["x"].double()).reshape(shape)
    mean, r = s["stats"].double().unbind(2)
    xhat, dz = (x - spread(mean)) * spread(r), s["dy"].double().view(shape)
    if c["act"] == "relu":
        dz = dz * (s["y"] > 0).double().view(shape)
    else:
        z = xhat * s["scale"].double() + s["shift"].double()
        dz = dz * _exact_act(c["act"], z if s["residual"] is None else z + s["residual"].double().view(shape))[1]
    g, count = dz * s["scale"].double(), x.shape[1] * per
    by_group = lambda v: spread(v.sum(1).view(-1, c["groups"], per).sum(2) / count)  # noqa: E731
    dx = (g - by_group(g) - xhat * by_group(g * xhat)) * spread(r)
    out = {"dx": dx.reshape(-1, ch), "d_scale": (dz * xhat).sum((0, 1)), "d_shift": dz.sum((0, 1))}
    return {**out, "d_residual": dz.reshape(-1, ch)} if c["residual"] else out
