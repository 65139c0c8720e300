"""Work of the feed-forward operators, as measurable cases: what a block of a gated residual network is made of.

  rms_norm        adds a residual, normalises the rows by their root mean square, and gives them as 8-bit integers with a
                  scale for each row, or as numbers
  rms_norm_train  the same in numbers, and its gradients
  quantize        rows of activations as 8-bit integers with a scale for each row
  linear_i8       the product of 8-bit activations with 8-bit weights, a scale for each row and each output channel
  gated           act(x W_gate^T) * (x W_up^T), on 16-bit numbers or on 8-bit integers with scales
  gated_train     the same on 16-bit numbers, and its gradients

`own` false: plain torch operations; true: the library's operators (paper_2505_03983_amd.operators).
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1}


def _norm(name, rows, width, dtype="bf16", out="i8", residual=True, gap=0, op="rms_norm"):
    return dict(name=name, op=op, rows=rows, width=width, dtype=dtype, out=out, residual=residual, gap=gap)


def _quantize(name, rows, width, dtype="bf16", gap=0):
    return dict(name=name, op="quantize", rows=rows, width=width, dtype=dtype, gap=gap)


def _linear(name, rows, width, channels, out="bf16", bias=False, gap=0):
    return dict(name=name, op="linear_i8", rows=rows, width=width, channels=channels, out=out, bias=bias, gap=gap)


def _gated(name, rows, width, channels, dtype="bf16", act="silu", gap=0, op="gated", out="bf16"):
    return dict(name=name, op=op, rows=rows, width=width, channels=channels, dtype=dtype, act=act, gap=gap,
                out=out if dtype == "i8" else dtype)


def listed():
    return [
        # one chain, one step: the norm in front of a block, where nothing but latency counts
        _norm("norm_one_row", 1, 1024),
        # a verify call of an image-shaped network, its residual stream in fp32
        _norm("norm_verify_call", 1984, 4096, dtype="f32"),
        # a long batch of rows
        _norm("norm_batch", 16384, 8192),
        # a training step's norm, at sizes that are no tile's multiple
        _norm("norm_train", 8191, 4104, out="bf16", op="rms_norm_train"),
        # hidden activations of a few chains, ahead of the second product of a block
        _quantize("quantize_few", 24, 8192),
        _quantize("quantize_batch", 8192, 16384),
        # one row against a matrix: a stream of its weights
        _linear("linear_one_row", 1, 4096, 4096),
        # odd sizes throughout: rows that start at no multiple of 16 bytes
        _linear("linear_odd", 999, 2001, 3999, out="f16", bias=True),
        # a large batch
        _linear("linear_batch", 8192, 8192, 8192),
        # one row through 8-bit weights
        _gated("gated_one_row", 1, 4096, 8192, dtype="i8"),
        # a verify call of an image-shaped network
        _gated("gated_verify_call", 1984, 4096, 8192),
        # a training step
        _gated("gated_train", 8192, 4096, 16384, op="gated_train"),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    largest = {}
    for c in listed():
        largest[c["op"]] = max(largest.get(c["op"], 0.0), _cost(c))
    while True:
        op = rng.choice(["rms_norm", "rms_norm", "rms_norm_train", "quantize", "linear_i8", "linear_i8", "linear_i8", "gated",
                         "gated", "gated_train"])
        step = rng.choice([1, 8, 64, 256])   # odd sizes, ones that keep rows on 16 bytes, whole tiles
        rows = _log_int(rng, 1, 16384)
        width = _log_int(rng, max(64, step), 16384, step)
        gap = rng.choice([0, 0, 0, 8, 256, 3])   # elements between the rows of the activations
        if op == "quantize":
            c = _quantize("", rows, width, rng.choice(["bf16", "f16", "f32"]), gap)
        elif op in ("rms_norm", "rms_norm_train"):
            dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
            out = dtype if op == "rms_norm_train" else rng.choice(["i8", "i8", dtype, "bf16"])
            c = _norm("", rows, width, dtype, out, rng.random() < 0.7, gap, op)
        else:
            channels = _log_int(rng, max(64, step), 16384, step)
            if op == "linear_i8":
                c = _linear("", rows, width, channels, rng.choice(["bf16", "f16", "f32"]), rng.random() < 0.5, gap)
            else:
                dtype = rng.choice(["bf16", "bf16", "f16", "i8"] if op == "gated" else ["bf16", "f16"])
                c = _gated("", rows, width, channels, dtype, rng.choice(["silu", "silu", "gelu"]), gap, op,
                           rng.choice(["bf16", "f16"]))
        del c["name"]
        if _cost(c) <= largest[op] and _bytes_held(c) < 3e9:
            return c


def _weights(g, channels, width):
    return torch.randn(channels, width, generator=g, device=DEV) / math.sqrt(width)


def _activations(g, rows, width, gap=0, dtype=torch.float32, quiet=False):
    """Rows of about unit size, some coordinates several times larger than the rest, as a network's are."""
    x = torch.randn(rows, width, generator=g, device=DEV)
    if not quiet:
        x *= 1.0 + 7.0 * (torch.rand(width, generator=g, device=DEV) < 0.01).float()
    return _apart(x.to(dtype), gap)


def _apart(x, gap):
    """The same rows, `gap` elements between them."""
    if not gap:
        return x
    held = torch.zeros(x.shape[0], x.shape[1] + gap, dtype=x.dtype, device=DEV)
    held[:, : x.shape[1]] = x
    return held[:, : x.shape[1]]


def _as_i8(x):
    """Rows as 8-bit integers, and their scales."""
    amax = x.abs().amax(1, keepdim=True)
    return torch.round(x * (127.0 / amax)).to(torch.int8), (amax / 127.0).reshape(-1).contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op, rows, width, gap = case["op"], case["rows"], case["width"], case["gap"]
    s = dict(case)
    if op in ("rms_norm", "rms_norm_train", "quantize"):
        t = TYPES[case["dtype"]]
        s["x"] = _activations(g, rows, width, gap, t)
        if op == "quantize":
            return s
        s["gain"] = (1.0 + 0.1 * torch.randn(width, generator=g, device=DEV)).to(t)
        s["res"] = _activations(g, rows, width, gap, t, True) if case["residual"] else None
        if op == "rms_norm_train":
            s["dy"] = _activations(g, rows, width, gap, t, True)
            s["dsum"] = _activations(g, rows, width, 0, t, True) if case["residual"] else None
        return s
    channels = case["channels"]
    x = _activations(g, rows, width)
    if op == "linear_i8":
        s["x"], s["xs"] = _as_i8(x)
        s["w"], s["ws"] = _as_i8(_weights(g, channels, width))
        s["x"] = _apart(s["x"], gap)
        s["bias"] = torch.randn(channels, generator=g, device=DEV) if case["bias"] else None
        return s
    wg, wu = _weights(g, channels, width), _weights(g, channels, width)
    if case["dtype"] == "i8":
        s["x"], s["xs"] = _as_i8(x)
        s["x"] = _apart(s["x"], gap)
        (s["wg"], s["gs"]), (s["wu"], s["us"]) = _as_i8(wg), _as_i8(wu)
        return s
    t = TYPES[case["dtype"]]
    s["x"], s["wg"], s["wu"] = _apart(x.to(t), gap), wg.to(t), wu.to(t)
    if op == "gated_train":
        s["dh"] = _activations(g, rows, channels, 0, t, True)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2505_03983_amd import operators as O
    op = s["op"]
    if op == "rms_norm":
        out, scale, total = O.rms_norm(s["x"], s["gain"], EPS, residual=s["res"],
                                       out_type=torch.int8 if s["out"] == "i8" else TYPES[s["out"]])
        y = out if scale is None else out * scale[:, None]
        return {"y": y} if total is None else {"y": y, "sum": total}
    if op == "rms_norm_train":
        y, _, total = O.rms_norm(s["x"], s["gain"], EPS, residual=s["res"])
        dx, dgain = O.rms_norm_backward(s["dy"], s["x"] if total is None else total, s["gain"], EPS, dsum=s["dsum"])
        return {"y": y, "dx": dx, "dgain": dgain}
    if op == "quantize":
        q, scale = O.quantize_rows(s["x"])
        return q * scale[:, None]
    if op == "linear_i8":
        return O.linear_i8(s["x"], s["xs"], s["w"], s["ws"], bias=s["bias"], out_type=TYPES[s["out"]])
    if s["dtype"] == "i8":
        return O.gated_ff(s["x"], s["wg"], s["wu"], s["act"], x_scale=s["xs"], gate_scale=s["gs"], up_scale=s["us"],
                          out_type=TYPES[s["out"]])
    h = O.gated_ff(s["x"], s["wg"], s["wu"], s["act"])
    if op == "gated":
        return h
    dx, dwg, dwu = O.gated_ff_backward(s["dh"], s["x"], s["wg"], s["wu"], s["act"])
    return {"h": h, "dx": dx, "dw_gate": dwg, "dw_up": dwu}


def _round_rows(v):
    """127 v / max |v| of each row to the nearest integer, ties to even (v in 64 bits: a value next to a border), and the
    row's largest magnitude."""
    top = v.abs().amax(1, keepdim=True)
    return torch.round(127.0 * v / top), top


def _act(z, kind):
    """The activation and its derivative."""
    if kind == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        return z * sig, sig * (1.0 + z * (1.0 - sig))
    c = math.sqrt(2.0 / math.pi)
    t = 1.0 - 2.0 / (1.0 + torch.exp(2.0 * c * (z + 0.044715 * z * z * z)))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)


def _run_plain(s):
    op = s["op"]
    if op == "quantize":
        q, top = _round_rows(s["x"].double())
        return q.float() * (top / 127.0).float()
    if op in ("rms_norm", "rms_norm_train"):
        t = s["x"].dtype
        r = s["x"].float()
        if s["res"] is not None:
            r = r + s["res"].float()
        gain = s["gain"].float()
        rstd = 1.0 / torch.sqrt(r.double().square().mean(1, keepdim=True) + EPS)
        if s["out"] == "i8":
            q, top = _round_rows(r.double() * gain.double())
            y = q.float() * (top * rstd / 127.0).float()
        else:
            y = (r * rstd.float() * gain).to(TYPES[s["out"]])
        if op == "rms_norm":
            return {"y": y, "sum": r.to(t)} if s["res"] is not None else {"y": y}
        # the gradient is the formula's at the sum as it is stored
        r = r.to(t).float()
        rstd = (1.0 / torch.sqrt(r.double().square().mean(1, keepdim=True) + EPS)).float()
        gy = s["dy"].float() * gain
        n = r * rstd
        dx = rstd * (gy - n * (gy * n).mean(1, keepdim=True))
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        return {"y": y, "dx": dx.to(t), "dgain": (s["dy"].float() * n).sum(0).to(t)}
    if op == "linear_i8":
        y = (s["x"].float() @ s["w"].float().T) * s["xs"][:, None] * s["ws"]
        if s["bias"] is not None:
            y = y + s["bias"]
        return y.to(TYPES[s["out"]])
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    zg, zu = x @ wg.T, x @ wu.T
    if s["dtype"] == "i8":
        zg, zu = zg * s["xs"][:, None] * s["gs"], zu * s["xs"][:, None] * s["us"]
    a, da = _act(zg, s["act"])
    t = TYPES[s["out"]]
    h = (a * zu).to(t)
    if op == "gated":
        return h
    dh = s["dh"].float()
    dg, du = dh * zu * da, dh * a
    return {"h": h, "dx": (dg @ wg + du @ wu).to(t), "dw_gate": (dg.T @ x).to(t), "dw_up": (du.T @ x).to(t)}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    wide = lambda k: s[k].to(torch.float64)   # noqa: E731
    if op == "quantize":
        x = wide("x")
        unit = x.abs().max(dim=1).values.unsqueeze(1)
        return torch.round(x * 127.0 / unit) * (unit / 127.0)
    if op in ("rms_norm", "rms_norm_train"):
        gain = wide("gain")
        total = wide("x") if s["res"] is None else wide("x") + wide("res")
        length = torch.sqrt(torch.linalg.vector_norm(total, dim=1, keepdim=True) ** 2 / case["width"] + EPS)
        y = total / length * gain
        if case["out"] == "i8":
            # (the integers go by the sum in 32 bits, as it enters the norm)
            v = total.float().double() * gain
            unit = v.abs().max(dim=1).values.unsqueeze(1)
            y = torch.round(v * 127.0 / unit) * (unit / 127.0 / length)
        if op == "rms_norm":
            return {"y": y, "sum": total} if s["res"] is not None else {"y": y}
        total = total.to(s["x"].dtype).double()
        length = torch.sqrt(torch.linalg.vector_norm(total, dim=1, keepdim=True) ** 2 / case["width"] + EPS)
        along = total / length
        up = wide("dy") * gain
        dx = (up - along * torch.sum(up * along, dim=1, keepdim=True) / case["width"]) / length
        if s["dsum"] is not None:
            dx = dx + wide("dsum")
        return {"y": y, "dx": dx, "dgain": torch.sum(wide("dy") * along, dim=0)}
    if op == "linear_i8":
        y = torch.matmul(wide("x") * wide("xs")[:, None], (wide("w") * wide("ws")[:, None]).t())
        return y if s["bias"] is None else y + wide("bias")
    x, wg, wu = wide("x"), wide("wg"), wide("wu")
    if case["dtype"] == "i8":
        x, wg, wu = x * wide("xs")[:, None], wg * wide("gs")[:, None], wu * wide("us")[:, None]
    zg, zu = torch.matmul(x, wg.t()), torch.matmul(x, wu.t())
    if case["act"] == "silu":
        on = torch.sigmoid(zg)
        slope = on + zg * on * (1.0 - on)
    else:
        c = math.sqrt(2.0 / math.pi)
        bent = torch.tanh(c * zg * (1.0 + 0.044715 * zg * zg))
        on = 0.5 * (1.0 + bent)
        slope = on + zg * (1.0 - bent * bent) * (0.5 * c * (1.0 + 0.134145 * zg * zg))
    if op == "gated":
        return zg * on * zu
    dh = wide("dh")
    dg, du = dh * zu * slope, dh * zg * on
    return {"h": zg * on * zu, "dx": torch.matmul(dg, wg) + torch.matmul(du, wu), "dw_gate": torch.matmul(dg.t(), x),
            "dw_up": torch.matmul(du.t(), x)}


def work(case):
    """Inputs read once, outputs written once, and the products' operations."""
    op, rows, width = case["op"], float(case["rows"]), float(case["width"])
    if op == "quantize":
        return {"bytes": rows * width * (SIZE[case["dtype"]] + 1) + 4 * rows, "flops": 2 * rows * width}
    if op in ("rms_norm", "rms_norm_train"):
        e = SIZE[case["dtype"]]
        moved = rows * width * (e * (3 if case["residual"] else 1) + SIZE[case["out"]]) + e * width
        if case["out"] == "i8":
            moved += 4 * rows
        if op == "rms_norm_train":   # the gradient reads the sum and dy (and the residual stream's), writes dx and dgain
            moved += rows * width * e * (4 if case["residual"] else 3) + 2 * e * width
        return {"bytes": moved, "flops": 5 * rows * width * (3 if op == "rms_norm_train" else 1)}
    n = float(case["channels"])
    if op == "linear_i8":
        return {"bytes": rows * width + n * width + 4 * (rows + n) + SIZE[case["out"]] * rows * n, "flops": 2 * rows * n * width}
    e = SIZE[case["dtype"]]
    moved = e * (rows * width + 2 * n * width) + SIZE[case["out"]] * rows * n
    if case["dtype"] == "i8":
        moved += 4 * (rows + 2 * n)
    if op == "gated":
        return {"bytes": moved, "flops": 4 * rows * n * width}
    # the gradient reads dh, x and the weights, and writes as much as x and the weights; two more products of the first's size
    moved += e * (rows * n + 2 * rows * width + 4 * n * width)
    return {"bytes": moved, "flops": 12 * rows * n * width}


def _cost(case):
    """Microseconds, roughly, of the plain form: what a drawn case is held to."""
    w = work(case)
    return w["bytes"] / 1e6 + w["flops"] / 8e7


def _bytes_held(case):
    """What the plain form holds at once, roughly."""
    n = case.get("channels", 0)
    return 24.0 * case["rows"] * case["width"] + 24.0 * case["rows"] * n + 16.0 * n * case["width"]
