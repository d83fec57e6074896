"""Operators for residual and per-grid-point surrogates: cases with their plain forms
and their 64-bit values.

Three operators, each forward and backward, that make up a trained block
h + dropout(dense(group_norm(h))):

  dense     z = x W^T + bias, y = act(z) + residual; z is kept for the backward where
            the layer has an activation.  Backward from dy and z: with dz = dy act'(z)
            dx = dz W, dW = dz^T x, dbias = the column sums of dz.
  norm      group norm over channels-last data, x of samples x positions x channels:
            mean and variance of each sample and group over its positions and
            channels, p = weight (x - mean) / sqrt(var + eps) + bias, y = act(p).
            Backward from x, dy and the forward's mean and 1 / sqrt(var + eps):
            dx, dweight, dbias.
  dropout   y = residual + keep x / (1 - p), the mask from a counter-based generator
            and never stored: Philox4x32-10 (Salmon et al., SC'11) with the seed as its
            key and the counter (column / 8, row, site, step) gives 16 random bits for
            each of 8 columns, in order, low halves first; a value is dropped where its
            bits are below round(65536 p), and 1 / (1 - p) is of that p.  Backward: the
            same mask on dy.

act is one of none, relu, silu (z / (1 + exp(-z))) and gelu (z Phi(z)).

Operands are fp32 or bf16; biases, weights of the norm, statistics and gradients of
parameters are fp32.  Rows are padded to whole 16-byte pieces, as the library
asks; the padding holds arbitrary values.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-5


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # One request to the output layer of the 16x16 net: latency only.
        {"name": "dense-one", "kind": "dense", "rows": 1, "in": 64, "out": 256, "type": "fp32", "y": "fp32",
         "act": "none", "bias": True, "residual": False, "save": False},
        # Four requests for 1000x1000 fields, answered in fp32: the weights are read for four rows.
        {"name": "dense-field", "kind": "dense", "rows": 4, "in": 1024, "out": 1_000_000, "type": "bf16", "y": "fp32",
         "act": "none", "bias": True, "residual": False, "save": False},
        # The 100x100 net's output layer on a training batch.
        {"name": "dense-heat", "kind": "dense", "rows": 1024, "in": 256, "out": 10_000, "type": "fp32", "y": "fp32",
         "act": "none", "bias": True, "residual": False, "save": False},
        # A layer over the channels of every grid point: 16 fields of 100x100 points, 256 channels, in training.
        {"name": "dense-points", "kind": "dense", "rows": 160_000, "in": 256, "out": 256, "type": "bf16", "y": "bf16",
         "act": "silu", "bias": True, "residual": True, "save": True},
        # Gradients of a hidden layer of the deep 1000x1000 net.
        {"name": "dense-hidden-back", "kind": "dense-back", "rows": 1024, "in": 2048, "out": 2048, "type": "bf16",
         "act": "gelu", "bias": True, "dx": True},
        # Odd sizes everywhere.
        {"name": "dense-ragged-back", "kind": "dense-back", "rows": 331, "in": 437, "out": 6561, "type": "fp32",
         "act": "relu", "bias": True, "dx": True},
        # Gradients of the 1000x1000 net's output layer: the largest.
        {"name": "dense-field-back", "kind": "dense-back", "rows": 512, "in": 1024, "out": 1_000_000, "type": "bf16",
         "act": "none", "bias": True, "dx": True},
        # Before a hidden layer of the deep net: one position per sample.
        {"name": "norm-hidden", "kind": "norm", "samples": 1024, "positions": 1, "channels": 2048, "groups": 32,
         "type": "bf16", "act": "silu", "affine": True, "save": True},
        # Feature maps of 64 fields of 100x100 points.
        {"name": "norm-points", "kind": "norm", "samples": 64, "positions": 10_000, "channels": 64, "groups": 8,
         "type": "bf16", "act": "relu", "affine": True, "save": True},
        # Their gradients.
        {"name": "norm-points-back", "kind": "norm-back", "samples": 64, "positions": 10_000, "channels": 64,
         "groups": 8, "type": "bf16", "act": "relu", "affine": True},
        # After a hidden layer of the deep net, added to the block's input.
        {"name": "dropout-hidden", "kind": "dropout", "rows": 1024, "cols": 2048, "type": "bf16", "p": 0.1,
         "residual": True},
        # The mask again, on the gradients of 64 fields' feature maps.
        {"name": "dropout-points-back", "kind": "dropout-back", "rows": 640_000, "cols": 64, "type": "bf16", "p": 0.25},
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["dense", "dense", "dense-back", "dense-back", "norm", "norm-back", "dropout", "dropout-back"])
    typ = rng.choice(["fp32", "bf16"])
    act = rng.choice(["none", "relu", "silu", "gelu"])
    if kind in ("dense", "dense-back"):
        n_in = _log(rng, 4, 2048)
        # layers between hidden widths, and output layers
        n_out = _log(rng, 4, 2048) if rng.random() < 0.6 else _log(rng, 1_000, 200_000)
        most = min(160_000, int((4e10 if typ == "fp32" else 1e11) / (2 * n_in * n_out)), 2 ** 27 // (n_in + n_out))
        rows = _log(rng, 1, most if rng.random() < 0.8 else 16)
        case = {"kind": kind, "rows": rows, "in": n_in, "out": n_out, "type": typ, "act": act,
                "bias": rng.random() < 0.8}
        if kind == "dense":
            case.update({"y": rng.choice(["fp32", typ]), "residual": rng.random() < 0.5, "save": rng.random() < 0.5})
        else:
            case.update({"dx": rng.random() < 0.8})
        return case
    if kind in ("norm", "norm-back"):
        positions = 1 if rng.random() < 0.3 else _log(rng, 2, 40_000)
        # a group has some sixteen values at least: of two, whatever they are, one lies above the mean and one below
        groups, per = _log(rng, 1, 64), _log(rng, max(1, 16 // positions), 96)
        channels = groups * per
        samples = _log(rng, 1, max(1, min(2048, 30_000_000 // (channels * positions))))
        case = {"kind": kind, "samples": samples, "positions": positions, "channels": channels, "groups": groups,
                "type": typ, "act": act, "affine": rng.random() < 0.8}
        if kind == "norm":
            case["save"] = rng.random() < 0.5
        return case
    cols = _log(rng, 1, 4096) if rng.random() < 0.7 else _log(rng, 1_000, 1_000_000)
    case = {"kind": kind, "rows": _log(rng, 1, max(1, min(640_000, 40_000_000 // cols))), "cols": cols, "type": typ,
            "p": rng.choice([0.1, 0.25, 0.5, round(rng.uniform(0.0, 0.9), 3)])}
    if kind == "dropout":
        case["residual"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs
def _dev():
    return torch.device("cuda:0")


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    gen = torch.Generator(device=_dev())
    gen.manual_seed(seed)
    return gen


def _empty(shape, typ):
    """Rows padded to whole 16-byte pieces."""
    n = shape[-1]
    return torch.zeros(*shape[:-1], (n + 7) // 8 * 8, dtype=_dtype(typ), device=_dev())[..., :n]


def _normal(gen, shape, std, typ):
    n = shape[-1]
    full = torch.empty(*shape[:-1], (n + 7) // 8 * 8, dtype=_dtype(typ), device=_dev())
    return full.normal_(0.0, std, generator=gen)[..., :n]


def _vector(gen, n, lo, hi):
    return torch.empty(n, device=_dev()).uniform_(lo, hi, generator=gen)


def _dense_inputs(case, seed):
    """A normalised batch, a layer under training, for a backward the gradient of its
    output and the values before the activation, as a forward kept them."""
    gen = _gen(seed)
    m, n_in, n_out, typ = case["rows"], case["in"], case["out"], case["type"]
    d = {"x": _normal(gen, (m, n_in), 1.0, typ), "w": _normal(gen, (n_out, n_in), 1.0 / math.sqrt(n_in), typ)}
    d["bias"] = _vector(gen, n_out, -0.5, 0.5) if case["bias"] else None
    if case["kind"] == "dense":
        d["residual"] = _normal(gen, (m, n_out), 1.0, case["y"]) if case["residual"] else None
        return d
    # a mean over the batch and the field, brought to the size of one value
    d["dy"] = _normal(gen, (m, n_out), 1.0, typ)
    d["pre"] = _normal(gen, (m, n_out), 1.0, typ) if case["act"] != "none" else None
    return d


def _norm_inputs(case, seed):
    """Feature maps whose channels differ in level and spread, the norm's parameters
    after some training; for a backward also dy and the statistics that the forward kept."""
    gen = _gen(seed)
    n, p, c, g, typ = case["samples"], case["positions"], case["channels"], case["groups"], case["type"]
    x = _normal(gen, (n, p, c), 1.0, typ)
    level, spread = _vector(gen, c, -3.0, 3.0), _vector(gen, c, 0.2, 2.0)
    x.mul_(spread.to(x.dtype)).add_(level.to(x.dtype))
    d = {"x": x, "weight": _vector(gen, c, 0.5, 1.5) if case["affine"] else None,
         "bias": _vector(gen, c, -0.5, 0.5) if case["affine"] else None}
    if case["kind"] == "norm-back":
        d["dy"] = _normal(gen, (n, p, c), 1.0, typ)
        d["stats"] = torch.stack(_moments(x, g), -1).float()
    return d


def _moments(x, groups):
    """Mean and 1 / sqrt(var + eps) of every sample and group, in 64 bits, some samples at a time."""
    n, p, c = x.shape
    step = max(1, (1 << 24) // (p * c))
    mean, rstd = [], []
    for lo in range(0, n, step):
        v = x[lo:lo + step].double().reshape(-1, p, groups, c // groups)
        m = v.mean((1, 3), keepdim=True)
        mean.append(m[:, 0, :, 0])
        rstd.append((((v - m) ** 2).mean((1, 3)) + EPS) ** -0.5)
    return torch.cat(mean), torch.cat(rstd)


def _dropout_inputs(case, seed):
    gen = _gen(seed)
    m, n, typ = case["rows"], case["cols"], case["type"]
    d = {"x": _normal(gen, (m, n), 1.0, typ)}
    d["residual"] = _normal(gen, (m, n), 1.0, typ) if case.get("residual") else None
    d["seed"] = 0x9E3779B97F4A7C15 * (seed + 1) % (1 << 63)
    d["site"], d["step"] = 3, 1000 + seed % 1000
    return d


def prepare(case, seed):
    d = {"case": dict(case), "own": own}
    typ, back = case["type"], case["kind"].endswith("-back")
    if own:
        import paper_2309_16743_amd as lib
        prec = lib.OT_BF16 if typ == "bf16" else lib.OT_FP32
        act = {"none": lib.OT_ACT_NONE, "relu": lib.OT_ACT_RELU, "silu": lib.OT_ACT_SILU,
               "gelu": lib.OT_ACT_GELU}[case.get("act", "none")]
    if case["kind"] in ("dense", "dense-back"):
        d.update(_dense_inputs(case, seed))
        m, n_in, n_out = case["rows"], case["in"], case["out"]
        if not back:
            d["out_y"] = _empty((m, n_out), case["y"])
            d["out_pre"] = _empty((m, n_out), typ) if case["save"] else None
        else:
            d["out_dx"] = _empty((m, n_in), typ) if case["dx"] else None
            d["out_dw"] = _empty((n_out, n_in), "fp32")
            d["out_db"] = torch.zeros(n_out, device=_dev()) if case["bias"] else None
        if own:
            d["op"] = lib.DenseLayer(n_in, n_out, precision=prec, activation=act, max_rows=m)
    elif case["kind"] in ("norm", "norm-back"):
        d.update(_norm_inputs(case, seed))
        n, p, c, g = case["samples"], case["positions"], case["channels"], case["groups"]
        if not back:
            d["out_y"] = _empty((n, p, c), typ)
            d["out_stats"] = torch.zeros(n, g, 2, device=_dev()) if case["save"] else None
        else:
            d["out_dx"] = _empty((n, p, c), typ)
            for k in ("out_dw", "out_db"):
                d[k] = torch.zeros(c, device=_dev()) if case["affine"] else None
        if own:
            d["op"] = lib.GroupNorm(c, g, positions=p, precision=prec, activation=act, eps=EPS, max_samples=n)
    else:
        d.update(_dropout_inputs(case, seed))
        d["out_y"] = _empty((case["rows"], case["cols"]), typ)
        if own:
            d["op"] = lib.Dropout(case["p"], d["seed"], site=d["site"], precision=prec)
    return d


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    return {"dense": _dense, "dense-back": _dense_back, "norm": _norm, "norm-back": _norm_back, "dropout": _dropout,
            "dropout-back": _dropout_back}[case["kind"]](state, case)


def _act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, name):
    """The activation's derivative at z."""
    if name == "relu":
        return (z > 0).float()
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _dense(s, case):
    if s["own"]:
        s["op"].forward(s["x"], s["w"], s["out_y"], bias=s["bias"], residual=s["residual"], pre=s["out_pre"])
    else:
        z = s["x"].float() @ s["w"].float().t()
        if s["bias"] is not None:
            z += s["bias"]
        if case["save"]:
            s["out_pre"].copy_(z)
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        s["out_y"].copy_(y)
    return {"y": s["out_y"], "pre": s["out_pre"]} if case["save"] else {"y": s["out_y"]}


def _dense_back(s, case):
    if s["own"]:
        s["op"].backward(s["x"], s["w"], s["dy"], pre=s["pre"], dx=s["out_dx"], dw=s["out_dw"], dbias=s["out_db"])
    else:
        dz = s["dy"].float()
        if s["pre"] is not None:
            dz = dz * _slope(s["pre"].float(), case["act"])
        s["out_dw"].copy_(dz.t() @ s["x"].float())
        if case["dx"]:
            s["out_dx"].copy_(dz @ s["w"].float())
        if case["bias"]:
            s["out_db"].copy_(dz.sum(0))
    return {k: s["out_" + k] for k in ("dx", "dw", "db") if s["out_" + k] is not None}


def _grouped(x, g):
    return x.float().reshape(x.shape[0], x.shape[1], g, x.shape[2] // g)


def _norm(s, case):
    if s["own"]:
        s["op"].forward(s["x"], s["out_y"], weight=s["weight"], bias=s["bias"], stats=s["out_stats"])
    else:
        x = _grouped(s["x"], case["groups"])
        mean = x.mean((1, 3), keepdim=True)
        x = x - mean
        rstd = 1.0 / torch.sqrt((x * x).mean((1, 3), keepdim=True) + EPS)
        p = (x * rstd).reshape(s["x"].shape)
        if case["affine"]:
            p = p * s["weight"] + s["bias"]
        s["out_y"].copy_(_act(p, case["act"]))
        if case["save"]:
            s["out_stats"].copy_(torch.stack((mean[:, 0, :, 0], rstd[:, 0, :, 0]), -1))
    return {"y": s["out_y"], "stats": s["out_stats"]} if case["save"] else {"y": s["out_y"]}


def _norm_back(s, case):
    if s["own"]:
        s["op"].backward(s["x"], s["stats"], s["dy"], weight=s["weight"], bias=s["bias"], dx=s["out_dx"],
                         dweight=s["out_dw"], dbias=s["out_db"])
    else:
        g, shape = case["groups"], s["x"].shape
        mean, rstd = s["stats"][:, None, :, None, 0], s["stats"][:, None, :, None, 1]
        xh = (_grouped(s["x"], g) - mean) * rstd
        flat = xh.reshape(shape)
        dp = s["dy"].float()
        if case["act"] != "none":
            dp = dp * _slope(flat * s["weight"] + s["bias"] if case["affine"] else flat, case["act"])
        if case["affine"]:
            s["out_db"].copy_(dp.sum((0, 1)))
            s["out_dw"].copy_((dp * flat).sum((0, 1)))
            dp = dp * s["weight"]
        dh = dp.reshape(xh.shape)
        dx = dh - dh.mean((1, 3), keepdim=True) - xh * (dh * xh).mean((1, 3), keepdim=True)
        s["out_dx"].copy_((dx * rstd).reshape(shape))
    return {k: s["out_" + k] for k in ("dx", "dw", "db") if s["out_" + k] is not None}


_M32 = 0xFFFFFFFF


def _bits(d, rows, cols):
    """16 random bits of every value: rows x (cols rounded up to 8)."""
    blocks = (cols + 7) // 8
    c0 = torch.arange(blocks, device=_dev())[None, :].expand(rows, blocks)
    c1 = torch.arange(rows, device=_dev())[:, None].expand(rows, blocks)
    c2, c3 = torch.full_like(c0, d["site"]), torch.full_like(c0, d["step"])
    k0, k1 = d["seed"] & _M32, d["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57            # modulo 2^64: the upper words survive the sign
        c0, c1, c2, c3 = ((b >> 32) & _M32) ^ c1 ^ k0, b & _M32, ((a >> 32) & _M32) ^ c3 ^ k1, a & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    w = torch.stack((c0, c1, c2, c3), -1)
    return torch.stack((w & 0xFFFF, w >> 16), -1).reshape(rows, 8 * blocks)


def _dropped(d, case):
    """(values that are kept, their scale)."""
    t = int(round(65536 * case["p"]))
    return _bits(d, case["rows"], case["cols"])[:, :case["cols"]] >= t, 65536 / (65536 - t)


def _dropout(s, case):
    if s["own"]:
        s["op"].forward(s["x"], s["out_y"], s["step"], residual=s["residual"])
    else:
        keep, scale = _dropped(s, case)
        y = torch.where(keep, s["x"].float() * scale, torch.zeros((), device=_dev()))
        if s["residual"] is not None:
            y = y + s["residual"].float()
        s["out_y"].copy_(y)
    return {"y": s["out_y"]}


def _dropout_back(s, case):
    if s["own"]:
        s["op"].backward(s["x"], s["out_y"], s["step"])
    else:
        keep, scale = _dropped(s, case)
        s["out_y"].copy_(torch.where(keep, s["x"].float() * scale, torch.zeros((), device=_dev())))
    return {"dx": s["out_y"]}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    e = 2 if case["type"] == "bf16" else 4
    kind = case["kind"]
    if kind in ("dense", "dense-back"):
        m, n_in, n_out = case["rows"], case["in"], case["out"]
        if kind == "dense":
            y = 2 if case["y"] == "bf16" else 4
            b = e * (m * n_in + n_in * n_out) + y * m * n_out * (2 if case["residual"] else 1)
            b += (4 * n_out if case["bias"] else 0) + (e * m * n_out if case["save"] else 0)
            return {"bytes": b, "flops": 2 * m * n_in * n_out}
        b = e * m * (n_in + n_out * (1 if case["act"] == "none" else 2)) + 4 * n_out * n_in
        b += 4 * n_out if case["bias"] else 0
        f = 2 * m * n_in * n_out
        if case["dx"]:
            b += e * (n_out * n_in + m * n_in)
            f *= 2
        return {"bytes": b, "flops": f}
    if kind in ("norm", "norm-back"):
        n = case["samples"] * case["positions"] * case["channels"]
        stats = 8 * case["samples"] * case["groups"]
        par = 4 * case["channels"] if case["affine"] else 0
        if kind == "norm":
            return {"bytes": 2 * e * n + 2 * par + (stats if case["save"] else 0), "flops": 8 * n}
        return {"bytes": 3 * e * n + 4 * par + stats, "flops": 16 * n}
    n = case["rows"] * case["cols"]
    return {"bytes": e * n * (3 if case.get("residual") else 2), "flops": 2 * n}


# ------------------------------------------------------------------ 64-bit values
_CHUNK = 32768      # rows or output columns at a time


def _phi(z):
    """The normal distribution's integral, from the complementary error function, which keeps its digits in the tail."""
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _value64(z, name):
    return {"none": lambda: z, "relu": lambda: torch.maximum(z, torch.zeros_like(z)),
            "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * _phi(z)}[name]()


def _slope64(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return torch.heaviside(z, torch.zeros_like(z))
    if name == "silu":
        return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
    return _phi(z) + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)


def _dense_exact(case, seed):
    d = _dense_inputs(case, seed)
    m, n_in, n_out = case["rows"], case["in"], case["out"]
    dev = d["x"].device
    wide = dict(dtype=torch.float64, device=dev)
    if case["kind"] == "dense":
        y = torch.empty(m, n_out, **wide)
        pre = torch.empty(m, n_out, **wide) if case["save"] else None
        for r in range(0, m, _CHUNK):
            x = d["x"][r:r + _CHUNK].double()
            for c in range(0, n_out, _CHUNK):
                z = torch.mm(x, d["w"][c:c + _CHUNK].double().t())
                if d["bias"] is not None:
                    z += d["bias"][c:c + _CHUNK].double()
                if pre is not None:
                    pre[r:r + _CHUNK, c:c + _CHUNK] = z
                v = _value64(z, case["act"])
                if d["residual"] is not None:
                    v = v + d["residual"][r:r + _CHUNK, c:c + _CHUNK].double()
                y[r:r + _CHUNK, c:c + _CHUNK] = v
        return {"y": y, "pre": pre} if case["save"] else {"y": y}
    out = {}
    if case["dx"]:
        out["dx"] = torch.zeros(m, n_in, **wide)
    out["dw"] = torch.zeros(n_out, n_in, **wide)
    if case["bias"]:
        out["db"] = torch.zeros(n_out, **wide)
    for r in range(0, m, _CHUNK):
        x = d["x"][r:r + _CHUNK].double()
        for c in range(0, n_out, _CHUNK):
            dz = d["dy"][r:r + _CHUNK, c:c + _CHUNK].double()
            if d["pre"] is not None:
                dz = dz * _slope64(d["pre"][r:r + _CHUNK, c:c + _CHUNK].double(), case["act"])
            out["dw"][c:c + _CHUNK] += torch.mm(dz.t(), x)
            if case["dx"]:
                out["dx"][r:r + _CHUNK] += torch.mm(dz, d["w"][c:c + _CHUNK].double())
            if case["bias"]:
                out["db"][c:c + _CHUNK] += torch.sum(dz, 0)
    return out


def _norm_exact(case, seed):
    """Channel by channel within a group: sums over the positions first."""
    d = _norm_inputs(case, seed)
    n, p, c, g = case["samples"], case["positions"], case["channels"], case["groups"]
    dev = d["x"].device
    per = c // g
    one, zero = torch.ones(c, dtype=torch.float64, device=dev), torch.zeros(c, dtype=torch.float64, device=dev)
    wt = d["weight"].double() if case["affine"] else one
    bs = d["bias"].double() if case["affine"] else zero
    spread = lambda v: v.repeat_interleave(per, dim=1)[:, None, :]          # samples x groups -> x channels
    fold = lambda v: v.sum(1).reshape(-1, g, per).sum(-1) / (p * per)       # the mean over a group
    if case["kind"] == "norm":
        mean, rstd = _moments(d["x"], g)
    else:
        mean, rstd = d["stats"][..., 0].double(), d["stats"][..., 1].double()
    out, dw, db = [], zero.clone(), zero.clone()
    step = max(1, (1 << 24) // (p * c))
    for lo in range(0, n, step):
        s = slice(lo, lo + step)
        xh = (d["x"][s].double() - spread(mean[s])) * spread(rstd[s])
        pre = xh * wt + bs
        if case["kind"] == "norm":
            out.append(_value64(pre, case["act"]))
            continue
        dp = d["dy"][s].double() * _slope64(pre, case["act"])
        db += dp.sum((0, 1))
        dw += (dp * xh).sum((0, 1))
        dp = dp * wt
        out.append(spread(rstd[s]) * (dp - spread(fold(dp)) - xh * spread(fold(dp * xh))))
    out = torch.cat(out)
    if case["kind"] == "norm":
        return {"y": out, "stats": torch.stack((mean, rstd), -1)} if case["save"] else {"y": out}
    return {"dx": out, "dw": dw, "db": db} if case["affine"] else {"dx": out}


def _philox(c0, c1, c2, c3, key):
    """Four words of 32 bits per counter, in unsigned 64-bit arithmetic."""
    u = np.uint64
    mask, half = u(0xFFFFFFFF), u(32)
    x = [np.asarray(v, dtype=u) for v in (c0, c1, c2, c3)]
    k = [key % 2 ** 32, key // 2 ** 32]
    for _ in range(10):
        p, q = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(q >> half) ^ x[1] ^ u(k[0]), q & mask, (p >> half) ^ x[3] ^ u(k[1]), p & mask]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return x


def _dropout_exact(case, seed):
    d = _dropout_inputs(case, seed)
    m, n = case["rows"], case["cols"]
    t = int(round(65536 * case["p"]))
    blocks = -(-n // 8)
    y = torch.empty(m, n, dtype=torch.float64, device=d["x"].device)
    step = max(1, (1 << 21) // blocks)
    for lo in range(0, m, step):
        rows = np.arange(lo, min(m, lo + step), dtype=np.uint64)
        words = _philox(np.tile(np.arange(blocks), len(rows)), np.repeat(rows, blocks), d["site"], d["step"], d["seed"])
        parts = [f(w) for w in words for f in (lambda v: v % np.uint64(65536), lambda v: v // np.uint64(65536))]
        drawn = np.stack(parts, axis=-1).reshape(len(rows), 8 * blocks)[:, :n]
        keep = torch.from_numpy(drawn >= np.uint64(t)).to(y.device)
        v = d["x"][lo:lo + step].double() / (1.0 - t / 65536.0)
        y[lo:lo + step] = torch.where(keep, v, torch.zeros_like(v))
    if d["residual"] is not None:
        y += d["residual"].double()
    return {"y" if case["kind"] == "dropout" else "dx": y}


def exact(case, seed):
    if case["kind"] in ("dense", "dense-back"):
        return _dense_exact(case, seed)
    if case["kind"] in ("norm", "norm-back"):
        return _norm_exact(case, seed)
    return _dropout_exact(case, seed)
