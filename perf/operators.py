"""Operators for adapting one trained surrogate to many ensembles at once: cases
with their plain forms and their 64-bit values.

A bank of G low-rank adapters stands beside one frozen projection (a layer of the
surrogate): row m of a batch names its adapter ids[m] (negative or past the bank:
none), and with s_g the adapter's scale

    t_m = down_g x_m                       (rank values)
    y_m = W x_m + bias + s_g up_g^T t_m    (then ReLU, if asked)

down is G x rank x in and up is G x rank x out: both keep the layer's long axis
contiguous.  Kinds of case (the key "kind"):

  forward   y, and t where a later backward needs it.
  backward  from dy: dx = W^T dy + s_g down_g^T dt', with dt = s_g up_g dy, and the
            gradients of both banks (W is frozen); dx is masked where the layer's
            input was a ReLU's zero, if asked.
  clip      the global norm over a list of gradient tensors, and the list scaled by
            min(1, max_norm / norm) into a second list.
  step      the same norm, then Adam with the clipped gradients over the list,
            with a bf16 copy of the parameters where the layer computes in bf16.

Operands are fp32 or bf16; bias, scales, t and every gradient of a parameter are
fp32.  Rows are padded to whole 16-byte pieces, as the library asks; the padding
holds arbitrary values.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # One request to the hidden-to-output layer of the 16x16 net: latency only.
        {"name": "serve-one", "kind": "forward", "rows": 1, "in": 64, "out": 256, "rank": 4, "adapters": 4,
         "type": "fp32", "y": "fp32", "relu": False, "bias": True, "save": False, "none": 0.0},
        # Sixteen requests for 1000x1000 fields, eight ensembles, answered in fp32: every
        # weight is read for sixteen rows.
        {"name": "serve-field", "kind": "forward", "rows": 16, "in": 1024, "out": 1_000_000, "rank": 16, "adapters": 8,
         "type": "bf16", "y": "fp32", "relu": False, "bias": True, "save": False, "none": 0.1},
        # The 100x100 net's output layer in training: a batch drawn at random from 16 ensembles.
        {"name": "forward-heat", "kind": "forward", "rows": 1024, "in": 256, "out": 10_000, "rank": 8, "adapters": 16,
         "type": "fp32", "y": "fp32", "relu": False, "bias": True, "save": True, "none": 0.0},
        # A hidden layer of the deep 1000x1000 net in training.
        {"name": "forward-hidden", "kind": "forward", "rows": 1024, "in": 2048, "out": 2048, "rank": 16,
         "adapters": 32, "type": "bf16", "y": "bf16", "relu": True, "bias": True, "save": True, "none": 0.0},
        # The deep net's output layer: the largest product.
        {"name": "forward-deep", "kind": "forward", "rows": 1024, "in": 2048, "out": 1_000_000, "rank": 16,
         "adapters": 8, "type": "bf16", "y": "bf16", "relu": False, "bias": True, "save": True, "none": 0.0},
        # Gradients of that hidden layer, dx masked for the layer before it.
        {"name": "backward-hidden", "kind": "backward", "rows": 1024, "in": 2048, "out": 2048, "rank": 16,
         "adapters": 32, "type": "bf16", "mask": True, "dx": True, "none": 0.0},
        # Odd sizes everywhere, a rank that is no multiple of anything, rows without an adapter.
        {"name": "backward-ragged", "kind": "backward", "rows": 331, "in": 437, "out": 6561, "rank": 5, "adapters": 7,
         "type": "fp32", "mask": True, "dx": True, "none": 0.1},
        # Gradients through the 1000x1000 net's output layer.
        {"name": "backward-field", "kind": "backward", "rows": 512, "in": 1024, "out": 1_000_000, "rank": 16,
         "adapters": 8, "type": "bf16", "mask": True, "dx": True, "none": 0.0},
        # Every adapter of the 100x100 net, one tensor per ensemble, layer and side: 96 small tensors.
        {"name": "clip-adapters", "kind": "clip", "set": "adapters", "widths": "6-256-256-10000", "rank": 8,
         "adapters": 16, "type": "fp32", "above": True},
        # All parameters of a net with fields of 100,000 values.
        {"name": "clip-net", "kind": "clip", "set": "net", "widths": "6-1024-1024-100000", "type": "fp32",
         "above": True},
        # The adapters again, their fp32 masters updated and copied to bf16.
        {"name": "step-adapters", "kind": "step", "set": "adapters", "widths": "6-256-256-10000", "rank": 8,
         "adapters": 16, "copies": True, "above": True},
        # The whole net trained with a bounded gradient.
        {"name": "step-net", "kind": "step", "set": "net", "widths": "6-1024-1024-100000", "copies": False,
         "above": True},
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["forward", "forward", "backward", "backward", "clip", "step"])
    if kind in ("forward", "backward"):
        typ = rng.choice(["fp32", "bf16"])
        rank = _log(rng, 1, 64)
        n_in = _log(rng, 16, 512 if typ == "fp32" else 2048)
        # layers between hidden widths, and output layers
        n_out = _log(rng, 16, 2048) if rng.random() < 0.5 else _log(rng, 1_000, 300_000 if typ == "fp32" else 1_000_000)
        adapters = min(_log(rng, 1, 64), max(1, 2 ** 28 // (rank * (n_in + n_out))))
        case = {"kind": kind, "rows": _log(rng, 1, 1024), "in": n_in, "out": n_out, "rank": rank, "adapters": adapters,
                "type": typ, "none": rng.choice([0.0, 0.0, 0.2])}
        if kind == "forward":
            case.update({"y": rng.choice(["fp32", typ]), "relu": rng.random() < 0.5, "bias": rng.random() < 0.8,
                         "save": rng.random() < 0.5})
        else:
            case.update({"mask": rng.random() < 0.5, "dx": rng.random() < 0.8})
        return case
    case = {"kind": kind, "set": "spread", "total": _log(rng, 1_000, 100_000_000), "tensors": _log(rng, 1, 400),
            "mix": rng.randrange(1 << 30), "above": rng.random() < 0.7}
    if kind == "clip":
        case["type"] = rng.choice(["fp32", "bf16"])
    else:
        case["copies"] = rng.random() < 0.5
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


def _uniform(gen, shape, bound, typ):
    """Values in (-bound, bound), the last axis padded to whole 16-byte pieces."""
    n = shape[-1]
    ld = (n + 7) // 8 * 8
    full = torch.empty(*shape[:-1], ld, dtype=_dtype(typ), device=_dev())
    full.uniform_(-bound, bound, generator=gen)
    return full[..., :n]


def _empty(shape, typ):
    n = shape[-1]
    return torch.zeros(*shape[:-1], (n + 7) // 8 * 8, dtype=_dtype(typ), device=_dev())[..., :n]


def _layer_inputs(case, seed):
    """Everything a caller has in hand: a batch of hidden activations (a ReLU's
    output), the frozen layer, both banks after some training, one adapter id per row
    and one scale per adapter; for a backward also dy and the saved t."""
    gen = _gen(seed)
    m, n_in, n_out, r, g = case["rows"], case["in"], case["out"], case["rank"], case["adapters"]
    typ = case["type"]
    d = {"x": _uniform(gen, (m, n_in), 2.0, typ), "w": _uniform(gen, (n_out, n_in), 1.0 / math.sqrt(n_in), typ),
         "down": _uniform(gen, (g, r, n_in), 1.0 / math.sqrt(n_in), typ),
         "up": _uniform(gen, (g, r, n_out), 0.5 / math.sqrt(r), typ)}
    d["x"].clamp_(min=0)
    ids = torch.randint(0, g, (m,), generator=gen, device=_dev())
    ids = torch.where(torch.rand(m, generator=gen, device=_dev()) < case["none"], -torch.ones_like(ids), ids)
    d["ids"] = ids.to(torch.int32)
    d["scale"] = torch.empty(g, device=_dev()).uniform_(0.5, 2.0, generator=gen)
    if case["kind"] == "forward":
        d["bias"] = torch.empty(n_out, device=_dev()).uniform_(-1, 1, generator=gen) if case["bias"] else None
    else:
        # a mean over the batch and the field, brought to the size of one value
        d["dy"] = _uniform(gen, (m, n_out), 1.0, typ)
        idx = ids.clamp(min=0)
        t = torch.empty(m, r, device=_dev())
        for lo in range(0, m, 64):                       # the saved forward values, rounded to fp32
            a = d["down"][idx[lo:lo + 64]].double()
            t[lo:lo + 64] = (a * d["x"][lo:lo + 64].double()[:, None, :]).sum(-1).float()
        t[ids < 0] = 0.0
        d["t"] = t
    return d


def _sizes(case):
    """Elements of every tensor of a case's list."""
    if case["set"] == "net":
        w = [int(v) for v in case["widths"].split("-")]
        return [n for i, o in zip(w, w[1:]) for n in (o * i, o)]
    if case["set"] == "adapters":
        w = [int(v) for v in case["widths"].split("-")]
        r = case["rank"]
        return [n for _ in range(case["adapters"]) for i, o in zip(w, w[1:]) for n in (r * i, r * o)]
    rng = random.Random(case["mix"])
    share = [math.exp(rng.uniform(0.0, 8.0)) for _ in range(case["tensors"])]
    return [max(1, int(case["total"] * s / sum(share))) for s in share]


def _split(flat, sizes):
    """Consecutive pieces of one array, at whatever offsets they fall on."""
    return list(torch.split(flat, sizes))


def _list_inputs(case, seed):
    """Gradients in one array whose pieces are the tensors (as a bank's per-ensemble
    slices are), and for a step the parameters and moments of a training under way."""
    gen = _gen(seed)
    sizes = _sizes(case)
    n = sum(sizes)
    typ = case.get("type", "fp32")
    g = torch.empty(n, device=_dev()).normal_(0.0, 1e-3, generator=gen)
    # tensors of a net differ in the size of their gradients
    for i, piece in enumerate(_split(g, sizes)):
        if i < 64:
            piece.mul_(0.25 + 0.5 * (i % 5))
    g = g.to(_dtype(typ))
    d = {"sizes": sizes, "g": g}
    d["max_norm"] = (0.1 if case["above"] else 10.0) * 1e-3 * math.sqrt(n)
    if case["kind"] == "step":
        d["p"] = torch.empty(n, device=_dev()).normal_(0.0, 0.05, generator=gen)
        d["m"] = torch.empty(n, device=_dev()).normal_(0.0, 3e-4, generator=gen)
        d["v"] = torch.empty(n, device=_dev()).uniform_(1e-8, 1e-6, generator=gen)
        d["t"] = 10                                      # steps taken so far
    return d


def prepare(case, seed):
    d = {"case": dict(case), "own": own}
    if case["kind"] in ("forward", "backward"):
        d.update(_layer_inputs(case, seed))
        m, n_in, n_out, r, g = case["rows"], case["in"], case["out"], case["rank"], case["adapters"]
        if own:
            from paper_2309_16743_amd import OT_BF16, OT_FP32, LowRankAdapters
            d["bank"] = LowRankAdapters(n_in, n_out, r, g, precision=OT_BF16 if case["type"] == "bf16" else OT_FP32,
                                        max_rows=m)
            if case["kind"] == "forward":
                d["out_y"] = _empty((m, n_out), case["y"])
                d["out_t"] = torch.zeros(m, r, device=_dev()) if case["save"] else None
            else:
                d["out_dx"] = _empty((m, n_in), case["type"]) if case["dx"] else None
                d["out_ddown"] = _empty((g, r, n_in), "fp32")
                d["out_dup"] = _empty((g, r, n_out), "fp32")
        return d
    flat = _list_inputs(case, seed)
    sizes, n = flat["sizes"], sum(flat["sizes"])
    if case["kind"] == "clip":
        flat["out"] = torch.empty_like(flat["g"])
    elif case["copies"]:
        flat["copies"] = torch.empty(n, dtype=torch.bfloat16, device=_dev())
    d["flat"] = flat
    d["norm"] = torch.zeros(1, device=_dev())
    d.update({"max_norm": flat["max_norm"], "t": flat.get("t")})
    d.update({k: _split(flat[k], sizes) for k in ("g", "out", "p", "m", "v", "copies") if k in flat})
    if own:
        from paper_2309_16743_amd import AdamTensors, GradientClip
        if case["kind"] == "clip":
            d["clip"] = GradientClip(d["g"], d["out"])
        else:
            d["adam"] = AdamTensors(d["p"], d["g"], d["m"], d["v"], copies=d.get("copies"), lr=LR, beta1=BETA1,
                                    beta2=BETA2, eps=EPS, steps=d["t"])
    return d


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    return {"forward": _forward, "backward": _backward, "clip": _clip, "step": _step}[case["kind"]](state, case)


def _members(ids, g):
    """M x G: 1 where row m uses adapter g."""
    return (ids[:, None] == torch.arange(g, dtype=ids.dtype, device=ids.device)[None, :]).float()


def _forward(s, case):
    if s["own"]:
        s["bank"].forward(s["x"], s["w"], s["down"], s["up"], s["ids"], s["out_y"], bias=s["bias"], scale=s["scale"],
                          t=s["out_t"], relu=case["relu"])
        return {"y": s["out_y"], "t": s["out_t"]} if case["save"] else {"y": s["out_y"]}
    g, r, n_in, n_out = case["adapters"], case["rank"], case["in"], case["out"]
    x = s["x"].float()
    own_rows = _members(s["ids"], g)                                     # M x G
    # all adapters' low-rank values, of which a row keeps its own adapter's
    t = (x @ s["down"].float().reshape(g * r, n_in).t()).reshape(-1, g, r) * own_rows[:, :, None]
    y = x @ s["w"].float().t()
    y += (t * s["scale"][None, :, None]).reshape(-1, g * r) @ s["up"].float().reshape(g * r, n_out)
    if s["bias"] is not None:
        y += s["bias"]
    if case["relu"]:
        y = y.clamp(min=0)
    y = y.to(_dtype(case["y"]))
    return {"y": y, "t": t.sum(1)} if case["save"] else {"y": y}


def _backward(s, case):
    if s["own"]:
        s["bank"].backward(s["x"], s["w"], s["down"], s["up"], s["ids"], s["dy"], s["t"], s["out_ddown"], s["out_dup"],
                           dx=s["out_dx"], scale=s["scale"], relu_input=case["mask"])
        out = {"ddown": s["out_ddown"], "dup": s["out_dup"]}
        if case["dx"]:
            out["dx"] = s["out_dx"]
        return out
    g, r, n_in, n_out = case["adapters"], case["rank"], case["in"], case["out"]
    x, dy = s["x"].float(), s["dy"].float()
    own_rows = _members(s["ids"], g) * s["scale"][None, :]               # M x G, with the scales
    down, up = s["down"].float().reshape(g * r, n_in), s["up"].float().reshape(g * r, n_out)
    dt = ((dy @ up.t()).reshape(-1, g, r) * own_rows[:, :, None]).reshape(-1, g * r)
    ts = (s["t"][:, None, :] * own_rows[:, :, None]).reshape(-1, g * r)
    out = {"ddown": (dt.t() @ x).reshape(g, r, n_in), "dup": (ts.t() @ dy).reshape(g, r, n_out)}
    if case["dx"]:
        dx = dy @ s["w"].float() + dt @ down
        if case["mask"]:
            dx = dx * (x > 0)
        out["dx"] = dx.to(_dtype(case["type"]))
    return out


def _norm(grads):
    total = torch.zeros((), device=_dev())
    for piece in grads:
        total = total + (piece.float() * piece.float()).sum()
    return total.sqrt()


def _coefficient(norm, max_norm):
    """min(1, max_norm / norm); 1 where the norm is zero or not a number to divide by."""
    c = torch.where(norm > max_norm, max_norm / norm, torch.ones_like(norm))
    return torch.where(torch.isfinite(norm), c, torch.ones_like(norm))


def _clip(s, case):
    if s["own"]:
        s["clip"].apply(s["max_norm"], norm=s["norm"])
        return {"norm": s["norm"], "g": s["flat"]["out"]}
    norm = _norm(s["g"])
    c = _coefficient(norm, s["max_norm"])
    for src, dst in zip(s["g"], s["out"]):
        dst.copy_(src.float() * c)
    s["norm"].copy_(norm)
    return {"norm": s["norm"], "g": s["flat"]["out"]}


def _step(s, case):
    if s["own"]:
        s["adam"].step(max_norm=s["max_norm"], norm=s["norm"])
    else:
        norm = _norm(s["g"])
        c = _coefficient(norm, s["max_norm"])
        take = torch.isfinite(norm)                      # no step on a gradient that is not finite
        s["t"] += 1
        c1, c2 = 1.0 - BETA1 ** s["t"], 1.0 - BETA2 ** s["t"]
        for i, (p, g, m, v) in enumerate(zip(s["p"], s["g"], s["m"], s["v"])):
            gc = g * c
            mn = BETA1 * m + (1.0 - BETA1) * gc
            vn = BETA2 * v + (1.0 - BETA2) * gc * gc
            pn = p - LR * (mn / c1) / ((vn / c2).sqrt() + EPS)
            p.copy_(torch.where(take, pn, p))
            m.copy_(torch.where(take, mn, m))
            v.copy_(torch.where(take, vn, v))
            if case["copies"]:
                s["copies"][i].copy_(p)
        s["norm"].copy_(norm)
    return {"norm": s["norm"], **{k: s["flat"][k] for k in ("p", "m", "v", "copies") if k in s["flat"]}}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] in ("forward", "backward"):
        m, n_in, n_out, r = case["rows"], case["in"], case["out"], case["rank"]
        e = 2 if case["type"] == "bf16" else 4
        used = min(case["adapters"], m)                   # adapters that rows name
        banks = used * r * (n_in + n_out)
        if case["kind"] == "forward":
            y = 2 if case["y"] == "bf16" else 4
            b = e * (m * n_in + n_in * n_out + banks) + y * m * n_out + 4 * m
            b += (4 * n_out if case["bias"] else 0) + (4 * m * r if case["save"] else 0)
            f = 2 * m * (n_in * n_out + r * (n_in + n_out))
            return {"bytes": b, "flops": f}
        grads = case["adapters"] * r * (n_in + n_out)
        b = e * (m * n_in + m * n_out + used * r * n_out) + 4 * m * (r + 1) + 4 * grads
        f = 2 * m * r * (2 * n_out + n_in)
        if case["dx"]:
            b += e * (n_in * n_out + m * n_in + used * r * n_in)
            f += 2 * m * (n_in * n_out + r * n_in)
        return {"bytes": b, "flops": f}
    n = sum(_sizes(case))
    if case["kind"] == "clip":
        e = 2 if case["type"] == "bf16" else 4
        return {"bytes": 2 * e * n + 4, "flops": 3 * n}
    return {"bytes": (28 + (2 if case["copies"] else 0)) * n + 4, "flops": 14 * n}


# ------------------------------------------------------------------ 64-bit values
_CHUNK = 32768      # output columns at a time


def _layer_exact(case, seed):
    """From the effective weight of each ensemble, V_g = W + s_g up_g^T down_g: y = V_g x,
    dx = V_g^T dy, and with E_g = sum dy x^T over the ensemble's rows the chain rule
    through V_g: dup_g = s_g (E_g down_g^T)^T, ddown_g = s_g up_g E_g."""
    d = _layer_inputs(case, seed)
    g, r, n_in, n_out, m = case["adapters"], case["rank"], case["in"], case["out"], case["rows"]
    dev = d["x"].device
    x = d["x"].double()
    ids = d["ids"].tolist()
    rows = {}
    for i, k in enumerate(ids):
        rows.setdefault(k if 0 <= k < g else -1, []).append(i)
    rows = {k: torch.tensor(v, device=dev) for k, v in rows.items()}
    scale = d["scale"].double()
    if case["kind"] == "forward":
        y = torch.empty(m, n_out, dtype=torch.float64, device=dev)
        for c in range(0, n_out, _CHUNK):
            w = d["w"][c:c + _CHUNK].double()
            for k, idx in rows.items():
                v = w if k < 0 else w + scale[k] * (d["up"][k][:, c:c + _CHUNK].double().t() @ d["down"][k].double())
                y[idx, c:c + _CHUNK] = x[idx] @ v.t()
        if d["bias"] is not None:
            y += d["bias"].double()
        if case["relu"]:
            y = y.clamp(min=0)
        out = {"y": y}
        if case["save"]:
            t = torch.zeros(m, r, dtype=torch.float64, device=dev)
            for k, idx in rows.items():
                if k >= 0:
                    t[idx] = x[idx] @ d["down"][k].double().t()
            out["t"] = t
        return out
    dx = torch.zeros(m, n_in, dtype=torch.float64, device=dev)
    ddown = torch.zeros(g, r, n_in, dtype=torch.float64, device=dev)
    dup = torch.zeros(g, r, n_out, dtype=torch.float64, device=dev)
    for c in range(0, n_out, _CHUNK):
        w = d["w"][c:c + _CHUNK].double()
        dy = d["dy"][:, c:c + _CHUNK].double()
        for k, idx in rows.items():
            if k < 0:
                dx[idx] += dy[idx] @ w
                continue
            up, down = d["up"][k][:, c:c + _CHUNK].double(), d["down"][k].double()
            dx[idx] += dy[idx] @ (w + scale[k] * (up.t() @ down))
            ddown[k] += scale[k] * (up @ (dy[idx].t() @ x[idx]))
            # t is an input: what the forward saved, in 32 bits
            dup[k][:, c:c + _CHUNK] = scale[k] * (d["t"][idx].double().t() @ dy[idx])
    out = {"ddown": ddown, "dup": dup}
    if case["dx"]:
        out["dx"] = dx * (x > 0) if case["mask"] else dx
    return out


def _list_exact(case, seed):
    d = _list_inputs(case, seed)
    g = d["g"].double()
    norm = float(torch.linalg.vector_norm(g))
    c = min(1.0, d["max_norm"] / norm) if norm > 0 else 1.0
    g = g * c
    out_norm = torch.tensor([norm], dtype=torch.float64, device=g.device)
    if case["kind"] == "clip":
        return {"norm": out_norm, "g": g}
    t = d["t"] + 1
    m = BETA1 * d["m"].double() + (1 - BETA1) * g
    v = BETA2 * d["v"].double() + (1 - BETA2) * g ** 2
    p = d["p"].double() - LR * (m / (1 - np.power(BETA1, t))) / (torch.sqrt(v / (1 - np.power(BETA2, t))) + EPS)
    out = {"norm": out_norm, "p": p, "m": m, "v": v}
    if case["copies"]:
        out["copies"] = p
    return out


def exact(case, seed):
    if case["kind"] in ("forward", "backward"):
        return _layer_exact(case, seed)
    return _list_exact(case, seed)
