"""The operators on node rows that stand between two aggregations of a model, as cases that can be measured.

A case is a frame's worth of node rows (n nodes, k snapshots, a width), how they are stored, and one operator:

  ff             the gated feed-forward block, forward: Y = (act(X Wg + bg) * (X Wu + bu)) Wd + bd
  ff_backward    its gradients from X and dY: dX and those of the three matrices and the three biases
  norm           R' = R + scale * sigmoid(gate) * post(B), Z = pre(R'): the norm after a block, its gate and
                 residual scale, and the norm before the next block
  norm_backward  its gradients from R', dR' and dZ (and B, gate): dR, dB, dgate, and those of the scale and of both norms

Sizes are those of the benchmark workloads, of the tests and of what lies between (1 to 8 million rows, 2 to 256
columns, hidden widths that are 8/3 or 4 times the row's and odd ones).  `layout` "list" is one matrix per snapshot,
its rows dense; "padded" the same with the row stride that aggregations like; "wide" the concatenated operand [n, k, F].
"""
import math

import torch

own = False  # False: elementary torch operations; True: the framework's operators

DEVICE = "cuda:0"

# What a drawn case may cost: the products of the large feed-forward cases, and the bytes of the large norm.
MOST_FLOPS = 5.2e11
MOST_ELEMENTS = 1_000_000 * 8 * 64
EPS = 1e-5


def _ff(name, op, n, k, feat, hidden, out, act, layout="list", bias=True):
    return _named(name, {"op": op, "n": n, "k": k, "feat": feat, "hidden": hidden, "out": out, "act": act, "layout": layout,
                         "bias": bias})


def _norm(name, op, n, k, feat, post, pre, gate=True, layout="list", bias=False):
    return _named(name, {"op": op, "n": n, "k": k, "feat": feat, "post": post, "pre": pre, "gate": gate, "layout": layout,
                         "bias": bias})


def _named(name, c):
    return {"name": name, **c} if name else c


def listed():
    return [
        # one node's row scored when its features change: what a call costs
        _ff("ff one row", "ff", 1, 1, 64, 256, 64, "silu"),
        # the tiny workload, concatenated, a hidden width of 8/3 of the row's
        _ff("ff tiny", "ff", 2_000, 4, 16, 43, 16, "relu", layout="wide"),
        # the medium workload's hidden layer
        _ff("ff medium", "ff", 200_000, 8, 64, 256, 64, "gelu", layout="padded"),
        # the large workload, 8/3 of the row's width, no biases
        _ff("ff large", "ff", 1_000_000, 8, 64, 171, 64, "silu", bias=False),
        # training on the small workload
        _ff("ff back small", "ff_backward", 20_000, 4, 32, 128, 32, "silu"),
        # training on the medium workload
        _ff("ff back medium", "ff_backward", 200_000, 8, 64, 256, 64, "silu", bias=False),
        # wide rows in, narrower ones out, sizes that divide nothing
        _ff("ff back ragged", "ff_backward", 62_503, 5, 128, 341, 100, "gelu"),
        # a few nodes scored: what a call costs
        _norm("norm few rows", "norm", 7, 1, 64, "rms", "rms"),
        # the large workload
        _norm("norm large", "norm", 1_000_000, 8, 64, "rms", "rms"),
        # wide rows that no vector load fits
        _norm("norm odd", "norm", 50_001, 3, 253, "layer", "layer", gate=False, bias=True),
        # training on the medium workload
        _norm("norm back medium", "norm_backward", 200_000, 8, 64, "rms", "rms", layout="padded"),
        # training on wide rows with everything that can be learnt
        _norm("norm back wide", "norm_backward", 500_000, 8, 128, "layer", "layer", bias=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["ff", "ff_backward", "norm", "norm_backward"])
    k = rng.randint(1, 16)
    feat = rng.choice([_log(rng, 2, 256), rng.choice([16, 32, 64, 128])])
    layout = rng.choice(["list", "padded", "wide"])
    if op.startswith("ff"):
        out = rng.choice([feat, _log(rng, 2, 256)])
        hidden = min(1024, max(8, rng.choice([4 * feat, 8 * feat // 3, _log(rng, 8, 1024)])))
        products = 2 * feat + out if op == "ff" else 6 * feat + 2 * out
        rows = _log(rng, 1, max(1, min(MOST_FLOPS / (2 * hidden * products), MOST_ELEMENTS / max(feat, out, 64))))
        # (not relu backward: its gradient jumps where G changes sign, and which side of it a value of 1e-8 lies on is rounding)
        act = rng.choice(["sigmoid", "gelu", "silu", "relu"][:4 if op == "ff" else 3])
        return _ff(None, op, max(1, rows // k), k, feat, hidden, out, act, layout, rng.random() < 0.5)
    rows = _log(rng, 1, MOST_ELEMENTS / max(feat, 64))
    return _norm(None, op, max(1, rows // k), k, feat, rng.choice(["rms", "layer", "none"]), rng.choice(["rms", "layer"]),
                 rng.random() < 0.7, layout, rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _room(case, width):
    """Memory for node rows: [k, n, width] or, concatenated, [n, k, width]."""
    n, k = case["n"], case["k"]
    if case["layout"] == "wide":
        return torch.empty((n, k, width), device=DEVICE)
    stride = width
    if case["layout"] == "padded":
        stride = 32 * ((width + 31) // 32 | 1) if width > 32 else 1 << (width - 1).bit_length()
    return torch.empty((k, n, stride), device=DEVICE)[:, :, :width]


def _operand(rows, case):
    """Node rows as a program of the framework holds them: k matrices, or the concatenated operand."""
    return rows if case["layout"] == "wide" else list(rows.unbind(0))


def _vector(gen, width, low, high):
    return torch.empty(width, device=DEVICE).uniform_(low, high, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    feat, op = case["feat"], case["op"]
    s = {"case": case}
    if op.startswith("ff"):
        hidden, out = case["hidden"], case["out"]
        given = {"X": (feat, 1.0), "dY": (out, 1e-2)} if op == "ff_backward" else {"X": (feat, 1.0)}
        made = {"dX": feat} if op == "ff_backward" else {"Y": out}
        for name, rows, columns in (("Wg", feat, hidden), ("Wu", feat, hidden), ("Wd", hidden, out)):
            s[name] = torch.empty((rows, columns), device=DEVICE).uniform_(-1, 1, generator=gen).mul_(math.sqrt(3.0 / rows))
        for name, columns in (("bg", hidden), ("bu", hidden), ("bd", out)):
            s[name] = _vector(gen, columns, -0.2, 0.2) if case["bias"] else None
    else:
        given, made = {"R": (feat, 1.0), "B": (feat, 1.0), "gate": (feat, 1.0)}, {"R_out": feat, "Z": feat}
        if op == "norm_backward":
            given.update(dR_out=(feat, 1e-2), dZ=(feat, 1e-2))
            made = {"dR": feat, "dB": feat, "dgate": feat}
        if not case["gate"]:
            given.pop("gate")
            made.pop("dgate", None)
        s["scale"] = _vector(gen, feat, 0.05, 0.5)
        s["w_post"] = _vector(gen, feat, 0.5, 1.5) if case["post"] != "none" else None
        s["b_post"] = _vector(gen, feat, -0.5, 0.5) if case["post"] != "none" and case["bias"] else None
        s["w_pre"] = _vector(gen, feat, 0.5, 1.5)
        s["b_pre"] = _vector(gen, feat, -0.5, 0.5) if case["bias"] else None
    # node rows are normally distributed; a program that runs epoch after epoch keeps the memory of its results, too
    for name, (width, scale) in given.items():
        s[name] = _room(case, width).normal_(0, scale, generator=gen)
    for name, width in made.items():
        s[name] = _room(case, width)
    s["operands"] = {name: _operand(s[name], case) for name in (*given, *made)}
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------------


def _act(name, g):
    if name == "relu":
        return torch.clamp(g, min=0)
    if name == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    sig = 1 / (1 + torch.exp(-g))
    return sig if name == "sigmoid" else g * sig


def _act_slope(name, g):
    if name == "relu":
        return (g > 0).to(g.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    sig = 1 / (1 + torch.exp(-g))
    return sig * (1 - sig) if name == "sigmoid" else sig * (1 + g * (1 - sig))


def _times(a, w, b):
    return a @ w if b is None else a @ w + b


def _column_sums(a):
    return a.reshape(-1, a.shape[-1]).sum(0, dtype=torch.float64).float()


def _over_rows(a, b):
    """a^T b over all rows, summed in pieces of up to 8192 rows and over these in 64 bits."""
    a, b = a.reshape(-1, a.shape[-1]), b.reshape(-1, b.shape[-1])
    whole = a.shape[0] // 8192 * 8192
    pieces = torch.bmm(a[:whole].view(-1, 8192, a.shape[1]).transpose(1, 2), b[:whole].view(-1, 8192, b.shape[1]))
    return (pieces.sum(0, dtype=torch.float64) + a[whole:].T @ b[whole:]).float()


def _ff_plain(s):
    c = s["case"]
    h = _act(c["act"], _times(s["X"], s["Wg"], s["bg"])) * _times(s["X"], s["Wu"], s["bu"])
    return {"Y": _times(h, s["Wd"], s["bd"])}


def _ff_backward_plain(s):
    c, x, dy = s["case"], s["X"], s["dY"]
    g, u = _times(x, s["Wg"], s["bg"]), _times(x, s["Wu"], s["bu"])
    a = _act(c["act"], g)
    dh = dy @ s["Wd"].T
    du, dg = dh * a, dh * u * _act_slope(c["act"], g)
    o = {"dX": dg @ s["Wg"].T + du @ s["Wu"].T, "dWg": _over_rows(x, dg), "dWu": _over_rows(x, du), "dWd": _over_rows(a * u, dy)}
    if c["bias"]:
        o.update(dbg=_column_sums(dg), dbu=_column_sums(du), dbd=_column_sums(dy))
    return o


def _unit(kind, x):
    """x normalised, and the factor that it was scaled by."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _unit_back(kind, d, x, r):
    d = d - x * (d * x).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - d.mean(-1, keepdim=True)
    return d * r


def _affine(x, w, b):
    return x * w if b is None else x * w + b


def _norm_plain(s):
    c, p = s["case"], s["B"]
    if c["post"] != "none":
        p = _affine(_unit(c["post"], p)[0], s["w_post"], s["b_post"])
    p = p * s["scale"]
    if c["gate"]:
        p = p / (1 + torch.exp(-s["gate"]))
    r = s["R"] + p
    return {"R_out": r, "Z": _affine(_unit(c["pre"], r)[0], s["w_pre"], s["b_pre"])}


def _norm_backward_plain(s):
    c = s["case"]
    r, f = _unit(c["pre"], s["R"])
    g = s["dR_out"] + _unit_back(c["pre"], s["dZ"] * s["w_pre"], r, f)
    o = {"dR": g, "dw_pre": _column_sums(s["dZ"] * r)}
    p = s["B"]
    if c["post"] != "none":
        b, f = _unit(c["post"], p)
        p = _affine(b, s["w_post"], s["b_post"])
    d = g * s["scale"]
    if c["gate"]:
        sig = 1 / (1 + torch.exp(-s["gate"]))
        o["dgate"] = d * p * sig * (1 - sig)
        d = d * sig
        o["dscale"] = _column_sums(g * sig * p)
    else:
        o["dscale"] = _column_sums(g * p)
    if c["post"] != "none":
        o["dw_post"] = _column_sums(d * b)
        if c["bias"]:
            o["db_post"] = _column_sums(d)
        d = _unit_back(c["post"], d * s["w_post"], b, f)
    o["dB"] = d
    if c["bias"]:
        o["db_pre"] = _column_sums(s["dZ"])
    return o


# ---- the framework's operators ----------------------------------------------------------------------------------------


def _run_own(s):
    import paper_2301_00391_amd as pipad
    c, m = s["case"], s["operands"]
    post = None if c.get("post") == "none" else c.get("post")
    if c["op"] == "ff":
        pipad.gated_ff(m["X"], s["Wg"], s["Wu"], s["Wd"], s["bg"], s["bu"], s["bd"], activation=c["act"], Y=m["Y"])
        return {"Y": s["Y"]}
    if c["op"] == "ff_backward":
        d = pipad.gated_ff_backward(m["X"], m["dY"], s["Wg"], s["Wu"], s["Wd"], s["bg"], s["bu"], activation=c["act"],
                                    biases=c["bias"], dX=m["dX"])
        o = {"dX": s["dX"], "dWg": d.dWg, "dWu": d.dWu, "dWd": d.dWd}
        if c["bias"]:
            o.update(dbg=d.dbg, dbu=d.dbu, dbd=d.dbd)
        return o
    if c["op"] == "norm":
        pipad.residual_norm(m["R"], m["B"], m.get("gate"), post=post, pre=c["pre"], scale=s["scale"], w_post=s["w_post"],
                            b_post=s["b_post"], w_pre=s["w_pre"], b_pre=s["b_pre"], eps=EPS, R_out=m["R_out"], Z=m["Z"])
        return {"R_out": s["R_out"], "Z": s["Z"]}
    d = pipad.residual_norm_backward(m["R"], m["dR_out"], m["dZ"], m["B"], m.get("gate"), post=post, pre=c["pre"], scale=s["scale"],
                                     w_post=s["w_post"], b_post=s["b_post"], w_pre=s["w_pre"], eps=EPS, biases=c["bias"],
                                     dR=m["dR"], dB=m["dB"], dgate=m.get("dgate"))
    o = {"dR": s["dR"], "dB": s["dB"], "dscale": d.dscale, "dw_pre": d.dw_pre}
    if c["gate"]:
        o["dgate"] = s["dgate"]
    if post:
        o["dw_post"] = d.dw_post
    if c["bias"]:
        o["db_pre"] = d.db_pre
        if post:
            o["db_post"] = d.db_post
    return o


def run(state):
    if own:
        return _run_own(state)
    return {"ff": _ff_plain, "ff_backward": _ff_backward_plain, "norm": _norm_plain, "norm_backward": _norm_backward_plain}[
        state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------


def work(case):
    rows, feat = case["n"] * case["k"], case["feat"]
    if case["op"].startswith("ff"):
        hidden, out = case["hidden"], case["out"]
        weights = hidden * (2 * feat + out) + (2 * hidden + out if case["bias"] else 0)
        if case["op"] == "ff":
            return {"bytes": 4 * (rows * (feat + out) + weights), "flops": 2 * rows * hidden * (2 * feat + out)}
        return {"bytes": 4 * (rows * (2 * feat + out) + 2 * weights), "flops": 2 * rows * hidden * (6 * feat + 2 * out)}
    gate = 1 if case["gate"] else 0
    matrices, per_element = (4 + gate, 16) if case["op"] == "norm" else (6 + 2 * gate, 40)
    return {"bytes": 4 * rows * feat * matrices, "flops": rows * feat * per_element}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------


def exact(case, seed):
    """By reverse differentiation of the formulas in 64 bits, a piece of the rows at a time."""
    s = prepare(case, seed)
    feat, forward = case["feat"], not case["op"].endswith("backward")
    ff = case["op"].startswith("ff")
    learnt = ("Wg", "Wu", "Wd", "bg", "bu", "bd") if ff else ("scale", "w_post", "b_post", "w_pre", "b_pre")
    p = {q: None if s[q] is None else s[q].double().requires_grad_(not forward) for q in learnt}
    matrices = [q for q in ("X", "dY", "R", "B", "gate", "dR_out", "dZ") if (forward, q) != (True, "dZ") and q in s]
    flat = {q: s[q].reshape(-1, s[q].shape[-1]) for q in matrices}
    rows = case["n"] * case["k"]
    out, step = {}, max(1, 40_000_000 // (case["hidden"] if ff else feat))

    def unit(kind, x):
        if kind == "layer":
            return torch.nn.functional.layer_norm(x, (feat,), eps=EPS)
        return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() if kind == "rms" else x

    def affine(x, w, b):
        x = x if w is None else x * w
        return x if b is None else x + b

    for at in range(0, rows, step):
        v = {q: flat[q][at:at + step].double() for q in matrices}
        if ff:
            leaves = [v["X"]]
        else:
            leaves = [v[q] for q in ("R", "B", "gate") if q in v]
        for x in leaves:
            x.requires_grad_(not forward)
        if ff:
            act = {"relu": torch.relu, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}
            h = act[case["act"]](affine(v["X"] @ p["Wg"], None, p["bg"])) * affine(v["X"] @ p["Wu"], None, p["bu"])
            results = {"Y": affine(h @ p["Wd"], None, p["bd"])}
            if not forward:
                results["Y"].backward(v["dY"])
                results = {"dX": v["X"].grad}
        else:
            b = affine(unit(case["post"], v["B"]), p["w_post"], p["b_post"])
            b = p["scale"] * (torch.sigmoid(v["gate"]) * b if "gate" in v else b)
            if forward:
                r = v["R"] + b
                results = {"R_out": r, "Z": affine(unit(case["pre"], r), p["w_pre"], p["b_pre"])}
            else:  # R is what the forward pass gave: the sum's other term is not seen again
                z = affine(unit(case["pre"], v["R"]), p["w_pre"], p["b_pre"])
                z.backward(v["dZ"])
                total = v["dR_out"] + v["R"].grad
                b.backward(total)
                results = {"dR": total, "dB": v["B"].grad}
                if "gate" in v:
                    results["dgate"] = v["gate"].grad
        for q, x in results.items():
            out.setdefault(q, torch.empty((rows, x.shape[1]), dtype=torch.float64, device=DEVICE))[at:at + step] = x.detach()
    first = s["X"] if ff else s["R"]
    out = {q: x.view(*first.shape[:2], x.shape[1]) for q, x in out.items()}
    if not forward:
        out.update({"d" + q: x.grad for q, x in p.items() if x is not None})
    return out
