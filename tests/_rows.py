"""Helpers of the tests of the operators on node rows: operands in every layout, the operators' definitions in 64 bits, and what
32-bit arithmetic may be off by, derived rounding by rounding (first order, U = half a step)."""
import torch

U = 2.0 ** -24
LAYOUTS = ("list", "padded", "odd", "wide", "wide padded")


def room(layout, n, k, F, fill=77.0, device="cuda:0"):
    """An operand of n rows of F columns and what surrounds it: rows behind the last, columns behind the last."""
    if layout.startswith("wide"):
        whole = torch.full((n + 2, k + (2 if layout == "wide padded" else 0), F + (5 if layout == "wide padded" else 0)), fill, device=device)
        return whole, whole[:n, :k, :F]
    stride = {"list": F, "padded": (F + 31) // 32 * 32 + 32, "odd": F + 3 if F % 2 == 0 else F + 2}[layout]
    whole = torch.full((k, (n + 2) * stride + 1), fill, device=device)
    first = 1 if layout == "odd" else 0  # (rows off any 8- or 16-byte boundary)
    mats = whole[:, first:first + n * stride].unflatten(1, (n, stride))[:, :, :F]
    return whole, list(mats.unbind(0))


def stacked(x):
    """[n, k, F] or a list -> [k * n, F], snapshot after snapshot."""
    x = x.transpose(0, 1) if isinstance(x, torch.Tensor) else torch.stack(list(x))
    return x.reshape(-1, x.shape[-1])


def fill_with(x, values):
    """Writes [k, n, F] values into an operand."""
    if isinstance(x, torch.Tensor):
        x.copy_(values.transpose(0, 1))
    else:
        for m, v in zip(x, values):
            m.copy_(v)
    return x


def untouched(whole, part, fill=77.0):
    """Nothing but the operand was written."""
    seen = whole.clone()
    n, F = (part.shape[0], part.shape[-1]) if isinstance(part, torch.Tensor) else part[0].shape
    for m in ((part,) if isinstance(part, torch.Tensor) else part):
        at = (m.data_ptr() - whole.data_ptr()) // 4
        seen.view(-1).as_strided(m.shape, m.stride(), at).fill_(fill)
    return bool((seen == fill).all())


def within(got, want, bound, what):
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, first at {torch.nonzero(bad)[0].tolist()}, worst ratio "
                                 f"{float((err / bound.clamp(min=1e-300)).nan_to_num(posinf=1e30).max()):.3g}")


# ---- the gated feed-forward block --------------------------------------------------------------------------------------


def act(name, g):
    return {"relu": torch.relu, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[name](g)


def act_slope(name, g):
    g = g.detach().clone().requires_grad_(True)
    if name == "relu":
        return (g > 0).double().detach()
    act(name, g).sum().backward()
    return g.grad


#: the largest slope of each activation, and of its slope
SLOPES = {"sigmoid": (0.25, 0.1), "relu": (1.0, 0.0), "silu": (1.1, 0.5), "gelu": (1.13, 0.8)}


def steps(depth):
    """Roundings of a product of that depth, in U: six instructions for each 16 of it, one rounding each of a whole step (2 U) into the
    accumulator, the 16 sums within an instruction, and the piece products that are left out (2^-22) and 3 of each kind of slack for a
    bias, the sum of the parts and the store."""
    return 2 * (6 * ((depth + 15) // 16) + 16) + 4 + 6


def own_error(g):
    """Relative error of an activation computed from one exponential of g or g^2 / 2, in U: the argument's rounding comes out multiplied by the
    argument; the exponential, the reciprocal, the polynomial and four more operations 16."""
    return (g * g + 2 * g.abs() + 16) * U


class GatedFF:
    """Definition and bounds for x [rows, F] and float32 weights; all in 64 bits."""

    def __init__(self, x, Wg, Wu, Wd, bg, bu, bd, activation):
        d = lambda v, c: torch.zeros(c, dtype=torch.float64, device=x.device) if v is None else v.double()  # noqa: E731
        self.x, self.name = x.double(), activation
        self.Wg, self.Wu, self.Wd = Wg.double(), Wu.double(), Wd.double()
        self.bg, self.bu, self.bd = d(bg, Wg.shape[1]), d(bu, Wg.shape[1]), d(bd, Wd.shape[1])
        ax, cF = self.x.abs(), steps(Wg.shape[0]) * U
        self.G, self.Ug = self.x @ self.Wg + self.bg, self.x @ self.Wu + self.bu
        self.eG, self.eU = cF * (ax @ self.Wg.abs() + self.bg.abs()), cF * (ax @ self.Wu.abs() + self.bu.abs())
        self.a = act(activation, self.G)
        self.ea = SLOPES[activation][0] * self.eG + self.a.abs() * own_error(self.G)
        self.H = self.a * self.Ug
        self.eH = self.ea * self.Ug.abs() + self.a.abs() * self.eU + 2 * U * self.H.abs()

    def forward(self):
        c = steps(self.Wd.shape[0]) * U
        return self.H @ self.Wd + self.bd, self.eH @ self.Wd.abs() + c * (self.H.abs() @ self.Wd.abs() + self.bd.abs())

    def backward(self, dy):
        """{name: (gradient, bound)}"""
        dy, rows, hidden = dy.double(), self.x.shape[0], self.Wd.shape[0]
        dH, edH = dy @ self.Wd.T, steps(dy.shape[1]) * U * (dy.abs() @ self.Wd.abs().T)
        s = act_slope(self.name, self.G)
        es = SLOPES[self.name][1] * self.eG + (1.13 + self.G.abs()) * own_error(self.G) * (self.name != "relu")
        dU, edU = dH * self.a, edH * self.a.abs() + dH.abs() * self.ea + U * (dH * self.a).abs()
        dG = dH * self.Ug * s
        edG = edH * (self.Ug * s).abs() + (dH * s).abs() * self.eU + (dH * self.Ug).abs() * es + 3 * U * dG.abs()
        out = {"dX": (dG @ self.Wg.T + dU @ self.Wu.T, edG @ self.Wg.abs().T + edU @ self.Wu.abs().T +
                      steps(2 * hidden) * U * (dG.abs() @ self.Wg.abs().T + dU.abs() @ self.Wu.abs().T))}
        c = (steps(rows) + 64) * U  # (parts of the rows are added up behind the products)
        for q, a, b, eb in (("dWg", self.x, dG, edG), ("dWu", self.x, dU, edU)):
            out[q] = (a.T @ b, a.abs().T @ eb + c * (a.abs().T @ b.abs()))
        out["dWd"] = (self.H.T @ dy, self.eH.T @ dy.abs() + c * (self.H.abs().T @ dy.abs()))
        for q, b, eb in (("dbg", dG, edG), ("dbu", dU, edU), ("dbd", dy, torch.zeros_like(dy))):
            out[q] = (b.sum(0), eb.sum(0) + (rows + 64) * U * b.abs().sum(0))
        return out


# ---- the norms around a block --------------------------------------------------------------------------------------------


class Unit:
    """x normalised: value, factor, and what they may be off by when x is off by ex."""

    def __init__(self, kind, x, ex, eps):
        F = x.shape[1]
        self.kind, self.F = kind, F
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        if kind is None:
            self.v, self.e, self.r, self.er = x, ex, torch.ones_like(x[:, :1]), torch.zeros_like(x[:, :1])
            return
        c = x - mean(x) if kind == "layer" else x
        ec = ex + (mean(ex) + (F + 3) * U * (x.abs() + mean(x.abs())) if kind == "layer" else 0)
        var = mean(c * c)
        self.r = (var + eps).rsqrt()
        # relative: half of the variance's, which is that of F squares summed and of the errors of c; eps added, the root, 2 more
        self.er = 0.5 * self.r ** 2 * (2 * mean(c.abs() * ec) + (F + 3) * U * var) + 4 * U
        self.v = c * self.r
        self.e = ec * self.r + self.v.abs() * (self.er + U)

    def back(self, d, ed):
        """The gradient of x from that of the normalised value."""
        if self.kind is None:
            return d, ed
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        s, es = mean(d * self.v), mean(ed * self.v.abs() + d.abs() * self.e) + (self.F + 3) * U * mean((d * self.v).abs())
        m, em = torch.zeros_like(s), torch.zeros_like(s)
        if self.kind == "layer":
            m, em = mean(d), mean(ed) + (self.F + 3) * U * mean(d.abs())
        t = d - m - self.v * s
        et = ed + em + self.v.abs() * es + self.e * s.abs() + 3 * U * (d.abs() + m.abs() + (self.v * s).abs())
        return t * self.r, et * self.r + (t * self.r).abs() * (self.er + U)


class ResidualNorm:
    """Definition and bounds; rows are [rows, F] float32, vectors float32 or None.  `R`: the forward pass's input, or in `backward` its output."""

    def __init__(self, B, gate, post, pre, scale, w_post, b_post, w_pre, b_pre, eps):
        self.pre, self.eps, self.has_b = pre, eps, B is not None
        d = lambda v, o: o if v is None else v.double()  # noqa: E731
        self.scale, self.w_post, self.b_post, self.w_pre, self.b_pre = d(scale, 1.0), d(w_post, 1.0), d(b_post, 0.0), d(w_pre, 1.0), d(b_pre, 0.0)
        if not self.has_b:
            return
        B = B.double()
        self.b = Unit(post, B, torch.zeros_like(B), eps)
        self.p = self.b.v * self.w_post + self.b_post
        # (a vector that is not there is one more exact operation)
        self.ep = self.b.e * abs(self.w_post) + U * ((self.b.v * self.w_post).abs() + self.p.abs()) * (post is not None)
        if gate is None:
            self.sig, self.rest, self.es = torch.ones_like(B), None, torch.zeros_like(B)
        else:
            gate = gate.double()
            self.sig, self.rest = torch.sigmoid(gate), torch.sigmoid(-gate)
            self.es = (2 * gate.abs() + 8) * U  # relative

    def forward(self, R):
        R = R.double()
        r, er = R, torch.zeros_like(R)
        if self.has_b:
            q = self.scale * self.sig * self.p
            r = R + q
            er = abs(self.scale) * self.sig * self.ep + q.abs() * (self.es + 3 * U) + U * r.abs()
        z = Unit(self.pre, r, er, self.eps)
        return {"R_out": (r, er), "Z": (z.v * self.w_pre + self.b_pre, z.e * abs(self.w_pre) + 2 * U * ((z.v * self.w_pre).abs() + abs(self.b_pre)))}

    def backward(self, R_out, dR, dZ):
        zero = torch.zeros_like(R_out.double())
        rows = zero.shape[0]
        dR = zero if dR is None else dR.double()
        g, eg, out = dR, zero, {}
        total = lambda v, e: (v.sum(0), e.sum(0) + (rows + 64) * U * v.abs().sum(0))  # noqa: E731
        if dZ is not None:
            dZ = dZ.double()
            z = Unit(self.pre, R_out.double(), zero, self.eps)
            out["dw_pre"], out["db_pre"] = total(dZ * z.v, dZ.abs() * z.e + U * (dZ * z.v).abs()), total(dZ, zero)
            d, ed = z.back(dZ * self.w_pre, U * (dZ * self.w_pre).abs())
            g, eg = dR + d, ed + U * (dR + d).abs()
        out["dR"] = (g, eg)
        if not self.has_b:
            return out
        gp = g * self.sig * self.p
        out["dscale"] = total(gp, eg * (self.sig * self.p).abs() + (g * self.sig).abs() * self.ep + gp.abs() * (self.es + 3 * U))
        d = g * self.scale * self.sig
        ed = eg * (abs(self.scale) * self.sig).abs() + d.abs() * (self.es + 2 * U)
        if self.rest is not None:
            v = g * self.scale * self.p * self.sig * self.rest
            w = (self.scale * self.sig * self.rest)
            out["dgate"] = (v, eg * (w * self.p).abs() + (g * w).abs() * self.ep + v.abs() * (2 * self.es + 5 * U))
        if self.b.kind is not None:
            out["dw_post"], out["db_post"] = total(d * self.b.v, ed * self.b.v.abs() + d.abs() * self.b.e + U * (d * self.b.v).abs()), total(d, ed)
            d, ed = self.b.back(d * self.w_post, ed * abs(self.w_post) + U * (d * self.w_post).abs())
        out["dB"] = (d, ed)
        return out
