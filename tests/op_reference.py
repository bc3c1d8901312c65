"""The layer operators' definitions in 64 bits, and how far a result may be
from them (test infrastructure; shares no code with the library).

Bounds: u is the unit roundoff of the element type (2^-8 for bfloat16, 2^-11
for float16, 2^-24 for float32).  A sum of K products in 32 bits is off by at
most (K + 8) 2^-24 times the sum of the products' magnitudes (any order); an
operand rounded to the element type on its way adds u times the same sum; the
result's own rounding adds u times its magnitude.  Rounding below the type's
normal range, of an operand as of a result, is off by up to half a subnormal
step (`TINY`) instead.
"""

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
EPS32 = 2.0 ** -24


def act(z, name):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z.clamp(min=0) if name == "relu" else z


def slope(z, name):
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return (z > 0).double() if name == "relu" else torch.ones_like(z)


# Largest magnitudes of the activations' first and second derivatives
# (rounded up): an error e of z moves act(z) by at most STEEP e and act'(z) by
# at most BEND e.  relu's slope jumps: its inputs are kept away from zero.
STEEP = {"none": 1.0, "relu": 1.0, "silu": 1.1, "gelu": 1.13}
BEND = {"none": 0.0, "relu": 0.0, "silu": 0.51, "gelu": 0.81}
# expf, erff and their use: a few units of 32 bits of the value and its argument
CALLS = 16 * EPS32


def product(a, b, rounded=None):
    """a b^T and the bound of its sum; `rounded`: the type that a is rounded to on its way."""
    v, mag = a @ b.T, a.abs() @ b.abs().T
    bound = (a.shape[1] + 8) * EPS32 * mag
    if rounded is not None:
        bound = bound + U[rounded] * mag + TINY[rounded] * b.abs().sum(1)
    return v, bound


def close(got, want, bound, what):
    u, tiny = U[got.dtype], TINY[got.dtype]
    g = got.double()
    assert g.shape == want.shape, what
    assert torch.equal(torch.isfinite(g), torch.isfinite(want)), "%s: finite values differ" % what
    fin = torch.isfinite(want)
    assert torch.equal(g[~fin], want[~fin]), what
    over = (g - want).abs()[fin] - (bound + (u * (want.abs() + bound)) + tiny)[fin]
    if over.numel():
        worst = over.max().item()
        assert worst <= 0, "%s: %.3g beyond its bound" % (what, worst)


def linear(x, w, bias, residual, name):
    x, w = x.double(), w.double()
    z, ez = product(x, w)
    if bias is not None:
        z = z + bias.double()
        ez = ez + EPS32 * z.abs()
    y, ey = act(z, name), STEEP[name] * ez + CALLS * z.abs()
    if residual is not None:
        y = y + residual.double()
        ey = ey + EPS32 * y.abs()
    return z, ez, y, ey


def linear_grads(dy, x, w, z, ez, name):
    """(dx, dw, dbias) with their bounds; z is off by ez."""
    r = dy.dtype if name != "none" else None
    dy, x, w = dy.double(), x.double(), w.double()
    dz = dy * slope(z, name)
    edz = dy.abs() * (BEND[name] * ez + CALLS * (1 + z.abs())) if name != "none" else torch.zeros_like(dy)
    dx, ex = product(dz, w.T, r)
    dw, ew = product(dz.T, x.T, r)
    db, eb = dz.sum(0), edz.sum(0) + (dz.shape[0] + 8) * EPS32 * dz.abs().sum(0)
    return (dx, ex + 1.01 * (edz @ w.abs())), (dw, ew + 1.01 * (edz.T @ x.abs())), (db, eb)


def gated(x, wg, wu, name):
    g, eg = product(x.double(), wg.double())
    p, ep = product(x.double(), wu.double())
    a, ea = act(g, name), STEEP[name] * eg + CALLS * g.abs()
    return g, eg, p, ep, a * p, ea * p.abs() + (a.abs() + ea) * ep + 2 * EPS32 * (a * p).abs()


def gated_grads(dy, x, wg, wu, g, eg, p, ep, name):
    u = dy.dtype
    dy, x, wg, wu = dy.double(), x.double(), wg.double(), wu.double()
    s, a = slope(g, name), act(g, name)
    es = BEND[name] * eg + CALLS * (1 + g.abs())
    ea = STEEP[name] * eg + CALLS * g.abs()
    dg, du = dy * p * s, dy * a
    edg = dy.abs() * (p.abs() * es + (s.abs() + es) * ep) + 2 * EPS32 * dg.abs()
    edu = dy.abs() * ea + EPS32 * du.abs()
    dx1, e1 = product(dg, wg.T, u)
    dx2, e2 = product(du, wu.T, u)
    dwg, eg2 = product(dg.T, x.T, u)
    dwu, eu2 = product(du.T, x.T, u)
    k = (2 * dy.shape[1] + 8) * EPS32  # both terms run through one sum
    ex = e1 + e2 + k * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()) + 1.01 * (edg @ wg.abs() + edu @ wu.abs())
    return (dx1 + dx2, ex), (dwg, eg2 + 1.01 * edg.T @ x.abs()), (dwu, eu2 + 1.01 * edu.T @ x.abs())


def turn(v, cos, sin, rot, interleaved, sign=1):
    h = rot // 2
    out = v.clone()
    a, b = (v[..., 0:rot:2], v[..., 1:rot:2]) if interleaved else (v[..., :h], v[..., h:rot])
    ra, rb = a * cos - sign * b * sin, b * cos + sign * a * sin
    if interleaved:
        out[..., 0:rot:2], out[..., 1:rot:2] = ra, rb
    else:
        out[..., :h], out[..., h:rot] = ra, rb
    return out


def norm_rope(x, w, cos, sin, rot, interleaved, eps):
    x, w = x.double(), w.double()
    xh = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    v = xh * w
    y = turn(v, cos, sin, rot, interleaved) if rot else v
    d = x.shape[-1]
    # the mean's relative error, halved by the root, the root, three products
    # and the turn's two; a pair's magnitude bounds both of its values
    rel = (d / 2 + 24) * EPS32
    mag = turn(v.abs(), cos.abs(), sin.abs(), rot, interleaved, -1) if rot else v.abs()
    if rot:
        mag = torch.maximum(mag, turn(v.abs(), cos.abs(), sin.abs(), rot, interleaved, 1).abs())
    return y, rel * mag


def norm_rope_grads(dy, x, w, cos, sin, rot, interleaved, eps):
    dy, x, w = dy.double(), x.double(), w.double()
    d = x.shape[-1]
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    xh = x * r
    dv = turn(dy, cos, sin, rot, interleaved, -1) if rot else dy
    mv = dy.abs()
    if rot:
        mv = torch.maximum(turn(dy.abs(), cos.abs(), sin.abs(), rot, interleaved, -1),
                           turn(dy.abs(), cos.abs(), sin.abs(), rot, interleaved, 1)).abs()
    t = dv * w
    mean = (t * xh).mean(-1, keepdim=True)
    dx = r * (t - xh * mean)
    rel = (d + 48) * EPS32
    mmean = (mv * w.abs() * xh.abs()).mean(-1, keepdim=True)
    ex = rel * r * (mv * w.abs() + xh.abs() * mmean)
    axes = tuple(range(x.dim() - 1))
    rows = x.numel() // d
    dw = (dv * xh).sum(axes)
    ew = (rows + d + 48) * EPS32 * (mv * xh.abs()).sum(axes)
    return (dx, ex), (dw, ew)


def visible(tq, tk, n_q, n_k, window, sinks, device):
    i = torch.arange(tq, device=device)[:, None]
    j = torch.arange(tk, device=device)[None, :]
    pos = n_k - n_q + i
    ok = (j <= pos) & (j < n_k) & (i < n_q)
    if window:
        ok &= (pos - j < window) | (j < sinks)
    return ok


def attention(q, k, v, n_q, n_k, window, sinks, scale, do=None):
    """One head of one sequence: dict of value and bound for o, lse and, with
    do, dq, dk, dv.  q [tq][d], k, v [tk][d]; keys past n_k are not read."""
    u, tiny = U.get(q.dtype, 0.0), TINY.get(q.dtype, 0.0)
    tq, d = q.shape
    tk = k.shape[0]
    ok = visible(tq, tk, n_q, n_k, window, sinks, q.device)
    live = torch.arange(tk, device=q.device)[:, None] < n_k
    q, k, v = q.double(), torch.where(live, k.double(), 0.0), torch.where(live, v.double(), 0.0)
    here = torch.arange(tq, device=q.device)[:, None] < n_q
    q = torch.where(here, q, 0.0)
    s = (q @ k.T * scale).masked_fill(~ok, -math.inf)
    es = (d + 8) * EPS32 * abs(scale) * (q.abs() @ k.abs().T)
    es = torch.where(ok, es + 4 * EPS32 * s.abs().masked_fill(~ok, 0.0), 0.0)
    some = ok.any(1, keepdim=True)
    top = torch.where(some, s.amax(1, keepdim=True) if tk else torch.zeros_like(q[:, :1]), 0.0)
    total = torch.exp(s - top).sum(1, keepdim=True)
    lse = torch.where(some, top + torch.log(total), -math.inf)
    p = torch.where(ok, torch.exp(s - torch.where(some, lse, 0.0)), 0.0)
    row = es.amax(1, keepdim=True) if tk else torch.zeros_like(top)
    # a weight is off by its score's error and the sum's (weighted mean of the
    # scores' errors), the exponential's (2^-21 of its value, and 2^-22 of its
    # argument's magnitude) and 32-bit sums over the keys
    dist = torch.where(ok, (top - s).masked_fill(~ok, 0.0), 0.0)
    rel = 2.1 * row + 2.0 ** -20 + 2.0 ** -22 * (dist + top.abs()) + (tk + 8) * EPS32
    o = p @ v
    # weights are rounded relative to the largest one met so far, 2^8 times the
    # largest at most, and divided by their sum, at least that largest
    step = torch.where(ok, 2.0 ** 8 * tiny, 0.0)
    out = {"o": (o, ((u + rel) * p + step) @ v.abs()),
           "lse": (lse[:, 0], torch.where(some, 2 * row + 2.0 ** -20 + (tk + 8) * EPS32 + 4 * EPS32 * lse.abs(), 0.0)[:, 0])}
    if do is None:
        return out
    do = torch.where(here, do.double(), 0.0)
    dp = do @ v.T
    delta = (do * o).sum(1, keepdim=True)
    edp = (d + 8) * EPS32 * (do.abs() @ v.abs().T)
    # delta comes from the rounded o
    edelta = (u * do.abs() * o.abs() + do.abs() * out["o"][1] * (1 + u)).sum(1, keepdim=True) \
        + (d + 8) * EPS32 * (do * o).abs().sum(1, keepdim=True)
    ds = p * (dp - delta) * scale
    # the weight again from the stored lse: score's error twice, lse's, exponential's
    relp = rel + 4 * EPS32 * torch.where(some, lse, 0.0).abs() + out["lse"][1][:, None]
    eds = abs(scale) * p * (relp * (dp.abs() + delta.abs()) + (1 + relp) * (edp + edelta)) + 4 * EPS32 * ds.abs()
    n = (max(tk, tq) + 8) * EPS32
    here_step = torch.where(ok, tiny * max(1.0, abs(scale)), 0.0)
    out["dq"] = (ds @ k, (u * ds.abs() + (1 + u) * eds + n * ds.abs() + here_step) @ k.abs())
    out["dk"] = (ds.T @ q, (u * ds.abs() + (1 + u) * eds + n * ds.abs() + here_step).T @ q.abs())
    out["dv"] = (p.T @ do, ((u + (1 + u) * relp + n) * p + here_step).T @ do.abs())
    return out
