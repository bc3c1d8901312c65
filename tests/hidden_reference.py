"""Layer norm, dropout, embedding and router in 64 bits, and how far a result
may be from them (test infrastructure; shares no code with the library).

e is the unit roundoff of 32 bits.  A sum is off by at most e times the number
of additions that a term passes through, times the sum of the magnitudes; where
that number is not fixed by the operator's size, the number of terms bounds it.
A row of layer norm is dealt out over up to 1024 threads: a thread adds at most
16 values, or a 1024th of a longer row, and ten more additions join them.
"""

import torch

e = 2.0 ** -24


def depth(cols):
    return 32 + cols / 1024


def layer_norm(x, w, b, eps):
    """(mean, its bound), (rstd, its bound), (y, its bound)."""
    x = x.double()
    n = x.shape[1]
    mean = x.mean(1, keepdim=True)
    em = (depth(n) + 3) * e * x.abs().mean(1, keepdim=True)
    d = x - mean
    var = d.square().mean(1, keepdim=True)
    # every deviation is off by em and its rounding, the sum by its additions
    ev = (depth(n) + 8) * e * var + 2 * (em + e * d.abs().mean(1, keepdim=True)) * var.sqrt() + em ** 2
    rstd = (var + eps) ** -0.5
    # 1 / sqrt(1 - t) <= 1 + t up to a half; eps itself is rounded
    rel = (ev + e * eps) / (var + eps) + 6 * e
    assert not rel.numel() or rel.max() < 0.5
    v = d * rstd
    wd = 1.0 if w is None else w.double()
    bd = 0.0 if b is None else b.double()
    y = v * wd + bd
    lost = (em + e * d.abs()) * rstd * (1 + rel) + v.abs() * (rel + 2 * e)
    ey = lost * (wd if w is None else wd.abs()) + 2 * e * (y.abs() + (v * wd).abs())
    return (mean[:, 0], em[:, 0]), (rstd[:, 0], (rstd * rel)[:, 0]), (y, ey)


def layer_norm_grads(dy, x, w, mean, rstd, dres):
    """(dx, bound), (dw, bound), (dbias, bound); mean and rstd as the call gets them."""
    dy, x = dy.double(), x.double()
    rows, n = x.shape
    m, r = mean.double()[:, None], rstd.double()[:, None]
    v = (x - m) * r
    t = dy if w is None else dy * w.double()
    s0, s1 = t.mean(1, keepdim=True), (t * v).mean(1, keepdim=True)
    dx = r * (t - s0 - v * s1)
    e0 = (depth(n) + 4) * e * t.abs().mean(1, keepdim=True)
    e1 = (depth(n) + 8) * e * (t * v).abs().mean(1, keepdim=True)
    ex = r * (e0 + v.abs() * e1 + 8 * e * (t.abs() + s0.abs() + (v * s1).abs()))
    if dres is not None:
        dx = dx + dres.double()
        ex = ex + 2 * e * (dx.abs() + dres.double().abs())
    many = (rows + 8) * e
    return (dx, ex), ((dy * v).sum(0), (many + 4 * e) * (dy * v).abs().sum(0)), (dy.sum(0), many * dy.abs().sum(0))


# ------------------------------------------------------------------- dropout

MASK = 0xFFFFFFFF


def philox(counter, key):
    """Philox4x32-10 of Salmon, Moraes, Dror and Shaw (2011) on Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & MASK, (a >> 32) ^ c[3] ^ k[1], a & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def numbers(first, count, seed, offset, device="cpu"):
    """Those of the elements first .. first + count - 1, as int64."""
    four = torch.arange(first // 4, (first + count + 3) // 4, dtype=torch.int64, device=device)
    c = [four & MASK, four >> 32, torch.full_like(four, offset & MASK), torch.full_like(four, offset >> 32)]
    k = [seed & MASK, seed >> 32]
    for _ in range(10):
        hi, lo = [], []
        for v, m in ((c[0], 0xD2511F53), (c[2], 0xCD9E8D57)):
            # the product's 64 bits from two of 48, without a sign
            low, high = v * (m & 0xFFFF), v * (m >> 16)
            total = high + (low >> 16)
            hi.append(total >> 16)
            lo.append((total & 0xFFFF) << 16 | low & 0xFFFF)
        c = [hi[1] ^ c[1] ^ k[0], lo[1], hi[0] ^ c[3] ^ k[1], lo[0]]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return torch.stack(c, 1).view(-1)[first % 4:][:count]


def dropout(x, p, seed, offset, residual, first=0):
    """(y, bound) of elements that start at `first` of the whole."""
    least = min(round(p * 2 ** 32), 2 ** 32 - 1)
    keep = (numbers(first, x.numel(), seed, offset, x.device) >= least).view(x.shape)
    v = torch.where(keep, x.double() * (2.0 ** 32 / (2 ** 32 - least)), 0.0)
    y = v if residual is None else v + residual.double()
    return y, 2 * e * v.abs() + (e * y.abs() if residual is not None else 0 * v)


# ----------------------------------------------------------------- embedding

def embedding_rows(tokens, first, rows):
    """Each token's row of the table, `rows` for none."""
    at = tokens.long() - first
    return torch.where((at >= 0) & (at < rows) & (tokens >= 0), at, rows)


def embedding(tokens, table, scale, first):
    at = embedding_rows(tokens, first, table.shape[0])
    full = torch.cat((table.double(), torch.zeros(1, table.shape[1], dtype=torch.float64, device=table.device)))
    y = full[at] * scale
    return y, 2 * e * y.abs()


def embedding_grad(tokens, dy, rows, scale, first, base):
    at = embedding_rows(tokens, first, rows)

    def added(v):
        return torch.zeros(rows + 1, v.shape[1], dtype=torch.float64, device=v.device).index_add_(0, at, v)[:rows]

    terms = added(torch.ones(len(tokens), 1, dtype=torch.float64, device=dy.device))
    g, mag = added(dy.double()) * scale, added(dy.double().abs()) * abs(scale)
    bound = (terms + 4) * e * mag
    if base is not None:
        g = g + base.double()
        bound = bound + e * (g.abs() + base.double().abs())
    return g, bound


# -------------------------------------------------------------------- router

def router(logits, k, valid, normalize):
    """A dict of results and their bounds."""
    l = logits.double()
    t, n = l.shape
    ok = torch.ones(t, dtype=torch.bool, device=l.device) if valid is None else valid.bool()
    bad = ok & (l.isnan().any(1) | (l == float("inf")).any(1))
    dead = ~ok | (~bad & (l == float("-inf")).all(1))
    plain = ~bad & ~dead
    safe = torch.where(plain[:, None], l, 0.0)
    p = torch.softmax(safe, 1) * plain[:, None]
    order = torch.sort(safe, dim=1, descending=True, stable=True).indices[:, :k]
    chosen = torch.gather(safe, 1, order) > float("-inf")
    chosen &= plain[:, None]
    experts = torch.where(chosen, order, -1).int()
    w = torch.gather(p, 1, order) * chosen
    total = w.sum(1, keepdim=True)
    if normalize:
        w = torch.where(total > 0, w / total, 0.0)
    counts = torch.zeros(n + 1, dtype=torch.int64, device=l.device)
    counts.index_add_(0, torch.where(chosen, order, n).flatten(), chosen.flatten().long())
    took = int((~dead).sum())
    counts[n] = took
    many = max(took, 1)
    loss = n * (counts[:n].double() / (k * many) * p.sum(0) / many).sum()
    # the exponential's argument is rounded, itself and the sum are off by a few units
    top = safe.amax(1, keepdim=True)
    span = torch.where(safe > float("-inf"), (top - safe), 0.0).amax(1, keepdim=True)
    rel = (span + 64) * e
    w = torch.where(bad[:, None], float("nan"), w)
    if bad.any():
        loss = torch.full_like(loss, float("nan"))
    return dict(experts=experts, weights=w, eweights=2 * rel * w.abs() + 0 * w, counts=counts.int(), loss=loss[None],
                eloss=loss.abs()[None] * ((took + 32) * e + float(rel.max() if t else 0)), p=p, rel=rel, plain=plain,
                bad=bad, total=total)


def router_grad(r, logits, k, normalize, dweights, dloss):
    """(dlogits, bound) from what router() gave and the gradients of weights and loss."""
    t, n = logits.shape
    p, c = r["p"], r["counts"].double()
    many = max(float(c[n]), 1.0)
    dp = torch.zeros_like(p)
    size = torch.zeros_like(p)
    if dloss is not None:
        dp += dloss.double() * n * c[:n] / (k * many) / many
        size += dp.abs()
    if dweights is not None:
        d, w = dweights.double(), torch.nan_to_num(r["weights"])
        mag = d.abs()
        if normalize:
            mean = (d * w).sum(1, keepdim=True)
            over = torch.where(r["total"] > 0, 1 / r["total"], 0.0)
            mag = (mag + (mag * w.abs()).sum(1, keepdim=True)) * over
            d = (d - mean) * over
        chosen = r["experts"] >= 0
        at = torch.where(chosen, r["experts"].long(), 0)
        dp.scatter_add_(1, at, d * chosen)
        size.scatter_add_(1, at, mag * chosen)
    s = (p * dp).sum(1, keepdim=True)
    g = p * (dp - s)
    bound = p * (4 * r["rel"] + 64 * e) * (size + (p * size).sum(1, keepdim=True))
    g = torch.where(r["bad"][:, None], float("nan"), g)
    return g, bound
