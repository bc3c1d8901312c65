"""What a hidden state passes through between the products, as cases to time
and to compare: layer norm, dropout into the residual stream, the embedding
and an expert layer's router, forward and backward.  A plain form of each in
elementary 32-bit torch operations, the calls of the library's own (``own``),
and the operators' definitions in 64 bits.

Sizes are those of the workloads the library prices (hidden 4096 and 8192,
sequences of 2048 and 4096, 64 experts of which a token takes two), single
tokens and ragged ones."""

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # one token's hidden state ahead of attention
        dict(name="norm-token", op="norm", rows=1, cols=4096, bias=True, residual=False, backward=False, dtype="bf16"),
        # a training step's norm: hidden 8192, four sequences of 4096, the residual path's gradient added
        dict(name="norm-train", op="norm", rows=16384, cols=8192, bias=True, residual=True, backward=True,
             dtype="bf16"),
        # 32 bits, rows of no 16-byte multiple, a weight without a bias
        dict(name="norm-odd-fp32", op="norm", rows=4001, cols=2047, bias=False, residual=False, backward=True,
             dtype="fp32"),
        # a small micro-batch of a narrow model
        dict(name="dropout-small", op="dropout", rows=64, cols=1024, p=0.1, residual=True, backward=False,
             dtype="fp16"),
        # a training step's dropout into the residual stream: hidden 8192, four sequences of 4096
        dict(name="dropout-train", op="dropout", rows=16384, cols=8192, p=0.1, residual=True, backward=True,
             dtype="bf16"),
        # 32 bits, odd sizes, inside a block: no residual
        dict(name="dropout-odd-fp32", op="dropout", rows=4095, cols=2049, p=0.35, residual=False, backward=True,
             dtype="fp32"),
        # a decoding step's tokens
        dict(name="embed-tokens", op="embedding", t=16, shards=1, vocab=32000, cols=4096, scale=1.0, padded=False,
             backward=False, dtype="bf16"),
        # a training step of four sequences of 4096, a large vocabulary
        dict(name="embed-train", op="embedding", t=16384, shards=1, vocab=131072, cols=4096, scale=64.0, padded=False,
             backward=True, dtype="bf16"),
        # an eighth of the vocabulary, as a tensor-parallel shard holds it, padded sequences, odd sizes
        dict(name="embed-shard-odd", op="embedding", t=32771, shards=8, vocab=50008, cols=1023, scale=32.0,
             padded=True, backward=True, dtype="fp16"),
        # a decoding step's tokens choose their experts
        dict(name="router-tokens", op="router", t=16, experts=64, k=2, valid=False, normalize=True, backward=False,
             dtype="bf16"),
        # a training step of four sequences of 4096 through an expert layer
        dict(name="router-train", op="router", t=16384, experts=64, k=2, valid=False, normalize=True, backward=True,
             dtype="bf16"),
        # many small experts, logits in 32 bits, padded sequences
        dict(name="router-many-fp32", op="router", t=32771, experts=250, k=8, valid=True, normalize=False,
             backward=True, dtype="fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "dropout", "embedding", "router"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    backward = rng.random() < 0.7
    if op == "router":
        experts = rng.choice([_log(rng, 2, 512), rng.choice([8, 16, 64, 128, 256])])
        return dict(op=op, t=_log(rng, 1, 32768), experts=experts, k=min(experts, rng.choice([1, 2, 2, 4, 6, 8])),
                    valid=rng.random() < 0.4, normalize=rng.random() < 0.6, backward=backward, dtype=dtype)
    cols = _log(rng, 64, 8192)
    if rng.random() < 0.6:
        cols = cols // 64 * 64
    if op == "embedding":
        shards = rng.choice([1, 1, 2, 4, 8])
        vocab = _log(rng, 500, 131072) // shards * shards
        cols = min(cols, 4096)
        return dict(op=op, t=_log(rng, 1, 16384), shards=shards, vocab=vocab, cols=cols,
                    scale=rng.choice([1.0, round(cols ** 0.5 * 64) / 64]), padded=rng.random() < 0.4,
                    backward=backward, dtype="bf16" if dtype == "fp32" and vocab * cols > 2 ** 28 else dtype)
    rows = _log(rng, 1, 16384)
    if dtype == "fp32":
        rows = max(1, rows // 2)
    if op == "norm":
        return dict(op=op, rows=rows, cols=cols, bias=rng.random() < 0.7, residual=backward and rng.random() < 0.5,
                    backward=backward, dtype=dtype)
    return dict(op=op, rows=rows, cols=cols, p=rng.choice([0.05, 0.1, 0.1, 0.35, 0.5]), residual=rng.random() < 0.6,
                backward=backward, dtype=dtype)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def rand(*shape, std=1.0, to=dt):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(to)

    s = {"case": c}
    if c["op"] == "norm":
        m, n = c["rows"], c["cols"]
        # a hidden state has a mean of its own and a few channels far larger than the others
        far = 1 + 20 * (torch.rand(n, generator=g, device="cuda") < 0.002).float()
        s.update(x=(torch.randn(m, n, generator=g, device="cuda") * far + 0.3).to(dt), w=(1 + rand(n, std=0.1)),
                 b=rand(n, std=0.1) if c["bias"] else None)
        if c["backward"]:
            s.update(dy=rand(m, n), dres=rand(m, n) if c["residual"] else None)
    elif c["op"] == "dropout":
        m, n = c["rows"], c["cols"]
        s.update(x=rand(m, n), residual=rand(m, n) if c["residual"] else None, seed=seed * 0x9E3779B97F4A7C15 % 2 ** 64,
                 offset=seed % 1000)
        if c["backward"]:
            s["dy"] = rand(m, n)
    elif c["op"] == "embedding":
        t, vocab, n = c["t"], c["vocab"], c["cols"]
        rows = vocab // c["shards"]
        # words' frequencies fall off with their rank, and ranks lie anywhere in the vocabulary
        u = torch.rand(t, generator=g, device="cuda", dtype=torch.float64)
        rank = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp(0, vocab - 1)
        tokens = torch.randperm(vocab, generator=g, device="cuda")[rank]
        if c["padded"]:  # sequences of 128 that end early
            at = torch.arange(t, device="cuda")
            ends = torch.randint(64, 129, (t // 128 + 1,), generator=g, device="cuda")
            tokens = torch.where(at % 128 < ends[at // 128], tokens, torch.full_like(tokens, -1))
        s.update(tokens=tokens.int(), table=rand(rows, n), first=rows * (c["shards"] // 2))
        if c["backward"]:
            s["dy"] = rand(t, n)
    else:
        t, e = c["t"], c["experts"]
        # some experts are preferred
        like = torch.randn(e, generator=g, device="cuda") * 0.7
        s.update(logits=(torch.randn(t, e, generator=g, device="cuda") + like).to(dt),
                 valid=torch.rand(t, generator=g, device="cuda") < 0.8 if c["valid"] else None)
        if c["backward"]:
            s.update(dweights=rand(t, c["k"], to=torch.float32), dloss=torch.full((1,), 0.01, device="cuda"))
    return s


# ------------------------------------------------------------- plain forms

def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    xm = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(xm.square().mean(-1, keepdim=True) + EPS)
    xh = xm * r
    y = xh * w
    if s["b"] is not None:
        y = y + s["b"].float()
    out = {"y": y.to(dt)}
    if c["backward"]:
        dy = s["dy"].float()
        t = dy * w
        dx = r * (t - t.mean(-1, keepdim=True) - xh * (t * xh).mean(-1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        out.update(dx=dx.to(dt), dw=(dy * xh).sum(0))
        if s["b"] is not None:
            out["db"] = dy.sum(0)
    return out


def _uniform(n, seed, offset, device):
    """n 32-bit numbers: Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011),
    key = seed, counter = (index of four, offset)."""
    low = 0xFFFFFFFF
    at = torch.arange((n + 3) // 4, device=device, dtype=torch.int64)
    c = [at & low, at >> 32, torch.full_like(at, offset & low), torch.full_like(at, offset >> 32)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # 64 bits, whatever their sign
        c = [(b >> 32 & low) ^ c[1] ^ k0, b & low, (a >> 32 & low) ^ c[3] ^ k1, a & low]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack(c, 1).view(-1)[:n]


def _plain_dropout(s):
    c, dt = s["case"], s["x"].dtype
    x = s["x"].float()
    least = round(c["p"] * 2 ** 32)
    keep = (_uniform(x.numel(), s["seed"], s["offset"], x.device) >= least).view(x.shape)
    scale = 2 ** 32 / (2 ** 32 - least)
    y = torch.where(keep, x * scale, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(dt)}
    if c["backward"]:
        out["dx"] = torch.where(keep, s["dy"].float() * scale, 0.0).to(dt)
    return out


def _plain_embedding(s):
    c, table = s["case"], s["table"]
    at = s["tokens"].long() - s["first"]
    here = (at >= 0) & (at < table.shape[0]) & (s["tokens"] >= 0)
    at = torch.where(here, at, 0)
    out = {"y": torch.where(here[:, None], table[at].float() * c["scale"], 0.0).to(table.dtype)}
    if c["backward"]:
        grad = torch.zeros(table.shape, device=table.device)
        grad.index_add_(0, at[here], s["dy"][here].float())
        out["dtable"] = (grad * c["scale"]).to(table.dtype)
    return out


def _plain_router(s):
    c = s["case"]
    e, k = c["experts"], c["k"]
    l = s["logits"].float()
    some = torch.ones(c["t"], dtype=torch.bool, device=l.device) if s["valid"] is None else s["valid"]
    p = torch.exp(l - l.amax(1, keepdim=True))
    p = torch.where(some[:, None], p / p.sum(1, keepdim=True), 0.0)
    at, left, experts, weights = torch.arange(e, device=l.device), l.clone(), [], []
    for _ in range(k):  # the largest, the first of equal ones
        i = torch.where(left == left.amax(1, keepdim=True), at, e).amin(1, keepdim=True)
        experts.append(i), weights.append(p.gather(1, i))
        left.scatter_(1, i, -math.inf)
    experts, weights = torch.cat(experts, 1), torch.cat(weights, 1)
    taken = torch.zeros_like(l).scatter_(1, experts, 1.0) * some[:, None]
    counts, n = taken.sum(0), some.sum().clamp(min=1)
    f = counts / (k * n)
    total = torch.where(some, weights.sum(1), 1.0)[:, None]
    if c["normalize"]:
        weights = weights / total
    out = {"experts": torch.where(some[:, None], experts, -1).int(), "weights": weights,
           "counts": torch.cat((counts.int(), some.sum()[None].int())), "loss": (e * (f * p.sum(0)).sum() / n)[None]}
    if c["backward"]:
        g = s["dweights"]
        if c["normalize"]:
            g = (g - (g * weights).sum(1, keepdim=True)) / total
        dp = (s["dloss"] * e * f / n).expand(c["t"], e).scatter_add(1, experts, g)
        out["dlogits"] = (p * (dp - (p * dp).sum(1, keepdim=True))).to(s["logits"].dtype)
    return out


# ------------------------------------------------- the library's operators

_handle = []


def _library():
    from paper_2609_34244_gb300 import heddle as h
    if not _handle:
        _handle.append(h.heddle_create(torch.cuda.current_device()))
    return h, _handle[0]


def _own_norm(s):
    h, ctx = _library()
    c, x = s["case"], s["x"]
    out = {"y": torch.empty_like(x)}
    mean = rstd = None
    if c["backward"]:
        mean, rstd = (torch.empty(c["rows"], dtype=torch.float32, device=x.device) for _ in range(2))
    h.heddle_layer_norm(ctx, x, s["w"], s["b"], out["y"], mean=mean, rstd=rstd, eps=EPS)
    if c["backward"]:
        out.update(dx=torch.empty_like(x), dw=torch.empty(c["cols"], dtype=torch.float32, device=x.device))
        if c["bias"]:
            out["db"] = torch.empty(c["cols"], dtype=torch.float32, device=x.device)
        h.heddle_layer_norm_backward(ctx, s["dy"], x, s["w"], mean, rstd, dx=out["dx"], dw=out["dw"],
                                     dbias=out.get("db"), dres=s["dres"])
    return out


def _own_dropout(s):
    h, ctx = _library()
    c, x = s["case"], s["x"]
    out = {"y": torch.empty_like(x)}
    h.heddle_dropout(ctx, x, out["y"], c["p"], s["seed"], offset=s["offset"], residual=s["residual"])
    if c["backward"]:
        out["dx"] = torch.empty_like(x)
        h.heddle_dropout_backward(ctx, s["dy"], out["dx"], c["p"], s["seed"], offset=s["offset"])
    return out


def _own_embedding(s):
    h, ctx = _library()
    c, tokens, table = s["case"], s["tokens"], s["table"]
    out = {"y": torch.empty(c["t"], c["cols"], dtype=table.dtype, device=table.device)}
    rest = dict(scale=c["scale"], first=s["first"], vocab=c["vocab"])
    h.heddle_embedding(ctx, tokens, table, out["y"], **rest)
    if c["backward"]:
        out["dtable"] = torch.empty_like(table)
        h.heddle_embedding_backward(ctx, tokens, s["dy"], out["dtable"], **rest)
    return out


def _own_router(s):
    h, ctx = _library()
    c, l = s["case"], s["logits"]
    t, e, k = c["t"], c["experts"], c["k"]
    out = {"experts": torch.empty(t, k, dtype=torch.int32, device=l.device),
           "weights": torch.empty(t, k, dtype=torch.float32, device=l.device),
           "counts": torch.empty(e + 1, dtype=torch.int32, device=l.device),
           "loss": torch.empty(1, dtype=torch.float32, device=l.device)}
    rest = dict(valid=s["valid"], normalize=c["normalize"])
    h.heddle_router(ctx, l, out["experts"], out["weights"], out["counts"], loss=out["loss"], **rest)
    if c["backward"]:
        out["dlogits"] = torch.empty_like(l)
        h.heddle_router_backward(ctx, l, out["experts"], out["weights"], out["counts"], out["dlogits"],
                                 dweights=s["dweights"], dloss=s["dloss"], **rest)
    return out


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# ----------------------------------------------------- work and definitions

def work(case):
    c = case
    e = DTYPES[c["dtype"]].itemsize
    if c["op"] == "norm":
        n = c["rows"] * c["cols"]
        bytes_ = e * (2 * n + (2 if c["bias"] else 1) * c["cols"])
        if c["backward"]:  # gradients in and out, the residual path's in, and the weights' (the inputs count once)
            bytes_ += e * (2 + c["residual"]) * n + 4 * (2 if c["bias"] else 1) * c["cols"]
        return {"bytes": bytes_, "flops": (22 if c["backward"] else 8) * n}
    if c["op"] == "dropout":
        n = c["rows"] * c["cols"]
        return {"bytes": e * n * (2 + c["residual"] + (2 if c["backward"] else 0)),
                "flops": n * (2 + (1 if c["backward"] else 0))}
    if c["op"] == "embedding":
        rows, t = c["vocab"] // c["shards"], c["t"] * (0.75 if c["padded"] else 1)
        # tokens of the shard, and its distinct ones, on average over where the ranks lie
        rank = torch.arange(c["vocab"], dtype=torch.float64)
        p = (torch.log(rank + 2) - torch.log(rank + 1)) / math.log(c["vocab"] + 1)
        distinct = float((1 - (1 - p) ** t).sum()) / c["shards"]
        bytes_ = 4 * c["t"] + e * c["cols"] * (distinct + c["t"])
        if c["backward"]:
            bytes_ += e * c["cols"] * (t / c["shards"] + rows)
        return {"bytes": int(bytes_), "flops": int(c["cols"] * t / c["shards"] * (2 if c["backward"] else 1))}
    n, chosen = c["t"] * c["experts"], c["t"] * c["k"]
    bytes_ = e * n + 8 * chosen + 4 * c["experts"] + (c["t"] if c["valid"] else 0)
    if c["backward"]:
        bytes_ += e * n + 4 * chosen
    return {"bytes": bytes_, "flops": (12 if c["backward"] else 6) * n}


def _philox_by_halves(n, seed, offset):
    """The same numbers as ``_uniform``, products by halves of 16 bits, a word at a time."""
    def product(a, m):  # high and low 32 bits of a m
        ah, al, mh, ml = a >> 16, a & 0xFFFF, m >> 16, m & 0xFFFF
        low, mid, high = al * ml, ah * ml + (al * ml >> 16), ah * mh
        mid2 = (mid & 0xFFFF) + al * mh
        return high + (mid >> 16) + (mid2 >> 16), (mid2 & 0xFFFF) << 16 | low & 0xFFFF

    quad = torch.div(torch.arange(0, n, 4, device="cuda"), 4, rounding_mode="floor")
    x0, x1 = quad.remainder(2 ** 32), torch.div(quad, 2 ** 32, rounding_mode="floor")
    x2, x3 = torch.zeros_like(quad) + offset % 2 ** 32, torch.zeros_like(quad) + offset // 2 ** 32
    for r in range(10):
        key0 = (seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32
        key1 = (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        h0, l0 = product(x0, 0xD2511F53)
        h1, l1 = product(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ key0, l1, h0 ^ x3 ^ key1, l0
    return torch.stack((x0, x1, x2, x3), dim=-1).flatten()[:n]


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    f = {n: t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t for n, t in s.items()}
    if c["op"] == "norm":
        names = ["x", "w"] + (["b"] if c["bias"] else [])
        for n in names:
            f[n] = f[n].detach().requires_grad_(c["backward"])
        var, mean = torch.var_mean(f["x"], dim=1, correction=0, keepdim=True)
        y = (f["x"] - mean) / (var + EPS).sqrt() * f["w"]
        if c["bias"]:
            y = y + f["b"]
        out = {"y": y.detach()}
        if c["backward"]:
            got = torch.autograd.grad(y, [f[n] for n in names], f["dy"])
            out.update({"d" + n: t for n, t in zip(names, got)})
            if c["residual"]:
                out["dx"] = out["dx"] + f["dres"]
        return out
    if c["op"] == "dropout":
        n = f["x"].numel()
        least = round(c["p"] * 2 ** 32)
        kept = _philox_by_halves(n, s["seed"], s["offset"]) >= least
        mask = kept.view_as(f["x"]).double() / (1 - least / 2 ** 32)
        out = {"y": f["x"] * mask + (f["residual"] if c["residual"] else 0)}
        if c["backward"]:
            out["dx"] = f["dy"] * mask
        return out
    if c["op"] == "embedding":
        rows = c["vocab"] // c["shards"]
        # every token's row of the shard, or a last one of zeros
        row = torch.tensor([v - s["first"] if v >= 0 and 0 <= v - s["first"] < rows else rows
                            for v in s["tokens"].tolist()], device="cuda")
        full = torch.cat((f["table"], torch.zeros(1, c["cols"], dtype=torch.float64, device="cuda")))
        out = {"y": full[row] * c["scale"]}
        if c["backward"]:
            del full
            order = torch.argsort(row, stable=True)
            got, size = torch.unique_consecutive(row[order], return_counts=True)
            ends = torch.cumsum(size, 0)
            grad = torch.zeros(rows + 1, c["cols"], dtype=torch.float64, device="cuda")
            for j in range(0, c["cols"], 256):  # sums of neighbours as differences of running sums
                run_ = torch.cumsum(f["dy"][order, j:j + 256], 0)[ends - 1]
                grad[got, j:j + 256] = torch.diff(run_, dim=0, prepend=torch.zeros_like(run_[:1]))
            out["dtable"] = grad[:rows] * c["scale"]
        return out
    t, e, k = c["t"], c["experts"], c["k"]
    some = torch.ones(t, dtype=torch.bool, device="cuda") if s["valid"] is None else s["valid"]
    n = int(some.sum())
    order = torch.sort(f["logits"], dim=1, descending=True, stable=True).indices[:, :k]
    l = f["logits"].detach().requires_grad_(c["backward"])
    p = torch.softmax(l, 1) * some[:, None]
    w = torch.gather(p, 1, order)
    if c["normalize"]:
        w = torch.where(some[:, None], w / w.sum(1, keepdim=True), 0.0)
    counts = torch.bincount(order[some].flatten(), minlength=e)
    loss = e * (counts.double() / (k * max(n, 1)) * p.sum(0) / max(n, 1)).sum()
    out = {"experts": torch.where(some[:, None], order, -1).int(), "weights": w.detach(),
           "counts": torch.cat((counts, torch.tensor([n], device="cuda"))).int(), "loss": loss.detach()[None]}
    if c["backward"]:
        out["dlogits"], = torch.autograd.grad([w, loss], [l], [f["dweights"], f["dloss"][0]])
    return out
