"""The transformer layer's operators, as cases to time and to compare: a plain
form of each in elementary 32-bit torch operations, the calls of the library's
own (``own``), and the operators' definitions in 64 bits.

Sizes are those of the workloads the library prices (hidden 4096 with a
feed-forward width of 14336 and sequences of 2048; hidden 8192 with sequences
of 4096; tensor-parallel shards of both), single tokens and ragged ones."""

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # one token through a square projection with bias and residual
        dict(name="linear-token", op="linear", m=1, n=4096, k=4096, act="none", bias=True, residual=True,
             backward=False, dtype="bf16"),
        # a training step of the down projection of 2048 tokens, its residual added in the same pass
        dict(name="linear-down-train", op="linear", m=2048, n=4096, k=14336, act="none", bias=False, residual=True,
             backward=True, dtype="bf16"),
        # a training step at odd sizes: rows of no 16-byte multiple, bias and activation
        dict(name="linear-odd-train", op="linear", m=1023, n=2047, k=4099, act="gelu", bias=True, residual=True,
             backward=True, dtype="fp16"),
        # a handful of tokens through the gated block
        dict(name="ffn-few-tokens", op="ffn", m=16, n=14336, k=4096, act="silu", backward=False, dtype="bf16"),
        # a training step of the gated block, two sequences of 2048
        dict(name="ffn-train", op="ffn", m=4096, n=14336, k=4096, act="silu", backward=True, dtype="bf16"),
        # a tensor-parallel shard (an eighth) of the gated block of a hidden size of 8192
        dict(name="ffn-shard-train", op="ffn", m=4095, n=3584, k=8192, act="gelu", backward=True, dtype="fp16"),
        # one token's queries and keys
        dict(name="qknorm-token", op="qknorm", t=1, hq=32, hk=8, d=128, rot=128, interleaved=False, backward=False,
             dtype="bf16"),
        # a training step's queries and keys: hidden 8192, four sequences of 4096
        dict(name="qknorm-train", op="qknorm", t=16384, hq=64, hk=8, d=128, rot=128, interleaved=False, backward=True,
             dtype="bf16"),
        # a part of the head rotated, pairs interleaved, in 32 bits, odd lengths
        dict(name="qknorm-part-fp32", op="qknorm", t=4001, hq=12, hk=3, d=80, rot=32, interleaved=True, backward=True,
             dtype="fp32"),
        # single tokens against long ragged histories, window and sinks
        dict(name="attention-tokens", op="attention", b=16, tq=1, tk=8192, hq=32, hk=8, d=128, window=4096, sinks=4,
             ragged=True, backward=False, dtype="bf16"),
        # a training step of two full-causal sequences, hidden 4096
        dict(name="attention-causal-train", op="attention", b=2, tq=2048, tk=2048, hq=32, hk=8, d=128, window=0,
             sinks=0, ragged=False, backward=True, dtype="bf16"),
        # a training step of padded sequences with a window and sinks, narrow heads
        dict(name="attention-window-train", op="attention", b=2, tq=4095, tk=4095, hq=16, hk=4, d=64, window=1000,
             sinks=5, ragged=True, backward=True, dtype="fp16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "ffn", "ffn", "qknorm", "attention", "attention"])
    half = rng.choice(["bf16", "bf16", "fp16"])
    backward = rng.random() < 0.6
    if op in ("linear", "ffn"):
        while True:  # up to the products of the largest listed case
            m, n, k = _log(rng, 1, 4096), _log(rng, 64, 14336), _log(rng, 64, 14336)
            if m * n * k <= 2048 * 4096 * 14336:
                break
        if rng.random() < 0.6:
            n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
        if op == "ffn":
            return dict(op=op, m=m, n=n, k=k, act=rng.choice(["silu", "gelu", "relu"]), backward=backward, dtype=half)
        return dict(op=op, m=m, n=n, k=k, act=rng.choice(["none", "none", "silu", "gelu", "relu"]),
                    bias=rng.random() < 0.5, residual=rng.random() < 0.5, backward=backward, dtype=half)
    if op == "qknorm":
        hk = rng.choice([1, 2, 3, 4, 8])
        d = rng.choice([64, 80, 96, 128, 128, 256])
        return dict(op=op, t=_log(rng, 1, 12000), hq=hk * rng.choice([1, 2, 4, 6, 8]), hk=hk, d=d,
                    rot=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.5, backward=backward,
                    dtype=rng.choice(["bf16", "fp16", "fp32"]))
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 3, 4, 8])
    tk = _log(rng, 1, 4096)
    window = rng.choice([0, _log(rng, 1, 4096)])
    if backward:
        tq = tk
        while 2 * tq * tk * hq > 2 * 2048 * 2048 * 32:
            hq //= 2
            hk = math.gcd(hq, hk)
        b = rng.choice([1, 2])
    else:
        tq, b = rng.choice([(1, _log(rng, 1, 32)), (_log(rng, 1, tk), 1)])
    return dict(op=op, b=b, tq=tq, tk=tk, hq=hq, hk=hk, d=rng.choice([64, 128, 128, 96]), window=window,
                sinks=rng.choice([0, 4, 33]) if window else 0, ragged=rng.random() < 0.5, backward=backward, dtype=half)


def _lens(c):
    """Lengths of the sequences: full, or shortened by up to a half, the same for every seed."""
    if not c["ragged"]:
        return None
    cut = [(i * 7919 + 13) % max(1, c["tk"] // 2 + 1) for i in range(c["b"])]
    return [c["tk"] - x for x in cut]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def rand(*shape, std=1.0, to=dt):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(to)

    s = {"case": c}
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        s.update(x=rand(m, k), w=rand(n, k, std=k ** -0.5), bias=rand(n, std=0.5) if c["bias"] else None,
                 residual=rand(m, n) if c["residual"] else None, dy=rand(m, n) if c["backward"] else None)
    elif c["op"] == "ffn":
        m, n, k = c["m"], c["n"], c["k"]
        s.update(x=rand(m, k), wg=rand(n, k, std=k ** -0.5), wu=rand(n, k, std=k ** -0.5),
                 dy=rand(m, n) if c["backward"] else None)
    elif c["op"] == "qknorm":
        t, hq, hk, d, r = c["t"], c["hq"], c["hk"], c["d"], c["rot"]
        # queries, keys and values come out of one projection: rows of all heads
        qkv = rand(t, hq + 2 * hk, d, std=1.5)
        inv = 10000.0 ** (-torch.arange(r // 2, device="cuda", dtype=torch.float64) / (r // 2))
        ang = torch.arange(t + 64, device="cuda", dtype=torch.float64)[:, None] * inv
        s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], wq=1 + rand(d, std=0.1), wk=1 + rand(d, std=0.1),
                 cos=ang.cos().float(), sin=ang.sin().float(),
                 positions=torch.randint(0, t + 64, (t,), generator=g, device="cuda", dtype=torch.int32))
        if c["backward"]:
            s.update(dq=rand(t, hq, d), dk=rand(t, hk, d))
    else:
        b, tq, tk, hq, hk, d = (c[x] for x in ("b", "tq", "tk", "hq", "hk", "d"))
        s.update(q=rand(b, tq, hq, d), k=rand(b, tk, hk, d), v=rand(b, tk, hk, d))
        lens = _lens(c)
        s["kv_lens"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        # padded sequences have as many queries as keys; single tokens come last
        s["q_lens"] = s["kv_lens"] if lens is not None and tq == tk else None
        if c["backward"]:
            s["do"] = rand(b, tq, hq, d)
    return s


# ------------------------------------------------------------- plain forms

def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return torch.clamp(z, min=0) if act == "relu" else z


def _dact(z, act):
    if act == "silu":
        sg = torch.sigmoid(z)
        return sg * (1 + z * (1 - sg))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return (z > 0).to(z.dtype) if act == "relu" else torch.ones_like(z)


def _plain_linear(s):
    c, dt = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.T
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(dt)}
    if c["backward"]:
        dz = s["dy"].float()
        if c["act"] != "none":
            dz = dz * _dact(z, c["act"])
        out.update(dx=(dz @ w).to(dt), dw=(dz.T @ x).to(dt))
        if c["bias"]:
            out["dbias"] = dz.sum(0).to(dt)
    return out


def _plain_ffn(s):
    c, dt = s["case"], s["x"].dtype
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    gate, up = x @ wg.T, x @ wu.T
    a = _act(gate, c["act"])
    out = {"y": (a * up).to(dt)}
    if c["backward"]:
        dy = s["dy"].float()
        dgate, dup = dy * up * _dact(gate, c["act"]), dy * a
        out.update(dx=(dgate @ wg + dup @ wu).to(dt), dwg=(dgate.T @ x).to(dt), dwu=(dup.T @ x).to(dt))
    return out


def _rotate(v, cos, sin, c, sign):
    """Pairs of the head's first ``rot`` values turned by their position's angles."""
    h = c["rot"] // 2
    r, rest = v[..., :c["rot"]], v[..., c["rot"]:]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :h], r[..., h:])
    a, b = a * cos - sign * b * sin, b * cos + sign * a * sin
    r = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1)


def _norm_rope(x, w, cos, sin, c):
    return _rotate(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w, cos, sin, c, 1)


def _norm_rope_backward(dy, x, w, cos, sin, c):
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh = x * r
    dv = _rotate(dy, cos, sin, c, -1)
    t = dv * w
    return r * (t - xh * (t * xh).mean(-1, keepdim=True)), (dv * xh).sum((0, 1))


def _plain_qknorm(s):
    c, dt = s["case"], s["q"].dtype
    p = s["positions"].long()
    cos, sin = s["cos"][p][:, None], s["sin"][p][:, None]
    q, k, wq, wk = (s[x].float() for x in ("q", "k", "wq", "wk"))
    out = {"q": _norm_rope(q, wq, cos, sin, c).to(dt), "k": _norm_rope(k, wk, cos, sin, c).to(dt)}
    if c["backward"]:
        dq, dwq = _norm_rope_backward(s["dq"].float(), q, wq, cos, sin, c)
        dk, dwk = _norm_rope_backward(s["dk"].float(), k, wk, cos, sin, c)
        out.update(dq=dq.to(dt), dk=dk.to(dt), dwq=dwq, dwk=dwk)
    return out


def _visible(c, q_lens, kv_lens, device):
    """[b, tq, tk]: which keys a query sees."""
    kl = torch.full((c["b"],), c["tk"], device=device) if kv_lens is None else kv_lens.long()
    ql = torch.full((c["b"],), c["tq"], device=device) if q_lens is None else q_lens.long()
    i, j = torch.arange(c["tq"], device=device)[None, :, None], torch.arange(c["tk"], device=device)[None, None, :]
    kl, ql = kl[:, None, None], ql[:, None, None]
    pos = kl - ql + i
    ok = (j <= pos) & (j < kl) & (i < ql)
    if c["window"]:
        ok = ok & ((pos - j < c["window"]) | (j < c["sinks"]))
    return ok


def _plain_attention(s):
    c, dt = s["case"], s["q"].dtype
    b, tq, tk, hq, hk, d = (c[x] for x in ("b", "tq", "tk", "hq", "hk", "d"))
    scale, n = d ** -0.5, hq // hk
    q = s["q"].float().view(b, tq, hk, n, d).permute(0, 2, 3, 1, 4).reshape(b, hk, n * tq, d)
    k, v = s["k"].float().transpose(1, 2), s["v"].float().transpose(1, 2)
    bad = ~_visible(c, s["q_lens"], s["kv_lens"], q.device)[:, None, None]
    sc = (q @ k.transpose(2, 3) * scale).view(b, hk, n, tq, tk).masked_fill_(bad, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    lse = torch.where(torch.isinf(top), torch.zeros_like(top), top) + torch.log(total)
    p = (p / torch.where(total > 0, total, torch.ones_like(total))).view(b, hk, n * tq, tk)
    o = p @ v

    def back(t):  # [b, hk, n * tq, d] -> [b, tq, hq, d]
        return t.view(b, hk, n, tq, d).permute(0, 3, 1, 2, 4).reshape(b, tq, hq, d)

    out = {"o": back(o).to(dt), "lse": lse.view(b, hq, tq)}
    if c["backward"]:
        do = s["do"].float().view(b, tq, hk, n, d).permute(0, 2, 3, 1, 4).reshape(b, hk, n * tq, d)
        ds = p * (do @ v.transpose(2, 3) - (do * o).sum(-1, keepdim=True)) * scale
        # a row that sees nothing has p = 0 and gives no gradient
        out.update(dq=back(ds @ k).to(dt), dk=(ds.transpose(2, 3) @ q).transpose(1, 2).to(dt).contiguous(),
                   dv=(p.transpose(2, 3) @ do).transpose(1, 2).to(dt).contiguous())
    return out


# ------------------------------------------------- the library's operators

_handle = []


def _library():
    from paper_2609_34244_gb300 import heddle as h
    if not _handle:
        _handle.append(h.heddle_create(torch.cuda.current_device()))
    return h, _handle[0]


def _own_linear(s):
    h, ctx = _library()
    c, x, w = s["case"], s["x"], s["w"]
    m, n = c["m"], c["n"]
    act = h.ACTIVATIONS[c["act"]]
    y = torch.empty(m, n, dtype=x.dtype, device=x.device)
    pre = torch.empty(m, n, dtype=torch.float32, device=x.device) if c["backward"] and act else None
    h.heddle_linear(ctx, x, w, y, bias=s["bias"], residual=s["residual"], act=act, pre=pre)
    out = {"y": y}
    if c["backward"]:
        out.update(dx=torch.empty_like(x), dw=torch.empty_like(w))
        if c["bias"]:
            out["dbias"] = torch.empty_like(s["bias"])
        h.heddle_linear_backward(ctx, s["dy"], x, w, act=act, pre=pre, dx=out["dx"], dw=out["dw"],
                                 dbias=out.get("dbias"))
    return out


def _own_ffn(s):
    h, ctx = _library()
    c, x, wg, wu = s["case"], s["x"], s["wg"], s["wu"]
    act = h.ACTIVATIONS[c["act"]]
    y = torch.empty(c["m"], c["n"], dtype=x.dtype, device=x.device)
    gate = up = None
    if c["backward"]:
        gate, up = (torch.empty(c["m"], c["n"], dtype=torch.float32, device=x.device) for _ in range(2))
    h.heddle_gated_ffn(ctx, x, wg, wu, y, act=act, gate=gate, up=up)
    out = {"y": y}
    if c["backward"]:
        out.update(dx=torch.empty_like(x), dwg=torch.empty_like(wg), dwu=torch.empty_like(wu))
        h.heddle_gated_ffn_backward(ctx, s["dy"], x, wg, wu, gate, up, act=act, dx=out["dx"], dwg=out["dwg"],
                                    dwu=out["dwu"])
    return out


def _own_qknorm(s):
    h, ctx = _library()
    c, q, k = s["case"], s["q"], s["k"]
    out = {"q": torch.empty(q.shape, dtype=q.dtype, device=q.device),
           "k": torch.empty(k.shape, dtype=k.dtype, device=k.device)}
    rest = dict(positions=s["positions"], cos=s["cos"], sin=s["sin"], eps=EPS, interleaved=c["interleaved"])
    h.heddle_qk_norm_rope(ctx, q, k, s["wq"], s["wk"], out["q"], out["k"], **rest)
    if c["backward"]:
        out.update(dq=torch.empty_like(s["dq"]), dk=torch.empty_like(s["dk"]),
                   dwq=torch.empty(c["d"], dtype=torch.float32, device=q.device),
                   dwk=torch.empty(c["d"], dtype=torch.float32, device=q.device))
        h.heddle_qk_norm_rope_backward(ctx, s["dq"], s["dk"], q, k, s["wq"], s["wk"], out["dq"], out["dk"],
                                       out["dwq"], out["dwk"], **rest)
    return out


def _own_attention(s):
    h, ctx = _library()
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    out = {"o": torch.empty_like(q),
           "lse": torch.empty(c["b"], c["hq"], c["tq"], dtype=torch.float32, device=q.device)}
    rest = dict(q_lens=s["q_lens"], kv_lens=s["kv_lens"], window=c["window"], sinks=c["sinks"])
    h.heddle_attention(ctx, q, k, v, out["o"], out["lse"], **rest)
    if c["backward"]:
        out.update(dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v))
        h.heddle_attention_backward(ctx, s["do"], q, k, v, out["o"], out["lse"], out["dq"], out["dk"], out["dv"],
                                    **rest)
    return out


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# ----------------------------------------------------- work and definitions

def work(case):
    c = case
    e = DTYPES[c["dtype"]].itemsize
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        bytes_ = e * (m * k + n * k + m * n + (n if c["bias"] else 0) + (m * n if c["residual"] else 0))
        if c["backward"]:  # the gradient of the output in; those of x, the weights and the bias out
            bytes_ += e * (m * n + m * k + n * k + (n if c["bias"] else 0))
        return {"bytes": bytes_, "flops": (6 if c["backward"] else 2) * m * n * k}
    if c["op"] == "ffn":
        m, n, k = c["m"], c["n"], c["k"]
        bytes_ = e * (m * k + 2 * n * k + m * n)
        if c["backward"]:
            bytes_ += e * (m * n + m * k + 2 * n * k)
        return {"bytes": bytes_, "flops": (12 if c["backward"] else 4) * m * n * k}
    if c["op"] == "qknorm":
        values = c["t"] * (c["hq"] + c["hk"]) * c["d"]
        table = c["t"] * (4 + 4 * c["rot"])
        # forward: in and out; backward: the gradients in and out (the inputs count once)
        return {"bytes": (4 if c["backward"] else 2) * e * values + table,
                "flops": (20 if c["backward"] else 8) * values}
    lens = _lens(c) or [c["tk"]] * c["b"]
    pairs = keys = rows = 0
    for n in lens:
        first = 0 if c["tq"] == c["tk"] else n - c["tq"]
        last = n
        rows += last - max(0, first)
        w = c["window"] or last
        at = torch.arange(max(0, first), last, dtype=torch.int64)
        near = torch.clamp(at + 1, max=w)
        pairs += int((near + torch.clamp(at + 1 - near, min=0, max=c["sinks"])).sum())
        low = max(0, max(0, first) - w + 1)
        keys += last - low + min(low, c["sinks"])
    d = c["d"]
    bytes_ = e * d * (2 * rows * c["hq"] + 2 * keys * c["hk"]) + 4 * rows * c["hq"]
    if c["backward"]:
        bytes_ += e * d * (2 * rows * c["hq"] + 2 * keys * c["hk"])
    return {"bytes": bytes_, "flops": (14 if c["backward"] else 4) * d * pairs * c["hq"]}


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    f = {n: t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t for n, t in s.items()}

    def grads(outputs, given, wanted):
        got = torch.autograd.grad(outputs, [f[n] for n in wanted], given)
        return dict(zip(wanted, got))

    def want(*names):
        for n in names:
            f[n] = f[n].detach().requires_grad_(c["backward"])

    fn = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu,
          "none": lambda z: z}
    if c["op"] == "linear":
        want("x", "w", *(["bias"] if c["bias"] else []))
        y = fn[c["act"]](torch.nn.functional.linear(f["x"], f["w"], f["bias"]))
        out = {"y": (y if f["residual"] is None else y + f["residual"]).detach()}
        if c["backward"]:
            d = grads(y, f["dy"], ["x", "w"] + (["bias"] if c["bias"] else []))
            out.update({"d" + n: t for n, t in d.items()})
        return out
    if c["op"] == "ffn":
        want("x", "wg", "wu")
        y = fn[c["act"]](f["x"] @ f["wg"].T) * (f["x"] @ f["wu"].T)
        out = {"y": y.detach()}
        if c["backward"]:
            out.update({"d" + n: t for n, t in grads(y, f["dy"], ["x", "wg", "wu"]).items()})
        return out
    if c["op"] == "qknorm":
        want("q", "k", "wq", "wk")
        p = s["positions"].long()
        turn = torch.complex(f["cos"][p], f["sin"][p])[:, None]
        h, r = c["rot"] // 2, c["rot"]

        def one(x, w):
            v = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w
            pairs = v[..., :r].unflatten(-1, (h, 2)) if c["interleaved"] else \
                v[..., :r].unflatten(-1, (2, h)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
            return torch.cat((z, v[..., r:]), -1)

        q, k = one(f["q"], f["wq"]), one(f["k"], f["wk"])
        out = {"q": q.detach(), "k": k.detach()}
        if c["backward"]:
            d = grads([q, k], [f["dq"], f["dk"]], ["q", "k", "wq", "wk"])
            out.update({"d" + n: t for n, t in d.items()})
        return out
    b, tq, tk, hq, hk, d = (c[x] for x in ("b", "tq", "tk", "hq", "hk", "d"))
    out = {"o": torch.zeros(b, tq, hq, d, dtype=torch.float64, device="cuda"),
           "lse": torch.full((b, hq, tq), -math.inf, dtype=torch.float64, device="cuda")}
    if c["backward"]:
        out.update(dq=torch.zeros_like(out["o"]), dk=torch.zeros_like(f["k"]), dv=torch.zeros_like(f["v"]))
    at = torch.arange(tk, device="cuda")
    for i in range(b):
        n = tk if s["kv_lens"] is None else int(s["kv_lens"][i])
        m = tq if s["q_lens"] is None else int(s["q_lens"][i])
        pos = torch.arange(m, device="cuda")[:, None] + (n - m)
        far = at[None, :n] > pos
        if c["window"]:
            far = far | ((pos - at[None, :n] >= c["window"]) & (at[None, :n] >= c["sinks"]))
        some = ~far.all(1)
        for j in range(hq):
            kv = j // (hq // hk)
            q, k, v = f["q"][i, :m, j], f["k"][i, :n, kv], f["v"][i, :n, kv]
            sc = (q @ k.T / math.sqrt(d)).masked_fill(far, -math.inf)
            lse = torch.logsumexp(sc, 1)
            p = torch.where(some[:, None], torch.exp(sc - lse[:, None]), 0.0)
            o = p @ v
            out["o"][i, :m, j], out["lse"][i, j, :m] = o, lse
            if c["backward"]:
                do = f["do"][i, :m, j]
                ds = p * (do @ v.T - (do * o).sum(1, keepdim=True)) / math.sqrt(d)
                out["dq"][i, :m, j] = ds @ k
                out["dk"][i, :n, kv] += ds.T @ q
                out["dv"][i, :n, kv] += p.T @ do
    return out
