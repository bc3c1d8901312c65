"""The layer operators against their definitions in 64 bits (tests/op_reference.py
derives the bounds), at the sizes, masks, strides and alignments where such
kernels go wrong; their refusals; gradients against differences."""

import math

import pytest

torch = pytest.importorskip("torch")

import op_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def lib(heddle_lib):
    h = heddle_lib
    ctx = h.heddle_create(0)
    yield h, ctx
    torch.cuda.synchronize()
    flags = h.heddle_device_errors(ctx)
    h.heddle_destroy(ctx)
    assert flags == 0


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, *shape, dt, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dt)


CANARY = 77.0


def framed(rows, cols, dt, pad=0, skip=0):
    """A [rows][cols] view with `pad` spare columns and `skip` elements before
    it, and the buffer around it, filled with a canary."""
    buf = torch.full((skip + max(rows, 1) * (cols + pad) + 64,), CANARY, dtype=dt, device="cuda")
    return buf[skip:].as_strided((rows, cols), (cols + pad, 1)), buf


def frame_kept(view, buf, what):
    c = buf.clone()
    skip = view.storage_offset()
    c[skip:].as_strided(view.shape, view.stride()).fill_(CANARY)
    assert (c == CANARY).all(), "%s: written outside its elements" % what


# ------------------------------------------------------------------ products

PRODUCTS = [
    # m, n, k
    (1, 1, 1), (1, 17, 1), (5, 3, 7), (64, 64, 64), (1, 256, 512), (3, 130, 1000), (128, 256, 64), (129, 257, 65),
    (255, 511, 200), (300, 40, 1031), (33, 1200, 4096), (513, 72, 9), (2, 100, 20000),
    (640, 1300, 520), (1025, 2304, 264), (64, 2600, 128), (17, 4500, 320),
]


def product_inputs(m, n, k, dt, seed, pad=0, skip=0):
    g = gen(seed)

    def laid(t):
        if not pad and not skip:
            return t
        v, _ = framed(*t.shape, t.dtype, pad, skip)
        v.copy_(t)
        return v

    return g, laid(rand(g, m, k, dt=dt)), laid(rand(g, n, k, dt=dt, std=max(k, 1) ** -0.5))


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_linear(lib, m, n, k, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for i, (name, bias, res, pad, skip) in enumerate((("none", False, False, 0, 0), ("gelu", True, True, 8, 8),
                                                      ("silu", True, False, 3, 1), ("relu", False, True, 0, 0))):
        g, x, w = product_inputs(m, n, k, dt, 100 * i + m + n + k, pad, skip)
        b = rand(g, n, dt=dt) if bias else None
        r = rand(g, m, n, dt=dt) if res else None
        y, ybuf = framed(m, n, dt, pad, skip)
        pre, pbuf = framed(m, n, torch.float32, pad, skip)
        h.heddle_linear(ctx, x, w, y, bias=b, residual=r, act=h.ACTIVATIONS[name], pre=pre)
        z, ez, want, ey = R.linear(x, w, b, r, name)
        R.close(y, want, ey, "y %s" % name)
        R.close(pre, z, ez, "pre %s" % name)
        frame_kept(y, ybuf, "y")
        frame_kept(pre, pbuf, "pre")
        if res:  # the residual may be the output itself
            y2 = r.clone()
            h.heddle_linear(ctx, x, w, y2, bias=b, residual=y2, act=h.ACTIVATIONS[name])
            assert torch.equal(y2, y)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_linear_backward(lib, m, n, k, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for i, (name, pad, skip) in enumerate((("none", 0, 0), ("gelu", 8, 8), ("silu", 3, 1), ("relu", 0, 0))):
        g, x, w = product_inputs(m, n, k, dt, 100 * i + m + n + k, pad, skip)
        dy = rand(g, m, n, dt=dt)
        z, ez = R.product(x.double(), w.double())
        pre = z.float()
        if name == "relu":
            pre = torch.where(pre.abs() < 1e-3, torch.full_like(pre, 0.25), pre)
        zd = pre.double()  # what the call is given
        dx, xbuf = framed(m, k, dt, pad, skip)
        dw, wbuf = framed(n, k, dt, pad, skip)
        db = torch.empty(n, dtype=dt, device="cuda")
        h.heddle_linear_backward(ctx, dy, x, w, act=h.ACTIVATIONS[name], pre=None if name == "none" else pre,
                                 dx=dx, dw=dw, dbias=db)
        if name == "none":
            zd = z
        wx, ww, wb = R.linear_grads(dy, x, w, zd, torch.zeros_like(zd), name)
        R.close(dx, *wx, "dx %s" % name)
        R.close(dw, *ww, "dw %s" % name)
        R.close(db, *wb, "dbias %s" % name)
        frame_kept(dx, xbuf, "dx")
        frame_kept(dw, wbuf, "dw")
        only = torch.empty_like(db)  # each output alone
        h.heddle_linear_backward(ctx, dy, x, w, act=h.ACTIVATIONS[name], pre=None if name == "none" else pre,
                                 dbias=only)
        assert torch.equal(only, db)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_gated_ffn(lib, m, n, k, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for i, (name, pad, skip) in enumerate((("silu", 0, 0), ("gelu", 8, 8), ("relu", 3, 1), ("none", 0, 0))):
        g, x, wg = product_inputs(m, n, k, dt, 100 * i + m + n + k, pad, skip)
        wu = rand(g, n, k, dt=dt, std=max(k, 1) ** -0.5)
        y, ybuf = framed(m, n, dt, pad, skip)
        gate, gbuf = framed(m, n, torch.float32, pad, skip)
        up, ubuf = framed(m, n, torch.float32, pad, skip)
        act = h.ACTIVATIONS[name]
        h.heddle_gated_ffn(ctx, x, wg, wu, y, act=act, gate=gate, up=up)
        zg, eg, zu, eu, want, ey = R.gated(x, wg, wu, name)
        R.close(y, want, ey, "y %s" % name)
        R.close(gate, zg, eg, "gate")
        R.close(up, zu, eu, "up")
        for v, buf in ((y, ybuf), (gate, gbuf), (up, ubuf)):
            frame_kept(v, buf, "gated")
        y2 = torch.empty(m, n, dtype=dt, device="cuda")
        h.heddle_gated_ffn(ctx, x, wg, wu, y2, act=act)
        assert torch.equal(y2, y)

        dy = rand(g, m, n, dt=dt)
        if name == "relu":
            gate.copy_(torch.where(gate.abs() < 1e-3, torch.full_like(gate, 0.25), gate))
        dx, xbuf = framed(m, k, dt, pad, skip)
        dwg, gbuf = framed(n, k, dt, pad, skip)
        dwu, ubuf = framed(n, k, dt, pad, skip)
        h.heddle_gated_ffn_backward(ctx, dy, x, wg, wu, gate, up, act=act, dx=dx, dwg=dwg, dwu=dwu)
        zero = torch.zeros_like(zg)
        a, b, c = R.gated_grads(dy, x, wg, wu, gate.double(), zero, up.double(), zero, name)
        R.close(dx, *a, "dx %s" % name)
        R.close(dwg, *b, "dw_gate %s" % name)
        R.close(dwu, *c, "dw_up %s" % name)
        for v, buf in ((dx, xbuf), (dwg, gbuf), (dwu, ubuf)):
            frame_kept(v, buf, "gated grads")


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", [(3, 64, 4104), (4, 1000, 264), (5, 70, 520), (8, 900, 2048), (8, 31, 8),
                                   (6, 4000, 64), (9, 64, 1000)])
def test_few_rows(lib, m, n, k, dt):
    test_linear(lib, m, n, k, dt)
    test_gated_ffn(lib, m, n, k, dt)


def test_products_without_rows_or_steps(lib):
    h, ctx = lib
    dt = torch.bfloat16
    e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")
    h.heddle_linear(ctx, e(0, 8), e(4, 8), e(0, 4))
    h.heddle_linear(ctx, e(3, 8), e(0, 8), e(3, 0))
    y = e(3, 4)
    b = rand(gen(1), 4, dt=dt)
    h.heddle_linear(ctx, e(3, 0), e(4, 0), y, bias=b)  # an empty sum
    assert torch.equal(y, b.expand(3, 4))
    h.heddle_gated_ffn(ctx, e(3, 0), e(4, 0), e(4, 0), y)
    assert (y == 0).all()
    dw, db = e(4, 8).fill_(5), e(4).fill_(5)
    h.heddle_linear_backward(ctx, e(0, 4), e(0, 8), e(4, 8), dx=e(0, 8), dw=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()  # sums over no rows
    dx = e(3, 8).fill_(5)
    h.heddle_linear_backward(ctx, e(3, 0), e(3, 8), e(0, 8), dx=dx, dw=e(0, 8), dbias=e(0))
    assert (dx == 0).all()
    f = torch.empty(0, 4, device="cuda")
    dg, du = e(4, 8).fill_(5), e(4, 8).fill_(5)
    h.heddle_gated_ffn_backward(ctx, e(0, 4), e(0, 8), e(4, 8), e(4, 8), f, f, dx=e(0, 8), dwg=dg, dwu=du)
    assert (dg == 0).all() and (du == 0).all()


def test_infinities_and_nan_stay_in_their_rows(lib):
    h, ctx = lib
    for dt in (torch.bfloat16, torch.float16):
        g, x, w = product_inputs(200, 300, 130, dt, 5)
        x[7, 3], x[150, 0] = math.inf, math.nan
        y = torch.empty(200, 300, dtype=dt, device="cuda")
        h.heddle_linear(ctx, x, w, y)
        rows = torch.isfinite(y).all(1)
        bad = torch.zeros(200, dtype=torch.bool, device="cuda")
        bad[7] = bad[150] = True
        assert torch.equal(rows, ~bad)


def test_products_repeat_and_take_their_stream(lib):
    h, ctx = lib
    g, x, w = product_inputs(700, 1100, 2050, torch.bfloat16, 9)
    y = [torch.empty(700, 1100, dtype=x.dtype, device="cuda") for _ in range(2)]
    h.heddle_linear(ctx, x, w, y[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x2 = x * 1
        h.heddle_linear(ctx, x2, w, y[1])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y[0], y[1])


def test_products_against_differences(lib):
    """A step along a random direction of every input changes the loss by
    the gradients' product with it."""
    h, ctx = lib
    m, n, k, dt = 37, 29, 41, torch.float16
    g = gen(3)
    x, wg, wu = rand(g, m, k, dt=dt), rand(g, n, k, dt=dt, std=0.2), rand(g, n, k, dt=dt, std=0.2)
    dy = rand(g, m, n, dt=dt)
    y = torch.empty(m, n, dtype=dt, device="cuda")
    gate, up = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    h.heddle_gated_ffn(ctx, x, wg, wu, y, gate=gate, up=up)
    grads = [torch.empty_like(t) for t in (x, wg, wu)]
    h.heddle_gated_ffn_backward(ctx, dy, x, wg, wu, gate, up, dx=grads[0], dwg=grads[1], dwu=grads[2])
    zg, eg, zu, eu, _, _ = R.gated(x, wg, wu, "silu")
    bounds = [b + R.U[dt] * v.abs() for v, b in R.gated_grads(dy, x, wg, wu, zg, eg, zu, eu, "silu")]
    steps = [torch.randn(t.shape, generator=g, device="cuda").double() for t in (x, wg, wu)]

    def loss(e):
        a, b, c = (t.double() + e * s for t, s in zip((x, wg, wu), steps))
        return (R.act(a @ b.T, "silu") * (a @ c.T) * dy.double()).sum().item()

    e = 1e-3
    d1, d2 = ((loss(s) - loss(-s)) / (2 * s) for s in (e, 2 * e))
    slope, third = (4 * d1 - d2) / 3, abs(d2 - d1)  # the error of the better one is below what they differ by
    got = sum((gr.double() * s).sum().item() for gr, s in zip(grads, steps))
    assert abs(got - slope) <= third + sum((b * s.abs()).sum().item() for b, s in zip(bounds, steps))


# ------------------------------------------------------------ norm and rotation

NORMS = [
    # tokens, q heads, k heads, head_dim, rot_dim, interleaved
    (1, 1, 1, 128, 128, False), (3, 8, 2, 128, 128, True), (257, 12, 3, 64, 64, False), (33, 6, 1, 80, 32, True),
    (33, 5, 5, 96, 48, False), (7, 2, 0, 256, 256, False), (7, 0, 3, 256, 64, True), (19, 3, 1, 1, 0, False),
    (19, 3, 2, 7, 6, True), (19, 3, 2, 130, 10, False), (1000, 16, 2, 128, 64, False),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,hq,hk,d,rot,inter", NORMS)
def test_qk_norm_rope(lib, t, hq, hk, d, rot, inter, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for fused in (True, False):  # rows of all heads as one projection gives them, and a layout of its own
        g = gen(t + hq + d + rot)
        if fused:
            qkv = rand(g, t, hq + 2 * hk, d, dt=dt, std=2.0)
            q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
        else:
            q = rand(g, hq, t, d + 3, dt=dt).transpose(0, 1)[..., 1:d + 1]
            k = rand(g, t, hk, d, dt=dt)
        wq, wk = rand(g, d, dt=dt), rand(g, d, dt=dt)
        rest = dict(eps=1e-5, interleaved=inter)
        p = torch.randint(0, 50, (t,), generator=g, device="cuda", dtype=torch.int32)
        cos = sin = None
        if rot:
            ang = torch.rand(50, rot // 2, generator=g, device="cuda") * 7
            cos, sin = ang.cos(), ang.sin()
            rest.update(positions=p, cos=cos, sin=sin)
        qo, ko = torch.full_like(q, CANARY), torch.full_like(k, CANARY)
        h.heddle_qk_norm_rope(ctx, q, k, wq, wk, qo, ko, **rest)
        c, s = (None, None) if not rot else (cos.double()[p.long()][:, None], sin.double()[p.long()][:, None])
        for got, x, w in ((qo, q, wq), (ko, k, wk)):
            if x.numel():
                R.close(got, *R.norm_rope(x, w, c, s, rot, inter, 1e-5), "norm rope")
        gq, gk = rand(g, t, hq, d, dt=dt), rand(g, t, hk, d, dt=dt)
        dq, dk = torch.full_like(q, CANARY), torch.full_like(k, CANARY)
        dwq, dwk = torch.full((2, d), CANARY, device="cuda")
        h.heddle_qk_norm_rope_backward(ctx, gq, gk, q, k, wq, wk, dq, dk, dwq, dwk, **rest)
        for got, gotw, gy, x, w in ((dq, dwq, gq, q, wq), (dk, dwk, gk, k, wk)):
            if x.numel():
                a, b = R.norm_rope_grads(gy, x, w, c, s, rot, inter, 1e-5)
                R.close(got, *a, "dx")
                R.close(gotw, *b, "dw")
            else:
                assert (gotw == 0).all()
        q2, k2 = q.clone(), k.clone()  # in place, forward and backward
        h.heddle_qk_norm_rope(ctx, q2, k2, wq, wk, q2, k2, **rest)
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
        h.heddle_qk_norm_rope_backward(ctx, gq, gk, q, k, wq, wk, gq, gk, dwq, dwk, **rest)
        assert torch.equal(gq, dq) and torch.equal(gk, dk)


def test_qk_norm_rope_rows_of_zeros_and_positions_outside(lib):
    h, ctx = lib
    g = gen(4)
    q, k = rand(g, 5, 4, 64, dt=torch.bfloat16), rand(g, 5, 2, 64, dt=torch.bfloat16)
    q[2, 1] = 0
    w = rand(g, 64, dt=torch.bfloat16)
    ang = torch.rand(8, 32, generator=g, device="cuda")
    p = torch.tensor([0, 8, 7, -1, 3], dtype=torch.int32, device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rest = dict(positions=p, cos=ang.cos(), sin=ang.sin())
    h.heddle_qk_norm_rope(ctx, q, k, w, w, qo, ko, **rest)
    assert h.heddle_device_errors(ctx) == 32
    assert h.heddle_device_errors(ctx) == 0
    assert (qo[2, 1] == 0).all() and torch.isfinite(qo).all()
    for t in (1, 3):
        assert (qo[t] == 0).all() and (ko[t] == 0).all()
    assert (qo[0] != 0).any()
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    dwq, dwk = torch.empty(2, 64, device="cuda")
    h.heddle_qk_norm_rope_backward(ctx, q, k, q, k, w, w, dq, dk, dwq, dwk, **rest)
    assert h.heddle_device_errors(ctx) == 32
    assert torch.isfinite(dq).all() and (dq[1] == 0).all() and (dk[3] == 0).all()
    some = torch.tensor([0, 2, 4], device="cuda")
    c, s = ang.cos().double()[p[some].long()][:, None], ang.sin().double()[p[some].long()][:, None]
    for gotw, x in ((dwq, q), (dwk, k)):
        _, b = R.norm_rope_grads(x[some], x[some], w, c, s, 64, False, 1e-6)
        R.close(gotw, *b, "dw")


def test_qk_norm_rope_without_tokens(lib):
    h, ctx = lib
    e = torch.empty(0, 4, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    dwq, dwk = torch.full((2, 64), 3.0, device="cuda")
    h.heddle_qk_norm_rope(ctx, e, e, w, w, e, e)
    h.heddle_qk_norm_rope_backward(ctx, e, e, e, e, w, w, e, e, dwq, dwk)
    assert (dwq == 0).all() and (dwk == 0).all()


def test_qk_norm_rope_against_differences(lib):
    h, ctx = lib
    g = gen(8)
    t, hq, hk, d, rot = 11, 3, 1, 24, 16
    q, k = rand(g, t, hq, d, dt=torch.float32), rand(g, t, hk, d, dt=torch.float32)
    wq, wk = rand(g, d, dt=torch.float32), rand(g, d, dt=torch.float32)
    gq, gk = rand(g, t, hq, d, dt=torch.float32), rand(g, t, hk, d, dt=torch.float32)
    p = torch.arange(t, device="cuda", dtype=torch.int32)
    ang = torch.rand(t, rot // 2, generator=g, device="cuda") * 5
    rest = dict(positions=p, cos=ang.cos(), sin=ang.sin(), interleaved=True)
    grads = [torch.empty_like(x) for x in (q, k, wq, wk)]
    h.heddle_qk_norm_rope_backward(ctx, gq, gk, q, k, wq, wk, *grads, **rest)
    steps = [torch.randn(x.shape, generator=g, device="cuda").double() for x in (q, k, wq, wk)]
    c, s = ang.cos().double()[:, None], ang.sin().double()[:, None]

    def loss(e):
        a, b, wa, wb = (x.double() + e * st for x, st in zip((q, k, wq, wk), steps))
        return sum((R.norm_rope(x, w, c, s, rot, True, 1e-6)[0] * gy.double()).sum().item()
                   for x, w, gy in ((a, wa, gq), (b, wb, gk)))

    e = 1e-3
    d1, d2 = ((loss(z) - loss(-z)) / (2 * z) for z in (e, 2 * e))
    slope, third = (4 * d1 - d2) / 3, abs(d2 - d1)
    got = sum((gr.double() * st).sum().item() for gr, st in zip(grads, steps))
    bound = 0.0
    for x, w, gy, i in ((q, wq, gq, 0), (k, wk, gk, 1)):
        a, b = R.norm_rope_grads(gy, x, w, c, s, rot, True, 1e-6)
        for (v, eb), st in ((a, steps[i]), (b, steps[i + 2])):
            bound += ((eb + R.EPS32 * v.abs()) * st.abs()).sum().item()
    assert abs(got - slope) <= third + bound


# ------------------------------------------------------------------- attention

ATTENTION = [
    # batch, q_len, kv_len, q heads, kv heads, head_dim, window, sinks, lens
    (1, 1, 1, 1, 1, 64, 0, 0, None), (2, 1, 700, 8, 2, 128, 0, 0, None), (2, 1, 1500, 4, 4, 128, 100, 4, "kv"),
    (1, 128, 128, 2, 1, 128, 0, 0, None), (1, 129, 129, 3, 1, 64, 0, 0, None), (1, 300, 300, 6, 2, 128, 50, 3, None),
    (2, 257, 257, 5, 1, 64, 1, 0, None), (2, 257, 257, 2, 2, 96, 64, 130, "both"), (3, 200, 200, 4, 1, 128, 0, 0, "both"),
    (2, 100, 40, 2, 1, 64, 0, 0, None), (1, 40, 600, 7, 1, 80, 200, 0, None), (2, 5, 0, 2, 1, 64, 0, 0, None),
    (2, 60, 300, 2, 1, 128, 33, 2, "short"), (1, 90, 90, 2, 1, 160, 20, 1, None), (2, 64, 64, 4, 2, 33, 0, 0, "both"),
    (1, 500, 500, 16, 1, 64, 77, 5, None), (1, 260, 1100, 1, 1, 128, 300, 150, None),
    (2, 1100, 1100, 8, 2, 64, 257, 130, "both"), (1, 1500, 1500, 4, 4, 128, 0, 0, None),
    (1, 3, 3000, 9, 3, 128, 0, 0, None), (2, 130, 130, 4, 1, 64, 3, 2, None), (1, 70, 70, 128, 1, 64, 0, 0, None),
]


def lens_of(kind, b, tq, tk):
    if kind is None:
        return None, None
    i32 = dict(dtype=torch.int32, device="cuda")
    cut = [(i * 61 + 17) % (tk // 2 + 1) for i in range(b)]
    kv = torch.tensor([tk - c for c in cut], **i32)
    if kind == "kv":
        return None, kv
    if kind == "both":
        return kv.clone(), kv
    return torch.tensor([0, tq], **i32)[:b], torch.tensor([tk, 7], **i32)[:b]  # no queries; fewer keys than queries


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("b,tq,tk,hq,hk,d,window,sinks,kind", ATTENTION)
def test_attention(lib, b, tq, tk, hq, hk, d, window, sinks, kind, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for fused in (False, True):
        g = gen(tq + tk + hq + d)
        if fused and tq == tk:  # views of one projection's rows
            qkv = rand(g, b, tq, hq + 2 * hk, d, dt=dt)
            q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:]
        elif fused:  # heads before tokens, an odd start
            q = rand(g, b, hq, tq, d + 1, dt=dt).transpose(1, 2)[..., 1:]
            k, v = (rand(g, b, hk, tk, d, dt=dt).transpose(1, 2) for _ in range(2))
        else:
            q, k, v = rand(g, b, tq, hq, d, dt=dt), rand(g, b, tk, hk, d, dt=dt), rand(g, b, tk, hk, d, dt=dt)
        ql, kl = lens_of(kind, b, tq, tk)
        if kl is not None:  # what padding holds does not count
            for i in range(b):
                k[i, int(kl[i]):] = math.nan
                v[i, int(kl[i]):] = math.inf
        if ql is not None:
            for i in range(b):
                q[i, int(ql[i]):] = math.nan
        do = rand(g, b, tq, hq, d, dt=dt)
        o, dq = torch.full_like(do, CANARY), torch.full_like(do, CANARY)
        dk, dv = (torch.full((b, tk, hk, d), CANARY, dtype=dt, device="cuda") for _ in range(2))
        lse = torch.full((b, hq, tq), CANARY, device="cuda")
        rest = dict(q_lens=ql, kv_lens=kl, window=window, sinks=sinks, scale=0.11)
        h.heddle_attention(ctx, q, k, v, o, lse, **rest)
        o2 = torch.empty_like(o)
        h.heddle_attention(ctx, q, k, v, o2, None, **rest)
        assert torch.equal(o, o2)
        if ql is not None:
            for i in range(b):
                do[i, int(ql[i]):] = math.nan
        h.heddle_attention_backward(ctx, do, q, k, v, o, lse, dq, dk, dv, **rest)
        for i in range(b):
            n_q = tq if ql is None else int(ql[i])
            n_k = tk if kl is None else int(kl[i])
            sums = {n: [torch.zeros(tk, hk, d, dtype=torch.float64, device="cuda") for _ in range(2)]
                    for n in ("dk", "dv")}
            for j in range(hq):
                kv = j // (hq // hk)
                w = R.attention(q[i, :, j], k[i, :, kv], v[i, :, kv], n_q, n_k, window, sinks, 0.11,
                                do[i, :, j])
                R.close(o[i, :, j], *w["o"], "o")
                R.close(lse[i, j], *w["lse"], "lse")
                R.close(dq[i, :, j], *w["dq"], "dq")
                for n in sums:
                    sums[n][0][:, kv] += w[n][0]
                    sums[n][1][:, kv] += w[n][1] + (hq // hk) * 2.0 ** -23 * w[n][0].abs()
            R.close(dk[i], *sums["dk"], "dk")
            R.close(dv[i], *sums["dv"], "dv")


def test_attention_scores_of_large_spread(lib):
    """Scores far apart and far from zero: the running maximum has to hold."""
    h, ctx = lib
    g = gen(21)
    for dt in (torch.bfloat16, torch.float16):
        q, k, v = (rand(g, 1, 400, 1, 64, dt=dt, std=s) for s in (8.0, 8.0, 1.0))
        k[:, 200:] *= 4  # the maximum rises late
        o, lse = torch.empty_like(q), torch.empty(1, 1, 400, device="cuda")
        h.heddle_attention(ctx, q, k, v, o, lse)
        w = R.attention(q[0, :, 0], k[0, :, 0], v[0, :, 0], 400, 400, 0, 0, 0.125)
        R.close(o[0, :, 0], *w["o"], "o")
        R.close(lse[0, 0], *w["lse"], "lse")


def test_attention_against_differences(lib):
    h, ctx = lib
    g = gen(31)
    t, hq, d, dt = 45, 2, 32, torch.float16
    q, k, v = rand(g, 1, t, hq, d, dt=dt), rand(g, 1, t, 1, d, dt=dt), rand(g, 1, t, 1, d, dt=dt)
    do = rand(g, 1, t, hq, d, dt=dt)
    o, lse = torch.empty_like(q), torch.empty(1, hq, t, device="cuda")
    rest = dict(window=20, sinks=2, scale=0.3)
    h.heddle_attention(ctx, q, k, v, o, lse, **rest)
    grads = [torch.empty_like(x) for x in (q, k, v)]
    h.heddle_attention_backward(ctx, do, q, k, v, o, lse, *grads, **rest)
    steps = [torch.randn(x.shape, generator=g, device="cuda").double() for x in (q, k, v)]
    bound = 0.0
    for j in range(hq):
        w = R.attention(q[0, :, j], k[0, :, 0], v[0, :, 0], t, t, 20, 2, 0.3, do[0, :, j])
        for n, st in (("dq", steps[0][0, :, j]), ("dk", steps[1][0, :, 0]), ("dv", steps[2][0, :, 0])):
            bound += ((w[n][1] + R.U[dt] * (w[n][0].abs() + w[n][1])) * st.abs()).sum().item()

    def loss(e):
        a, b, c = (x.double() + e * s for x, s in zip((q, k, v), steps))
        return sum((R.attention(a[0, :, j], b[0, :, 0], c[0, :, 0], t, t, 20, 2, 0.3)["o"][0]
                    * do[0, :, j].double()).sum().item() for j in range(hq))

    e = 1e-4
    d1, d2 = ((loss(s) - loss(-s)) / (2 * s) for s in (e, 2 * e))
    slope, third = (4 * d1 - d2) / 3, abs(d2 - d1)
    got = sum((gr.double() * s).sum().item() for gr, s in zip(grads, steps))
    # the roundoff of two losses of this size in 64 bits, over the step
    assert abs(got - slope) <= third + bound + 1e-13 * abs(loss(0.0)) / e + 1e-9


def test_attention_repeats(lib):
    h, ctx = lib
    g = gen(41)
    q, k, v, do = (rand(g, 2, 333, n, 128, dt=torch.bfloat16) for n in (8, 2, 2, 8))
    got = []
    for _ in range(2):
        o, lse = torch.empty_like(q), torch.empty(2, 8, 333, device="cuda")
        h.heddle_attention(ctx, q, k, v, o, lse, window=100)
        d = [torch.empty_like(x) for x in (q, k, v)]
        h.heddle_attention_backward(ctx, do, q, k, v, o, lse, *d, window=100)
        got.append((o, lse, *d))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("t,hq,hk,d,groups", [
    (6000, 120, 12, 16, (0, 5, 6, 11)),  # the scores' gradients of six key heads at a time fit between the passes
    (5800, 128, 1, 8, (0,)),             # those of a single key head do not
])
def test_attention_backward_beyond_its_room(lib, t, hq, hk, d, groups):
    h, ctx = lib
    g = gen(t)
    q, k, v, do = (rand(g, 1, t, n, d, dt=torch.bfloat16) for n in (hq, hk, hk, hq))
    o, lse = torch.empty_like(q), torch.empty(1, hq, t, device="cuda")
    h.heddle_attention(ctx, q, k, v, o, lse)
    dq, dk, dv = (torch.full_like(x, CANARY) for x in (q, k, v))
    h.heddle_attention_backward(ctx, do, q, k, v, o, lse, dq, dk, dv)
    n = hq // hk
    for kv in groups:
        sums = {x: [torch.zeros(t, d, dtype=torch.float64, device="cuda") for _ in range(2)] for x in ("dk", "dv")}
        for j in range(kv * n, kv * n + n):
            w = R.attention(q[0, :, j], k[0, :, kv], v[0, :, kv], t, t, 0, 0, d ** -0.5, do[0, :, j])
            R.close(o[0, :, j], *w["o"], "o")
            R.close(dq[0, :, j], *w["dq"], "dq")
            for x in sums:
                sums[x][0] += w[x][0]
                sums[x][1] += w[x][1] + n * 2.0 ** -23 * w[x][0].abs()
        R.close(dk[0, :, kv], *sums["dk"], "dk")
        R.close(dv[0, :, kv], *sums["dv"], "dv")


def test_offsets_past_32_bits(lib):
    """Rows and tokens that lie more than 2^31 elements apart."""
    h, ctx = lib
    g = gen(51)
    far = 1 << 30  # elements: the third row and the third head start past 2^31
    room = torch.empty(2 * far + (1 << 20), dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((3, 72), (far, 1))
    x.copy_(rand(g, 3, 72, dt=x.dtype))
    w = rand(g, 40, 72, dt=x.dtype, std=0.1)
    y = room[4096:].as_strided((3, 40), (far, 1))
    h.heddle_linear(ctx, x, w, y)
    _, _, want, ey = R.linear(x, w, None, None, "none")
    R.close(y, want, ey, "y")
    step = (2 * far) // 199 // 8 * 8
    k, v = (room[8192 + 512 * i:].as_strided((1, 200, 1, 64), (0, step, 64, 1)) for i in range(2))
    for t in (k, v):
        t.copy_(rand(g, 1, 200, 1, 64, dt=x.dtype))
    q, do = rand(g, 1, 200, 2, 64, dt=x.dtype), rand(g, 1, 200, 2, 64, dt=x.dtype)
    o, lse = torch.empty_like(q), torch.empty(1, 2, 200, device="cuda")
    h.heddle_attention(ctx, q, k, v, o, lse)
    dq = torch.empty_like(q)
    dk, dv = (room[16384 + 512 * i:].as_strided((1, 200, 1, 64), (0, step, 64, 1)) for i in range(2))
    h.heddle_attention_backward(ctx, do, q, k, v, o, lse, dq, dk, dv)
    both = [R.attention(q[0, :, j], k[0, :, 0], v[0, :, 0], 200, 200, 0, 0, 0.125, do[0, :, j]) for j in range(2)]
    for j in range(2):
        R.close(o[0, :, j], *both[j]["o"], "o")
        R.close(dq[0, :, j], *both[j]["dq"], "dq")
    for got, n in ((dk, "dk"), (dv, "dv")):
        value = both[0][n][0] + both[1][n][0]
        bound = both[0][n][1] + both[1][n][1] + 2.0 ** -22 * (both[0][n][0].abs() + both[1][n][0].abs())
        R.close(got[0, :, 0], value, bound, n)


def test_captured_calls_repeat(lib):
    """A graph of calls whose scratch exists takes new inputs in place."""
    h, ctx = lib
    g = gen(61)
    x, w = rand(g, 100, 136, dt=torch.bfloat16), rand(g, 72, 136, dt=torch.bfloat16, std=0.1)
    q, k = rand(g, 1, 100, 2, 64, dt=torch.bfloat16), rand(g, 1, 100, 1, 64, dt=torch.bfloat16)
    y, o = torch.empty(100, 72, dtype=x.dtype, device="cuda"), torch.empty_like(q)
    lse = torch.empty(1, 2, 100, device="cuda")
    grads = [torch.empty_like(t) for t in (q, k, k)]

    def calls():
        h.heddle_linear(ctx, x, w, y, act=h.ACT_SILU)
        h.heddle_attention(ctx, q, k, k, o, lse, window=30)
        h.heddle_attention_backward(ctx, q, q, k, k, o, lse, *grads, window=30)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    x.mul_(0.5)
    q.mul_(2)
    graph.replay()
    got = [t.clone() for t in (y, o, *grads)]
    calls()
    assert all(torch.equal(a, b) for a, b in zip(got, (y, o, *grads)))


# -------------------------------------------------------------------- refusals

def refused(h, status, fn, *args, **kw):
    with pytest.raises(h.HeddleError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_refusals(lib):
    h, ctx = lib
    e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda")
    x, w, y = e(4, 8), e(6, 8), e(4, 6)
    refused(h, h.E_ARG, h.heddle_linear, ctx, x, e(6, 7), y)
    refused(h, h.E_ARG, h.heddle_linear, ctx, x, w, e(4, 7))
    refused(h, h.E_ARG, h.heddle_linear, ctx, x, w.half(), y)
    refused(h, h.E_ARG, h.heddle_linear, ctx, x.float(), w.float(), y.float())
    refused(h, h.E_ARG, h.heddle_linear, ctx, x.double(), w.double(), y.double())
    refused(h, h.E_ARG, h.heddle_linear, ctx, x.cpu(), w, y)
    refused(h, h.E_ARG, h.heddle_linear, ctx, x, w, y, act=9)
    refused(h, h.E_ARG, h.heddle_linear, ctx, x, w, y, bias=e(5))
    refused(h, h.E_ARG, h.heddle_linear, ctx, x, w, e(6, 4).T)
    refused(h, h.E_ARG, h.heddle_linear, ctx, x[:1].expand(4, 8), w, y)
    refused(h, h.E_ARG, h.heddle_linear, ctx, x, w, y, pre=y)
    refused(h, h.E_ARG, h.heddle_linear_backward, ctx, y, x, w, act=h.ACT_GELU, dx=e(4, 8))
    f = torch.empty(4, 6, device="cuda")
    refused(h, h.E_ARG, h.heddle_gated_ffn, ctx, x, w, w, y, gate=f)
    refused(h, h.E_ARG, h.heddle_gated_ffn_backward, ctx, y, x, w, w, f, f, dwg=e(6, 8))
    q, k, wt = e(3, 4, 64), e(3, 2, 64), e(64)
    p = torch.zeros(3, dtype=torch.int32, device="cuda")
    t = torch.zeros(5, 32, device="cuda")
    refused(h, h.E_ARG, h.heddle_qk_norm_rope, ctx, q, k, wt, e(63), q, k)
    refused(h, h.E_ARG, h.heddle_qk_norm_rope, ctx, q, k, wt, wt, q, k, eps=-1.0)
    refused(h, h.E_ARG, h.heddle_qk_norm_rope, ctx, q, k, wt, wt, q, k, positions=p, cos=t, sin=t[:4])
    refused(h, h.E_ARG, h.heddle_qk_norm_rope, ctx, q, k, wt, wt, q, k, positions=p.long(), cos=t, sin=t)
    wide = torch.zeros(5, 33, device="cuda")
    refused(h, h.E_ARG, h.heddle_qk_norm_rope, ctx, q, k, wt, wt, q, k, positions=p, cos=wide, sin=wide)
    refused(h, h.E_LIMIT, h.heddle_qk_norm_rope, ctx, e(3, 4, 257), e(3, 2, 257), e(257), e(257), e(3, 4, 257),
            e(3, 2, 257))
    q, k, o = e(2, 3, 4, 64), e(2, 5, 2, 64), e(2, 3, 4, 64)
    refused(h, h.E_ARG, h.heddle_attention, ctx, q, e(2, 5, 3, 64), e(2, 5, 3, 64), o)
    refused(h, h.E_ARG, h.heddle_attention, ctx, q, k, e(2, 4, 2, 64), o)
    refused(h, h.E_ARG, h.heddle_attention, ctx, q, k, k, o, window=-1)
    refused(h, h.E_LIMIT, h.heddle_attention, ctx, q, k, k, o, window=2 ** 31)
    refused(h, h.E_ARG, h.heddle_attention, ctx, q, k, k, o, scale=math.inf)
    refused(h, h.E_ARG, h.heddle_attention, ctx, q, k, k, e(1, 3, 4, 64).expand(2, 3, 4, 64))
    refused(h, h.E_ARG, h.heddle_attention, ctx, q, k, k, o, kv_lens=p)
    refused(h, h.E_ARG, h.heddle_attention, ctx, q.float(), k.float(), k.float(), o.float())
    big = e(1, 1, 1, 257)
    refused(h, h.E_LIMIT, h.heddle_attention, ctx, big, big, big, big)
    huge = e(1, 1, 1, 1).expand(1, 2 ** 30, 4, 1)
    refused(h, h.E_LIMIT, h.heddle_attention, ctx, e(1, 1, 4, 1), huge, huge, e(1, 1, 4, 1))
    assert h.heddle_last_error(ctx)
    L = h.load_library()
    for name in h.EXPORTS[-8:]:  # null arguments
        assert getattr(L, name)(ctx, None, None) == h.E_ARG
        assert getattr(L, name)(None, None, None) == h.E_ARG
    a = h.heddle_linear_args(4, 6, 8, 0, 0)
    assert L.heddle_linear(ctx, h.C.byref(a), None) == h.E_ARG
    a.m = -1
    assert L.heddle_linear(ctx, h.C.byref(a), None) == h.E_ARG
    a.m = 2 ** 31
    assert L.heddle_linear(ctx, h.C.byref(a), None) == h.E_LIMIT
