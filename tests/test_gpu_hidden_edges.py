"""The hidden state's operators where 32 bits are short, and what their results
may not depend on."""

import pytest

torch = pytest.importorskip("torch")

import hidden_reference as H  # noqa: E402
from op_reference import close  # noqa: E402
from test_gpu_hidden import floats, laid, lib  # noqa: E402, F401
from test_gpu_operators import TYPES, frame_kept, framed, gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [64, 100, 512, 1000, 2047, 4096, 8192, 12288, 20000])
@pytest.mark.parametrize("m", [5, 1300])
def test_layer_norm_gradients_whose_statistics_squares_leave_the_range(lib, m, n, dt):
    """rstd^2 is beyond 2^128 or, times the gradients, below 2^-149; rstd times
    what belongs to it is not."""
    h, ctx = lib
    dt = TYPES[dt]
    for scale, size in ((2e-20, 1e-2), (1e16, 1e-17)):
        g = gen(n)
        x, dy, w = rand(g, m, n, dt=dt) * scale, rand(g, m, n, dt=dt) * size, 1 + rand(g, n, dt=dt, std=0.3)
        dy += x / scale * size  # so that the third term counts
        mean, rstd = x.float().mean(1), torch.full((m,), 1 / scale, device="cuda")
        dx, dw, db = torch.empty_like(x), floats(n), floats(n)
        h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=dx, dw=dw, dbias=db)
        (wx, ex), (ww, ew), (wb, eb) = H.layer_norm_grads(dy, x, w, mean, rstd, None)
        close(dx, wx, ex, "dx")
        close(dw, ww, ew, "dw")
        close(db, wb, eb, "dbias")


# spare columns, elements before the first
PLACES = [(0, 0), (8, 8), (0, 1), (3, 1), (8, 3), (1, 0)]
BITS = [(7, 3), (50, 64), (33, 200), (21, 257), (17, 512), (9, 520), (9, 1000), (6, 2047), (6, 2048), (5, 4096),
        (5, 4104), (3000, 4608), (5, 6144), (5, 8184), (2000, 8192), (5, 8200), (4, 12288), (3, 16384), (2, 17000)]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n", BITS)
def test_layer_norm_results_do_not_depend_on_addresses(lib, m, n, dt):
    """Rows at 16 bytes, at other strides and at odd addresses, in and out: the
    same bits, statistics and gradients among them."""
    h, ctx = lib
    dt = TYPES[dt]
    g = gen(m + n)
    x, dy, dres = (rand(g, m, n, dt=dt) + 0.5 for _ in range(3))
    w, b = 1 + rand(g, n + 1, dt=dt, std=0.3), rand(g, n + 1, dt=dt)
    want = None
    for i, ((pad, skip), (pad_y, skip_y)) in enumerate(zip(PLACES, PLACES[1:] + PLACES[:1])):
        wi, bi = (t[1:].clone() if i % 2 else t[1:] for t in (w, b))
        xi, dyi, dri = laid(x, pad, skip), laid(dy, pad, skip), laid(dres, pad_y, skip_y)
        y, buf = framed(m, n, dt, pad_y, skip_y)
        dx, dbuf = framed(m, n, dt, pad_y, skip_y)
        mean, rstd, dw, db = floats(m), floats(m), floats(n), floats(n)
        h.heddle_layer_norm(ctx, xi, wi, bi, y, mean=mean, rstd=rstd)
        h.heddle_layer_norm_backward(ctx, dyi, xi, wi, mean, rstd, dx=dx, dw=dw, dbias=db, dres=dri)
        frame_kept(y, buf, "y")
        frame_kept(dx, dbuf, "dx")
        got = dict(mean=mean, rstd=rstd, y=y.clone(), dx=dx.clone(), dw=dw, db=db)
        want = want or got
        for name in want:
            assert torch.equal(got[name], want[name]), "%s of layout %d" % (name, i)


def far_from_zero(x, w, b, eps):
    """(mean, bound), (rstd, bound), (y, bound) where the deviations are taken
    from a 32-bit number near the mean, and their own mean is taken out again.

    That number, m, is off by em as in H.layer_norm.  v = x - m is off by e |v|;
    the mean of v by its additions and v's errors, ed; so v minus it, in one
    rounding, by e |v| + ed + e |mean of v| and its own rounding.

    For 16-bit values the mean of v is what the sum of x leaves beyond m.  That
    sum is exact while it stays below 2^24 times the last place of the row's
    smallest value, of which all values and sums are multiples; else it is off
    by its additions, em."""
    e, last = H.e, torch.finfo(x.dtype).eps
    x = x.double()
    n = x.shape[1]
    many = H.depth(n) + 5
    mean = x.mean(1, keepdim=True)
    em = (H.depth(n) + 3) * e * x.abs().mean(1, keepdim=True)
    d = x - mean
    var = d.square().mean(1, keepdim=True)
    size = d.abs().mean(1, keepdim=True) + em        # of v, on average; |mean of v| <= em
    ed = many * e * size
    # mean v^2 = var + (mean v)^2 <= var + em^2, off by its additions and v's errors
    ev = (many + 6) * e * (var + em ** 2) + 2 * em * ed + 4 * e * em ** 2
    rstd = (var + eps) ** -0.5
    rel = (ev + e * eps) / (var + eps) + 6 * e
    assert rel.max() < 0.5
    v = d * rstd
    wd = 1.0 if w is None else w.double()
    bd = 0.0 if b is None else b.double()
    y = v * wd + bd
    if last > 1e-6:
        last = last * 2.0 ** torch.floor(torch.log2(x.abs().amin(1, keepdim=True).clamp(min=1e-30)))
        ed = ed + em * (x.abs().sum(1, keepdim=True) > 2.0 ** 24 * last)
    lost = (e * (d.abs() + em) + ed + 3 * e * em) * rstd * (1 + rel) + v.abs() * (rel + 2 * e)
    ey = lost * (wd if w is None else wd.abs()) + 2 * e * (y.abs() + (v * wd).abs())
    return (mean[:, 0], (ed + 2 * e * em + e * mean.abs())[:, 0]), (rstd[:, 0], (rstd * rel)[:, 0]), (y, ey)


@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("n", [5, 64, 100, 257, 300, 512, 1023, 2047, 4096, 4100, 8192, 12288, 20000])
@pytest.mark.parametrize("center", [0.0, 300.0, -4096.0, 1e5])
def test_layer_norm_of_large_means(lib, n, center, dt):
    """The mean's rounding, up to 2^-24 of it, does not reach y: with a mean of
    100000 and deviations of 1 it was off by 0.004 from that alone."""
    h, ctx = lib
    dt = TYPES[dt]
    if abs(center) > 60000 and dt == torch.float16:
        center = 30000.0
    g = gen(n)
    x = (rand(g, 40, n, dt=torch.float32) * (1 if dt == torch.float32 else max(1.0, abs(center) / 64)) + center).to(dt)
    for pad, skip in PLACES[:4]:
        w, b = (None, None) if skip == 8 else (1 + rand(g, n, dt=dt, std=0.3), rand(g, n, dt=dt))
        y, mean, rstd = torch.empty_like(x), floats(40), floats(40)
        h.heddle_layer_norm(ctx, laid(x, pad, skip), w, b, y, mean=mean, rstd=rstd)
        (wm, em), (wr, er), (wy, ey) = far_from_zero(x, w, b, 1e-5)
        close(mean, wm, em, "mean")
        close(rstd, wr, er, "rstd")
        close(y, wy, ey, "y")


@pytest.mark.parametrize("n", [64, 100, 1000, 2047, 8192, 20000])
def test_layer_norm_of_squares_beyond_32_bits(lib, n):
    """Their sum past the largest float: y is the bias; below the smallest: eps
    alone is the variance, and eps 0 is not asked for."""
    h, ctx = lib
    sign = 1.0 - 2.0 * (torch.arange(n, device="cuda") % 2)
    x = torch.stack((sign * 1e25, sign * 1e-30))
    b, y, mean, rstd = torch.full((n,), 0.25, device="cuda"), torch.empty_like(x), floats(2), floats(2)
    h.heddle_layer_norm(ctx, x, None, b, y, mean=mean, rstd=rstd, eps=0.25)
    assert (y[0] == 0.25).all() and rstd[0] == 0
    assert torch.equal(y[1], x[1] * 2 + 0.25) and rstd[1] == 2
    assert mean[0].abs() <= 1.01e25 / n and mean[1].abs() <= 1.01e-30 / n


FAR = 2 ** 30 + 24  # elements between rows: the third begins past 2^31


def far(t, skip):
    v = torch.empty(skip + 2 * FAR + t.shape[1] + 16, dtype=t.dtype, device="cuda")[skip:]
    v = v.as_strided(t.shape, (FAR, 1))
    v.copy_(t)
    return v


@pytest.mark.parametrize("n", [64, 2047, 4096, 8192, 20000])
@pytest.mark.parametrize("skip", [0, 3])
def test_layer_norm_and_dropout_of_rows_far_apart(lib, n, skip):
    """The same bits as of rows that follow each other."""
    h, ctx = lib
    g = gen(n)
    x, dy, dres = (rand(g, 3, n, dt=torch.bfloat16) for _ in range(3))
    w, b = 1 + rand(g, n, dt=torch.bfloat16, std=0.3), rand(g, n, dt=torch.bfloat16)
    got = []
    for place in (lambda t: t, lambda t: far(t, skip)):
        xi, dyi, dri = (place(t) for t in (x, dy, dres))
        y, dx, d = (place(torch.zeros_like(x)) for _ in range(3))
        mean, rstd, dw, db = floats(3), floats(3), floats(n), floats(n)
        h.heddle_layer_norm(ctx, xi, w, b, y, mean=mean, rstd=rstd)
        h.heddle_layer_norm_backward(ctx, dyi, xi, w, mean, rstd, dx=dx, dw=dw, dbias=db, dres=dri)
        h.heddle_dropout(ctx, xi, d, 0.3, 5, residual=dri)
        got.append([t.clone() for t in (y, mean, rstd, dx, dw, db, d)])
    for one, other in zip(*got):
        assert torch.equal(one, other)


@pytest.mark.parametrize("skip", [0, 3])
def test_embedding_and_router_of_rows_far_apart(lib, skip):
    h, ctx = lib
    g = gen(skip)
    n, e, k = 1000, 250, 4
    table, dy = rand(g, 3, n, dt=torch.float16), rand(g, 3, n, dt=torch.float16)
    logits, dweights = rand(g, 3, e, dt=torch.float16), rand(g, 3, k, dt=torch.float32)
    tokens = torch.tensor([2, 0, 2], device="cuda")
    got = []
    for place in (lambda t: t, lambda t: far(t, skip)):
        y, dtable, dlogits = place(torch.zeros_like(dy)), place(torch.ones_like(table)), place(torch.zeros_like(logits))
        experts, weights = torch.empty(3, k, dtype=torch.int32, device="cuda"), torch.empty(3, k, device="cuda")
        counts, loss = torch.empty(e + 1, dtype=torch.int32, device="cuda"), floats(1)
        h.heddle_embedding(ctx, tokens, place(table), y, scale=3.0)
        h.heddle_embedding_backward(ctx, tokens, place(dy), dtable, scale=3.0)
        h.heddle_router(ctx, place(logits), experts, weights, counts, loss=loss)
        h.heddle_router_backward(ctx, place(logits), experts, weights, counts, dlogits, dweights=dweights, dloss=loss)
        got.append([t.clone() for t in (y, dtable, experts, weights, counts, loss, dlogits)])
    for one, other in zip(*got):
        assert torch.equal(one, other)
