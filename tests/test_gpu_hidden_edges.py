"""Layer norm where 32 bits are short, and what its results may not depend on."""

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
