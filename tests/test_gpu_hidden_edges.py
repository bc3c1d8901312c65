"""Layer norm where 32 bits are short, and what its results may not depend on."""

import pytest

torch = pytest.importorskip("torch")

import hidden_reference as H  # noqa: E402
from op_reference import close  # noqa: E402
from test_gpu_hidden import floats, lib  # noqa: E402, F401
from test_gpu_operators import TYPES, gen, rand  # noqa: E402

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
