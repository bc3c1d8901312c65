"""Calls at the edges of the layer operators' contract: empty sizes, values
that are not finite, the ends of the element types' ranges, single rows,
other devices."""

import math

import pytest

torch = pytest.importorskip("torch")

import op_reference as R  # noqa: E402
from test_gpu_operators import CANARY, gen, lib, rand, refused  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("scratch", [False, True])
def test_gradients_of_no_outputs_with_an_activation(heddle_lib, name, scratch):
    """A sum over no outputs is zero, whether or not an earlier call left
    scratch behind."""
    h = heddle_lib
    ctx = h.heddle_create(0)
    try:
        dt = torch.bfloat16
        e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")
        if scratch:
            x, w = rand(gen(1), 5, 9, dt=dt), rand(gen(2), 7, 9, dt=dt)  # odd rows are laid out
            h.heddle_linear(ctx, x, w, e(5, 7))
        dx, pre = e(3, 8).fill_(5), torch.empty(3, 0, device="cuda")
        h.heddle_linear_backward(ctx, e(3, 0), e(3, 8), e(0, 8), act=h.ACTIVATIONS[name], pre=pre, dx=dx, dw=e(0, 8),
                                 dbias=e(0))
        assert (dx == 0).all()
        dx.fill_(5)
        h.heddle_linear_backward(ctx, e(3, 0), e(3, 8), e(0, 8), act=h.ACTIVATIONS[name], pre=pre, dx=dx)
        assert (dx == 0).all()
    finally:
        h.heddle_destroy(ctx)


@pytest.mark.parametrize("name", ["none", "gelu"])
@pytest.mark.parametrize("scratch", [False, True])
def test_gradients_over_no_rows(heddle_lib, name, scratch):
    h = heddle_lib
    ctx = h.heddle_create(0)
    try:
        e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
        if scratch:
            x, w = rand(gen(1), 5, 9, dt=torch.bfloat16), rand(gen(2), 7, 9, dt=torch.bfloat16)
            h.heddle_linear(ctx, x, w, e(5, 7))
        dw, db, pre = e(4, 8).fill_(5), e(4).fill_(5), torch.empty(0, 4, device="cuda")
        h.heddle_linear_backward(ctx, e(0, 4), e(0, 8), e(4, 8), act=h.ACTIVATIONS[name], pre=pre, dx=e(0, 8), dw=dw,
                                 dbias=db)
        assert (dw == 0).all() and (db == 0).all()
        db.fill_(5)
        h.heddle_linear_backward(ctx, e(0, 4), e(0, 8), e(4, 8), act=h.ACTIVATIONS[name], pre=pre, dbias=db)
        assert (db == 0).all()
    finally:
        h.heddle_destroy(ctx)
