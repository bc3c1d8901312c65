"""The compiled marshalling of the layer operators: what it refuses before
the library is called, what it passes on, and that it holds on to nothing."""

import sys

import pytest


@pytest.fixture()
def ops():
    from paper_2609_34244_gb300 import heddle as h
    return h._op_setup(), h


def _calls(h, x):
    q3, q4 = x.view(1, 2, 16), x.view(1, 1, 2, 16)
    return [(h.heddle_linear, (None, x, x, x)), (h.heddle_linear_backward, (None, x, x, x)),
            (h.heddle_gated_ffn, (None, x, x, x, x)), (h.heddle_gated_ffn_backward, (None, x, x, x, x, x, x)),
            (h.heddle_qk_norm_rope, (None, q3, q3, x, x, q3, q3)),
            (h.heddle_qk_norm_rope_backward, (None, q3, q3, q3, q3, x, x, q3, q3, x, x)),
            (h.heddle_attention, (None, q4, q4, q4, q4)),
            (h.heddle_attention_backward, (None, q4, q4, q4, q4, q4, q4, q4, q4, q4))]


@pytest.mark.parametrize("i", range(8))
def test_host_tensors_types_and_objects_are_refused(ops, i):
    import torch
    _, h = ops
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    for bad, message in ((x, "expected a CUDA tensor of"), (x.double(), "unsupported element type")):
        f, args = _calls(h, bad)[i]
        with pytest.raises(h.HeddleError, match=message) as e:
            f(*args)
        assert e.value.status == h.E_ARG
    f, args = _calls(h, x)[i]
    for place in range(1, len(args)):
        other = list(args)
        other[place] = [1.0]
        with pytest.raises(h.HeddleError) as e:
            f(*other)
        assert e.value.status == h.E_ARG


def test_number_of_arguments(ops):
    native, h = ops
    for name in ("linear", "linear_backward", "gated_ffn", "gated_ffn_backward", "qk_norm_rope",
                 "qk_norm_rope_backward", "attention", "attention_backward"):
        with pytest.raises(h.HeddleError, match="arguments"):
            getattr(native, name)(None, None)


def test_refused_calls_keep_no_reference(ops):
    import torch
    _, h = ops
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    for f, args in _calls(h, x):
        before = [sys.getrefcount(a) for a in args]
        for _ in range(50):
            with pytest.raises(h.HeddleError):
                f(*args)
        assert [sys.getrefcount(a) for a in args][1:] == before[1:]


@pytest.mark.gpu
def test_streams_contexts_and_argument_types(ops):
    """A stream as an object, an address or a ctypes value, a context as an
    address; numbers of the wrong kind raise Python's own errors."""
    import ctypes
    import torch
    _, h = ops
    ctx = h.heddle_create(0)
    try:
        x = torch.randn(3, 64, device="cuda").bfloat16()
        w = torch.randn(32, 64, device="cuda").bfloat16()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        want = torch.empty(3, 32, device="cuda", dtype=torch.bfloat16)
        h.heddle_linear(ctx, x, w, want)
        torch.cuda.synchronize()
        before = [sys.getrefcount(a) for a in (x, w, want, side)]
        for st in (None, side, side.cuda_stream, ctypes.c_void_p(side.cuda_stream), 0):
            for c in (ctx, ctx.value):
                y = torch.zeros_like(want)
                torch.cuda.synchronize()
                h.heddle_linear(c, x, w, y, stream=st)
                torch.cuda.synchronize()
                assert torch.equal(y, want)
        assert [sys.getrefcount(a) for a in (x, w, want, side)] == before
        for kw, error in (({"act": "silu"}, TypeError), ({"act": 2 ** 40}, OverflowError),
                          ({"stream": "default"}, AttributeError)):
            with pytest.raises(error):
                h.heddle_linear(ctx, x, w, y, **kw)
        with pytest.raises(h.HeddleError) as e:
            h.heddle_linear(None, x, w, y)
        assert e.value.status == h.E_ARG
    finally:
        h.heddle_destroy(ctx)
