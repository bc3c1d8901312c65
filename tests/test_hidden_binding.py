"""The compiled marshalling of layer norm, dropout, embedding and router: what
it refuses before the library is called, and that it holds on to nothing; the
C structs' layout; what the kernels' sources promise about chained launches;
the random numbers' published answers (no GPU)."""

import ctypes as C
import os
import re
import subprocess
import sys

import pytest

import hidden_reference as H

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_34244_gb300", "csrc")
FILES = ["heddle_layernorm.cu", "heddle_dropout.cu", "heddle_embedding.cu", "heddle_router.cu"]
NAMES = ("layer_norm", "layer_norm_backward", "dropout", "dropout_backward", "embedding", "embedding_backward",
         "router", "router_backward")


@pytest.fixture()
def ops(heddle_lib):
    return heddle_lib._op_setup(), heddle_lib


def _calls(h, x):
    return [(h.heddle_layer_norm, (None, x, x, x, x)), (h.heddle_layer_norm_backward, (None, x, x, x, x, x)),
            (h.heddle_dropout, (None, x, x, 0.5, 1)), (h.heddle_dropout_backward, (None, x, x, 0.5, 1)),
            (h.heddle_embedding, (None, x, x, x)), (h.heddle_embedding_backward, (None, x, x, x)),
            (h.heddle_router, (None, x, x, x, x)), (h.heddle_router_backward, (None, x, x, x, x, x))]


@pytest.mark.parametrize("i", range(len(NAMES)))
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
        with pytest.raises((h.HeddleError, TypeError)):
            f(*other)


def test_number_of_arguments(ops):
    native, h = ops
    for name in NAMES:
        with pytest.raises(h.HeddleError, match="arguments"):
            getattr(native, name)(None, None)


def test_refused_calls_keep_no_reference(ops):
    import torch
    _, h = ops
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    for f, args in _calls(h, x):
        before = sys.getrefcount(x)  # numbers are shared with whatever else holds them
        for _ in range(50):
            with pytest.raises(h.HeddleError):
                f(*args)
        assert sys.getrefcount(x) == before


def test_struct_layouts_match_header(heddle_lib, tmp_path):
    names = ["layer_norm_args", "layer_norm_grad_args", "dropout_args", "embedding_args", "embedding_grad_args",
             "router_args", "router_grad_args"]
    lines, want = [], []
    for n in names:
        t = getattr(heddle_lib, "heddle_" + n)
        lines.append('printf("%%zu\\n", sizeof(heddle_%s));' % n)
        want.append(C.sizeof(t))
        for field, _ in t._fields_:
            lines.append('printf("%%zu\\n", offsetof(heddle_%s, %s));' % (n, field))
            want.append(getattr(t, field).offset)
    src = tmp_path / "op.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "heddle.h"\nint main(void) {\n%s\nreturn 0; }\n'
                   % "\n".join(lines))
    exe = tmp_path / "op"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(v) for v in subprocess.check_output([str(exe)], text=True).split()] == want


def test_chained_kernels_allow_and_wait_and_read_past_no_cache():
    seen = 0
    for name in FILES:
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        assert "<<<" not in text and "__ldg(" not in text and "__restrict__" not in text and "ld.global.nc" not in text
        for m in re.finditer(r"__global__[^{;]*?\b(\w+_kernel)\(", text):
            body = text[m.start():text.index("\n}\n", m.start())]
            assert "allow_dependents();" in body and "await_previous();" in body, m.group(1)
            seen += 1
    assert seen >= 14


def test_reference_random_numbers_are_the_published_ones():
    """The known answers that the generator's authors publish with it."""
    ones = H.MASK
    for counter, key, want in (
            ([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
            ([ones] * 4, [ones] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
            ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
             [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])):
        assert H.philox(counter, key) == want
    seed, offset = 0x0123456789ABCDEF, 0xFEDCBA9876543210
    got = H.numbers(4 * (2 ** 32 + 5) + 3, 6, seed, offset).tolist()
    key, high = [seed & ones, seed >> 32], [offset & ones, offset >> 32]
    words = [w for i in (5, 6, 7) for w in H.philox([i, 1] + high, key)]
    assert got == words[3:9]
