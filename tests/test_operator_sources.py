"""What the layer operators' sources promise about chained launches (no GPU):
a kernel that starts under the end of the one before allows the next one to,
waits before it touches what the call's kernels write, and reads nothing
through the read-only path, which that wait does not order."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34244_gb300", "csrc")
FILES = ["heddle_gemm.cu", "heddle_pointwise.cu", "heddle_qknorm.cu", "heddle_attn.cu", "heddle_attn_tc.cu"]
# launched the ordinary way, after all that the stream holds
ORDINARY = {"attn_row_kernel", "attn_dq_row_kernel", "attn_dkv_row_kernel"}


def kernels():
    for name in FILES:
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for m in re.finditer(r"__global__[^{;]*?\b(\w+_kernel)\(", text):
            yield name, m.group(1), text[m.start():text.index("\n}\n", m.start())]


def test_chained_kernels_allow_and_wait():
    seen = set()
    for name, kernel, body in kernels():
        seen.add(kernel)
        if kernel in ORDINARY:
            continue
        assert "allow_dependents();" in body, "%s: %s" % (name, kernel)
        assert "await_previous();" in body, "%s: %s" % (name, kernel)
    assert ORDINARY < seen and len(seen) >= 15


def test_ordinary_launches_are_the_row_kernels_and_the_products_of_few_rows():
    for name in FILES:
        launched = set(re.findall(r"\b(\w+)(?:<[^<>;]*>)?<<<", open(os.path.join(CSRC, name)).read()))
        assert launched <= ORDINARY, name


def test_no_read_only_path():
    for path in glob.glob(os.path.join(CSRC, "heddle_*")):
        if os.path.basename(path) in FILES + ["heddle_tc.cuh", "heddle_ops.cuh", "heddle_attn.cuh"]:
            text = open(path).read()
            assert "__ldg(" not in text and "__restrict__" not in text and "ld.global.nc" not in text, path
