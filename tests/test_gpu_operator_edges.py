"""Calls at the edges of the layer operators' contract: empty sizes, values
that are not finite, the ends of the element types' ranges, single rows, other
devices, graphs and streams that share a context, contractions of seconds."""

import math

import pytest

torch = pytest.importorskip("torch")

import op_reference as R  # noqa: E402
from test_gpu_operators import CANARY, gen, lib, rand, refused  # noqa: E402, F401
from test_gpu_operators import test_attention as attention_test  # noqa: E402

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


# Attention calls by the kernel that they run on this GPU: keys in parts, a
# tile taken twice (alone and in parts), neither, one warp a row.
FORMS = [
    # batch, q_len, kv_len, q heads, kv heads, head_dim, window, sinks
    (1, 1, 3000, 2, 1, 64, 0, 0), (2, 3, 2000, 4, 2, 128, 0, 0), (16, 1, 1100, 16, 8, 128, 0, 0),
    (20, 60, 700, 8, 4, 64, 250, 0), (9, 1, 1300, 16, 8, 64, 0, 0), (2, 300, 300, 4, 2, 64, 100, 3),
    (10, 128, 1024, 8, 8, 64, 128, 0),  # the last query sees keys of its tile's second half alone
    (1, 5, 40, 2, 1, 160, 0, 0), (1, 9, 9, 1, 1, 33, 0, 0),
]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("b,tq,tk,hq,hk,d,window,sinks", FORMS)
def test_queries_that_are_not_finite(lib, b, tq, tk, hq, hk, d, window, sinks, dt):
    """A NaN query gives NaN whichever kernels take it, and so does a score of
    +infinity; scores of -infinity weigh nothing.  Zeros and a logarithm of
    -infinity stay those of a query with no weights at all, and other queries
    keep their values."""
    h, ctx = lib
    g = gen(b + tq + tk + d)
    q, k, v = rand(g, b, tq, hq, d, dt=dt), rand(g, b, tk, hk, d, dt=dt), rand(g, b, tk, hk, d, dt=dt)
    k[..., 0] = k[..., 0].abs() + 0.5  # the sign of an infinite score is that of the query's first value
    rest = dict(window=window, sinks=sinks, scale=0.1)

    def run(q):
        o, lse = torch.full_like(q, CANARY), torch.full((b, hq, tq), CANARY, device="cuda")
        h.heddle_attention(ctx, q, k, v, o, lse, **rest)
        return o, lse

    want, want_lse = run(q)
    at = [(b - 1, tq - 1, hq - 1), (0, 0, 0)]
    for value in (math.nan, math.inf, -math.inf):
        p, other = q.clone(), torch.ones(b, tq, hq, dtype=torch.bool, device="cuda")
        for i, t, j in at:
            p[i, t, j] = math.nan if math.isnan(value) else 0.0
            p[i, t, j, 0] = value
            other[i, t, j] = False
        o, lse = run(p)
        for i, t, j in at:
            if value == -math.inf:
                assert (o[i, t, j] == 0).all() and lse[i, j, t] == -math.inf
            else:
                assert torch.isnan(o[i, t, j]).all() and (torch.isnan(lse[i, j, t]) or lse[i, j, t] == math.inf)
        assert torch.equal(o[other], want[other])
        assert torch.equal(lse.transpose(1, 2)[other], want_lse.transpose(1, 2)[other])


@pytest.mark.parametrize("b,t,hq,hk,d", [
    (1, 24, 2, 1, 64), (1, 200, 4, 2, 128),  # the scores' gradients are kept between the passes
    (80, 440, 128, 1, 64),                   # those of all heads do not fit, and are computed twice
])
def test_scores_gradients_near_the_end_of_float16(lib, b, t, hq, hk, d):
    """Gradients whose P (dP - delta) passes 65504 while the scores' gradients,
    which are `scale` of it, do not: as a loss scale brings about."""
    h, ctx = lib
    g, dt = gen(t), torch.float16
    q, k = rand(g, b, t, hq, d, dt=dt, std=0.1), rand(g, b, t, hk, d, dt=dt, std=0.1)
    v = rand(g, b, t, hk, d, dt=dt, std=4.0)
    do = (torch.randn(b, t, hq, d, generator=g, device="cuda") * (8000 if t < 100 else 4000)).clamp(-30000, 30000)
    do[:, 16:] *= 0.01  # the first queries' weights are large enough, and a key's sum stays in range
    do[:, :, 2:] *= 0.01
    do = do.to(dt)
    lens = [torch.full((b,), t, dtype=torch.int32, device="cuda") for _ in range(2)]
    o, lse = torch.empty_like(q), torch.empty(b, hq, t, device="cuda")
    rest = dict(q_lens=lens[0], kv_lens=lens[1])
    h.heddle_attention(ctx, q, k, v, o, lse, **rest)
    dq, dk, dv = (torch.full_like(x, CANARY) for x in (q, k, v))
    h.heddle_attention_backward(ctx, do, q, k, v, o, lse, dq, dk, dv, **rest)
    scale, n, beyond = d ** -0.5, hq // hk, 0.0
    for i in sorted({0, b - 1}):
        for kv in range(hk):
            sums = {x: [torch.zeros(t, d, dtype=torch.float64, device="cuda") for _ in range(2)] for x in ("dk", "dv")}
            for j in range(kv * n, kv * n + n):
                w = R.attention(q[i, :, j], k[i, :, kv], v[i, :, kv], t, t, 0, 0, scale, do[i, :, j])
                R.close(dq[i, :, j], *w["dq"], "dq")
                for x in sums:
                    sums[x][0] += w[x][0]
                    sums[x][1] += w[x][1] + n * 2.0 ** -23 * w[x][0].abs()
                s = (q[i, :, j].double() @ k[i, :, kv].double().T * scale).masked_fill(
                    ~R.visible(t, t, t, t, 0, 0, "cuda"), -math.inf)
                p, dp = s.softmax(1), do[i, :, j].double() @ v[i, :, kv].double().T
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                beyond = max(beyond, ds.abs().max().item())
                assert ds.abs().max().item() * scale < 60000
            assert all(x[0].abs().max().item() < 60000 for x in sums.values())
            R.close(dk[i, :, kv], *sums["dk"], "dk")
            R.close(dv[i, :, kv], *sums["dv"], "dv")
    assert beyond > 65504


def test_single_rows_at_any_stride(lib):
    """The stride of a single row means nothing, so two of them need not share it."""
    h, ctx = lib
    g, dt = gen(3), torch.bfloat16
    x, wg, wu = rand(g, 1, 40, dt=dt), rand(g, 24, 40, dt=dt), rand(g, 24, 40, dt=dt)
    y, want = (torch.empty(1, 24, dtype=dt, device="cuda") for _ in range(2))
    gates = [torch.empty(1, 24, device="cuda") for _ in range(2)]
    h.heddle_gated_ffn(ctx, x, wg, wu, want, gate=gates[0], up=gates[1])
    wide = torch.full((2, 100), CANARY, device="cuda")
    up = wide[:1, 8:32]
    gate = torch.empty(1, 24, device="cuda")
    h.heddle_gated_ffn(ctx, x, wg, wu, y, gate=gate, up=up)
    assert torch.equal(y, want) and torch.equal(gate, gates[0]) and torch.equal(up, gates[1])
    assert (wide[1] == CANARY).all() and (wide[0, :8] == CANARY).all() and (wide[0, 32:] == CANARY).all()
    dy = rand(g, 1, 24, dt=dt)
    first = [torch.empty_like(t) for t in (x, wg, wu)]
    h.heddle_gated_ffn_backward(ctx, dy, x, wg, wu, gates[0], gates[1], dx=first[0], dwg=first[1], dwu=first[2])
    again = [torch.empty_like(t) for t in (x, wg, wu)]
    h.heddle_gated_ffn_backward(ctx, dy, x, wg, wu, gate, up, dx=again[0], dwg=again[1], dwu=again[2])
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    # one output: its two weights' gradients
    dwg, dwu = torch.empty(1, 40, dtype=dt, device="cuda"), torch.empty(3, 72, dtype=dt, device="cuda")[1:2, :40]
    h.heddle_gated_ffn_backward(ctx, dy[:, :1], x, wg[:1], wu[:1], gate[:, :1], up[:, :1], dwg=dwg, dwu=dwu)
    assert torch.equal(dwg, first[1][:1]) and torch.equal(dwu, first[2][:1])
    refused(h, h.E_ARG, h.heddle_gated_ffn, ctx, x, wg, wu, y, gate=gate)
    two = torch.empty(2, 24, device="cuda")
    refused(h, h.E_ARG, h.heddle_gated_ffn, ctx, x.expand(2, 40).clone(), wg, wu, y.expand(2, 24).clone(), gate=two,
            up=wide[:, 8:32])


def test_tensors_of_another_device_are_refused(lib):
    """The context's device as a stand-in reports it is not the tensors': no
    operator's function may be entered."""
    import ctypes
    h, ctx = lib
    native = h._op_setup()
    entered = []

    @ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p)
    def operator(c, a, s):
        entered.append(c)
        return 0

    @ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p)
    def device(c):
        return where

    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    names = dict.fromkeys(h._OP_NAMES, address(operator))
    names["heddle_device"] = address(device)
    dt = dict(dtype=torch.bfloat16, device="cuda")
    x, p = torch.zeros(4, 8, **dt), torch.zeros(4, 4, device="cuda")
    q3, q4 = x.view(1, 2, 16), x.view(1, 1, 2, 16)
    f8, lse, w16 = torch.zeros(16, device="cuda"), torch.zeros(1, 2, 1, device="cuda"), torch.zeros(16, **dt)
    calls = [(h.heddle_linear, (x, x, x[:, :4])), (h.heddle_linear_backward, (x[:, :4], x, x)),
             (h.heddle_gated_ffn, (x, x, x, x[:, :4])), (h.heddle_gated_ffn_backward, (x[:, :4], x, x, x, p, p)),
             (h.heddle_qk_norm_rope, (q3, q3, w16, w16, q3, q3)),
             (h.heddle_qk_norm_rope_backward, (q3, q3, q3, q3, w16, w16, q3, q3, f8, f8)),
             (h.heddle_attention, (q4, q4, q4, q4)),
             (h.heddle_attention_backward, (q4, q4, q4, q4, q4, lse, q4, q4, q4))]
    assert len(calls) == len(h._OP_NAMES)
    try:
        native.bind(names, h.HeddleError, lambda index: 0)
        for where in (0, 1):
            for f, args in calls:
                entered.clear()
                if where == torch.cuda.current_device():
                    f(ctx, *args)
                    assert len(entered) == 1
                else:
                    refused(h, h.E_ARG, f, ctx, *args)
                    assert not entered
    finally:
        h._op_setup()


def _step(h, ctx, g, t):
    """A linear at odd rows and an attention, with their gradients: tensors, and
    the calls on them."""
    dt = torch.bfloat16
    x, w = rand(g, t, 137, dt=dt), rand(g, 71, 137, dt=dt, std=0.1)
    dy, pre = rand(g, t, 71, dt=dt), torch.empty(t, 71, device="cuda")
    q, k = rand(g, 1, t, 4, 64, dt=dt), rand(g, 1, t, 2, 64, dt=dt)
    y, dx, dw, o, dq, dk, dv = (torch.empty_like(v) for v in (dy, x, w, q, q, k, k))
    db, lse = torch.empty(71, dtype=dt, device="cuda"), torch.empty(1, 4, t, device="cuda")

    def calls():
        h.heddle_linear(ctx, x, w, y, act=h.ACT_SILU, pre=pre)
        h.heddle_linear_backward(ctx, dy, x, w, act=h.ACT_SILU, pre=pre, dx=dx, dw=dw, dbias=db)
        h.heddle_attention(ctx, q, k, k, o, lse)
        h.heddle_attention_backward(ctx, q, q, k, k, o, lse, dq, dk, dv)

    return (x, dy, q), (y, dx, dw, db, o, lse, dq, dk, dv), calls


@pytest.mark.parametrize("warm", [True, False])
def test_graphs_outlive_larger_calls(heddle_lib, warm):
    """A captured call's scratch stays, whatever later calls need, and a
    capture may be the first to need it."""
    h = heddle_lib
    ctx = h.heddle_create(0)
    try:
        inputs, outputs, calls = _step(h, ctx, gen(71), 150)
        if warm:
            calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        _, _, larger = _step(h, ctx, gen(72), 3000)
        larger()
        larger()
        # what was given back is taken again
        others = [torch.full((1 << 22,), CANARY, device="cuda") for _ in range(64)]
        for v in inputs:
            v.mul_(0.5)
        for v in outputs:
            v.fill_(CANARY)
        graph.replay()
        got = [v.clone() for v in outputs]
        assert all((v == CANARY).all() for v in others)
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, outputs))
        del graph
        torch.cuda.synchronize()
        assert h.heddle_device_errors(ctx) == 0
    finally:
        h.heddle_destroy(ctx)


@pytest.mark.parametrize("b,t,hq,hk,d,window,sinks,kind", [
    (1, 1100, 4, 2, 64, 50, 400, None), (2, 2100, 4, 4, 128, 30, 900, "both"), (1, 1500, 8, 1, 96, 1, 1400, None),
])
def test_first_tokens_of_several_tiles(lib, b, t, hq, hk, d, window, sinks, kind):
    """Many tokens that stay visible, whose gradients come in parts."""
    for dt in ("bf16", "fp16"):
        attention_test(lib, b, t, t, hq, hk, d, window, sinks, kind, dt)


def test_calls_on_several_streams_take_turns_at_scratch(heddle_lib):
    """Calls of one context on streams that nothing orders give what they give
    one after another."""
    h = heddle_lib
    ctx = h.heddle_create(0)
    try:
        sizes = (1500, 130, 700, 40, 1100, 257)
        steps = [_step(h, ctx, gen(80 + i), t) for i, t in enumerate(sizes)]
        want = []
        for _, outputs, calls in steps:
            calls()
            torch.cuda.synchronize()
            want.append([v.clone() for v in outputs])
        streams = [torch.cuda.Stream() for _ in range(3)]
        for turn in range(8):
            for _, outputs, _ in steps:
                for v in outputs:
                    v.fill_(CANARY)
            torch.cuda.synchronize()
            for i, (_, _, calls) in enumerate(steps):
                with torch.cuda.stream(streams[(i + turn) % 3]):
                    calls()
            torch.cuda.synchronize()
            for (_, outputs, _), values in zip(steps, want):
                assert all(torch.equal(a, b) for a, b in zip(outputs, values))
        assert h.heddle_device_errors(ctx) == 0
    finally:
        h.heddle_destroy(ctx)


def test_counters_left_by_calls_that_overlapped(heddle_lib, tmp_path):
    """What replays that overlap against the rule may leave in the context's
    work counters does not reach later calls."""
    import ctypes
    import os
    import subprocess
    from paper_2609_34244_gb300 import _build
    h = heddle_lib
    src, so = tmp_path / "counters.cu", tmp_path / "counters.so"
    src.write_text('#include "heddle_ops.cuh"\n'
                   'extern "C" int leave(heddle_ctx* c, int a, int b) {\n'
                   '    const int32_t v[2] = {a, b};\n'
                   '    return cudaMemcpy(heddle_op_context(c)->sched, v, sizeof v, cudaMemcpyHostToDevice);\n'
                   '}\n')
    pkg = os.path.dirname(h.LIB_PATH)
    subprocess.check_call([_build.nvcc(), *_build.ARCH, "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-I",
                           _build.INCLUDE, "-I", _build.CSRC, str(src), "-o", str(so), "-L", pkg, "-lheddle", "-Xlinker",
                           "-rpath", "-Xlinker", pkg])
    leave = ctypes.CDLL(str(so)).leave
    leave.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    ctx = h.heddle_create(0)
    try:
        for heads, t in ((8, 1000), (4, 33)):
            g, dt = gen(t), torch.bfloat16
            q, k, v, do = (rand(g, 4, t, n, 64, dt=dt) for n in (heads, 2, 2, heads))
            o, lse = torch.empty_like(q), torch.empty(4, heads, t, device="cuda")
            h.heddle_attention(ctx, q, k, v, o, lse)

            def grads():
                d = [torch.full_like(x, CANARY) for x in (q, k, v)]
                h.heddle_attention_backward(ctx, do, q, k, v, o, lse, *d)
                torch.cuda.synchronize()
                return d

            want = grads()
            for left in ((3, 0), (1 << 20, 5), (0, 1 << 20)):
                assert leave(ctx, *left) == 0
                for _ in range(2):
                    assert all(torch.equal(a, b) for a, b in zip(grads(), want))
    finally:
        h.heddle_destroy(ctx)


@pytest.mark.parametrize("m,n,k", [(1, 1, 2 ** 31 - 1), (9, 4, 1_000_000_000)])
def test_contractions_that_take_seconds(lib, m, n, k):
    """The longest contractions: a tile's one takes longer than any other wait
    lasts.  Products of +-1, whose sums are whole numbers in any order."""
    h, ctx = lib
    g, dt = gen(k % 1000), torch.bfloat16

    def signs(rows):
        t = torch.empty(rows, k, dtype=dt, device="cuda")
        for r in range(rows):
            for at in range(0, k, 1 << 28):
                part = t[r, at:at + (1 << 28)]
                bits = torch.randint(0, 2, part.shape, generator=g, device="cuda", dtype=torch.int8)
                part.copy_(bits.mul_(2).sub_(1))
        return t

    x, w = signs(m), signs(n)
    y, pre = torch.empty(m, n, dtype=dt, device="cuda"), torch.empty(m, n, device="cuda")
    h.heddle_linear(ctx, x, w, y, pre=pre)
    want = torch.zeros(m, n, dtype=torch.float64, device="cuda")
    for at in range(0, k, 1 << 24):
        want += x[:, at:at + (1 << 24)].float() @ w[:, at:at + (1 << 24)].float().T  # below 2^24: exact
    assert want.abs().max().item() < 2 ** 24
    assert torch.equal(pre.double(), want) and torch.equal(y, want.to(dt))
    assert h.heddle_device_errors(ctx) == 0


@pytest.mark.parametrize("b,t,hq,hk,d,kind", [(1, 2000, 2, 1, 64, None), (2, 600, 4, 2, 128, "both"),
                                              (80, 440, 128, 1, 64, "both")])
@pytest.mark.parametrize("power", [12, 16])
def test_small_gradients_in_float16(lib, b, t, hq, hk, d, kind, power):
    """Gradients are linear in the outputs': small ones have the bounds of
    2^power times larger ones, at that scale, and their results' own rounding."""
    h, ctx = lib
    g, dt = gen(t + power), torch.float16
    q, k, v = rand(g, b, t, hq, d, dt=dt), rand(g, b, t, hk, d, dt=dt), rand(g, b, t, hk, d, dt=dt)
    do = rand(g, b, t, hq, d, dt=dt, std=2.0 ** -power)
    lens = [torch.tensor([t - 7 * i % 50 for i in range(b)], dtype=torch.int32, device="cuda") for _ in range(2)]
    ql, kl = lens if kind else (None, None)
    if kind:  # what lies past a sequence gives no range
        for i in range(b):
            do[i, int(ql[i]):], v[i, int(kl[i]):] = 60000.0, 60000.0
    o, lse = torch.empty_like(q), torch.empty(b, hq, t, device="cuda")
    h.heddle_attention(ctx, q, k, v, o, lse, q_lens=ql, kv_lens=kl)
    dq, dk, dv = (torch.full_like(x, CANARY) for x in (q, k, v))
    h.heddle_attention_backward(ctx, do, q, k, v, o, lse, dq, dk, dv, q_lens=ql, kv_lens=kl)
    n, small = hq // hk, 2.0 ** -power
    for i in sorted({0, b - 1}):
        nq, nk = (t, t) if ql is None else (int(ql[i]), int(kl[i]))
        for kv in range(hk):
            sums = {x: [torch.zeros(t, d, dtype=torch.float64, device="cuda") for _ in range(2)] for x in ("dk", "dv")}
            for j in range(kv * n, kv * n + n):
                large = do[i, :, j].double() / small
                w = R.attention(q[i, :, j], k[i, :, kv], v[i, :, kv], nq, nk, 0, 0, d ** -0.5, large)
                R.close(dq[i, :, j], w["dq"][0] * small, w["dq"][1] * small, "dq")
                for x in sums:
                    sums[x][0] += w[x][0] * small
                    sums[x][1] += (w[x][1] + n * 2.0 ** -23 * w[x][0].abs()) * small
            R.close(dk[i, :, kv], *sums["dk"], "dk")
            R.close(dv[i, :, kv], *sums["dv"], "dv")


def test_scores_gradients_beyond_float16_with_small_keys(lib):
    """Scores' gradients past 65504 whose products with small keys and queries
    are finite."""
    h, ctx = lib
    g, dt, t, d = gen(5), torch.float16, 24, 64
    q, k = (rand(g, 1, t, 1, d, dt=dt, std=0.002) for _ in range(2))
    v = rand(g, 1, t, 1, d, dt=dt, std=60.0)
    do = (torch.randn(1, t, 1, d, generator=g, device="cuda") * 6000).clamp(-20000, 20000).to(dt)
    o, lse = torch.empty_like(q), torch.empty(1, 1, t, device="cuda")
    h.heddle_attention(ctx, q, k, v, o, lse)
    dq, dk, dv = (torch.full_like(x, CANARY) for x in (q, k, v))
    h.heddle_attention_backward(ctx, do, q, k, v, o, lse, dq, dk, dv)
    w = R.attention(q[0, :, 0], k[0, :, 0], v[0, :, 0], t, t, 0, 0, d ** -0.5, do[0, :, 0])
    s = (q[0, :, 0].double() @ k[0, :, 0].double().T * d ** -0.5).masked_fill(
        ~R.visible(t, t, t, t, 0, 0, "cuda"), -math.inf)
    p, dp = s.softmax(1), do[0, :, 0].double() @ v[0, :, 0].double().T
    assert (p * (dp - (p * dp).sum(1, keepdim=True))).abs().max().item() * d ** -0.5 > 65504
    assert all(w[x][0].abs().max().item() < 60000 for x in ("dq", "dk", "dv"))
    for got, x in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        R.close(got[0, :, 0], *w[x], x)
