"""The layer operators at sizes that reach each of their kernels -- every tile
of the products, with and without pairs of CTAs and in both forms of the
epilogue; attention's tiles taken twice and the gradients that compute their
scores twice; norms that walk several heads -- and, without a GPU, that the
rules which choose the kernels choose them at these sizes on 152 SMs."""

import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

import op_reference as R  # noqa: E402
from test_gpu_operators import CANARY, TYPES, frame_kept, framed, gen, lib, product_inputs, rand  # noqa: E402, F401
from test_gpu_operators import test_attention as attention_test  # noqa: E402
from test_gpu_operators import test_qk_norm_rope as norm_test  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# m, n, k: rows in whole 32-byte units (results straight from tensor memory's
# rows), and odd ones (by way of shared memory); tiles end inside a pair's
# second CTA, before it, and inside its first
LINEAR_WHOLE = [(145, 11728, 80), (3958, 304, 304), (683, 656, 3552), (1793, 2640, 1552), (1923, 4912, 912),
                (867, 4192, 2784), (4182, 3392, 720), (1257, 11584, 848), (3984, 2064, 2064)]
LINEAR_ODD = [(134, 5057, 195), (282, 10745, 67), (265, 225, 3609), (129, 2235, 1609), (3728, 207, 965),
              (132, 9903, 1585), (1978, 1845, 2839), (4196, 8255, 271), (3915, 1055, 2417), (2808, 4183, 889),
              (304, 8517, 4179)]
GATED_WHOLE = [(152, 5280, 80), (135, 3680, 464), (259, 192, 3568), (567, 272, 3936), (2643, 976, 2320),
               (1381, 2576, 2384)]
GATED_ODD = [(129, 3283, 137), (129, 7585, 193), (265, 225, 3609), (1886, 1333, 1867), (413, 2655, 4193),
             (2108, 2745, 1281)]

# batch, q_len, kv_len, q heads, kv heads, head_dim, window, sinks, lens
TWINS = [(16, 1, 1100, 16, 8, 128, 0, 0, "kv"), (10, 1, 900, 24, 8, 64, 300, 4, "kv"),
         (9, 1, 1300, 16, 8, 128, 0, 0, "kv"), (20, 60, 700, 8, 4, 96, 250, 0, "kv"),
         (10, 128, 1024, 8, 8, 64, 128, 0, None), (11, 3, 2000, 14, 7, 72, 700, 40, None)]

# tokens, q heads, k heads, head_dim, rot_dim, interleaved, type
NORMS = [(5000, 9, 3, 256, 256, False, "bf16"), (4000, 9, 3, 256, 64, True, "fp16"),
         (3000, 9, 3, 128, 128, False, "fp32"), (10000, 11, 3, 128, 128, False, "bf16"),
         (9000, 10, 2, 96, 48, True, "fp16"), (20000, 10, 2, 64, 64, True, "bf16"),
         (16000, 9, 3, 80, 32, True, "fp32"), (30000, 3, 1, 64, 64, False, "fp16")]

# dS of all heads together, 2 bytes a pair, does not fit its room
TWICE = dict(batch=80, length=440, heads=128)


# ------------------------------------------------------- what is chosen

def chosen(tmp_path, source, body):
    """Lines that `body` prints, compiled behind one of the library's sources."""
    from paper_2609_34244_gb300 import _build
    src, exe = tmp_path / "chosen.cu", tmp_path / "chosen"
    src.write_text('#include "%s"\n#include <cstdio>\nint main() {\n    using namespace hd;\n    OpContext x;\n'
                   "    x.num_sms = 152;\n%s    return 0;\n}\n" % (source, body))
    pkg = os.path.dirname(_build.LIB)
    quick = ["-gencode", "arch=compute_103a,code=compute_103a", "-Xcicc", "-O0"]  # its kernels are not run
    subprocess.check_call([_build.nvcc(), *quick, "-std=c++17", "-I", _build.INCLUDE, "-I", _build.CSRC, str(src), "-o",
                           str(exe), "-L", pkg, "-lheddle", "-Xlinker", "-rpath", "-Xlinker", pkg])
    return [line.split() for line in subprocess.check_output([str(exe)], text=True).splitlines()]


def test_products_reach_every_tile(heddle_lib, tmp_path):
    body = "    const long long s[][4] = {%s};\n" % ", ".join(
        "{%d, %d, %d, %d}" % (*s, 2 * gated + whole) for gated, whole, list_ in
        ((0, 1, LINEAR_WHOLE), (0, 0, LINEAR_ODD), (1, 1, GATED_WHOLE), (1, 0, GATED_ODD)) for s in list_)
    body += r"""
    for (auto& r : s) {
        const bool gated = r[3] & 2, whole = r[3] & 1;
        GemmArgs f{}, dx{}, dw{};
        f.M = r[0], f.N = r[1], f.K = r[2], f.kind = gated ? kGemmGated : kGemmLinear, f.count = 1;
        dx.M = r[0], dx.N = r[2], dx.K = r[1], dx.kind = kGemmSum, dx.count = gated ? 2 : 1;
        dw.M = r[1], dw.N = r[2], dw.K = r[0], dw.kind = kGemmPair, dw.count = gated ? 2 : 1;
        for (auto* g : {&f, &dx, &dw}) {
            const Tile t = choose_tile(x, *g, whole);
            std::printf("%d %d %d %d %d\n", (int)gated, (int)whole, g->kind, t.bn, (int)t.pair);
        }
    }
"""
    got = {tuple(map(int, line)) for line in chosen(tmp_path, "heddle_gemm.cu", body)}
    for whole in (0, 1):
        for bn, pair in ((256, 1), (224, 1), (192, 1), (128, 1), (256, 0), (128, 0)):
            assert (0, whole, 0, bn, pair) in got, ("linear", whole, bn, pair)
        for bn, pair in ((256, 1), (128, 1), (256, 0), (128, 0)):
            assert (1, whole, 1, bn, pair) in got, ("gated", whole, bn, pair)
            for gated in (0, 1):
                for kind in (2, 3):
                    assert (gated, whole, kind, bn, pair) in got, (gated, whole, kind, bn, pair)


def test_attention_takes_tiles_twice(heddle_lib, tmp_path):
    body = "    const long long s[][8] = {%s};\n" % ", ".join("{%s}" % ", ".join(map(str, s[:8])) for s in TWINS)
    body += r"""
    for (auto& r : s) {
        heddle_attention_args a{};
        a.batch = r[0], a.q_len = r[1], a.kv_len = r[2], a.q_heads = (int)r[3], a.kv_heads = (int)r[4];
        a.head_dim = (int)r[5], a.window = r[6], a.sinks = r[7], a.scale = 0.1f;
        const Params p = params_of(x, a);
        std::printf("%d %d\n", p.twins, p.splits);
    }
    const int32_t lens[2] = {};
    for (int window : {0, 300}) {
        heddle_attention_args a{};
        a.batch = BATCH, a.q_len = a.kv_len = LENGTH, a.q_heads = HEADS, a.kv_heads = 1, a.head_dim = 64;
        a.window = window, a.q_lens = lens, a.kv_lens = lens + 1, a.scale = 0.1f;
        Params p = params_of(x, a);
        std::printf("%lld 0\n", (long long)keep_ds(x, p));
    }
""".replace("BATCH", str(TWICE["batch"])).replace("LENGTH", str(TWICE["length"])).replace("HEADS", str(TWICE["heads"]))
    got = [tuple(map(int, line)) for line in chosen(tmp_path, "heddle_attn_tc.cu", body)]
    assert all(twins for twins, _ in got[:len(TWINS)])
    assert {splits > 1 for _, splits in got[:len(TWINS)]} == {True, False}
    assert got[len(TWINS):] == [(0, 0), (0, 0)]  # dS is not kept


def test_norms_walk_several_heads(heddle_lib, tmp_path):
    code = {"bf16": 0, "fp16": 1, "fp32": 2}
    body = "    const int s[][6] = {%s};\n" % ", ".join(
        "{%d, %d, %d, %d, %d, %d}" % (t, hq, hk, d, rot, code[dt]) for t, hq, hk, d, rot, _, dt in NORMS)
    body += r"""
    for (auto& r : s) {
        heddle_qk_norm_rope_grad_args g{};
        g.fwd.tokens = r[0], g.fwd.q_heads = r[1], g.fwd.k_heads = r[2], g.fwd.head_dim = r[3];
        g.fwd.rot_dim = r[4], g.fwd.dtype = r[5];
        const Launch l = plan_rows(x, g, true);
        std::printf("%d %d %d\n", (int)l.wide, l.lanes, l.chunk);
    }
"""
    got = [tuple(map(int, line)) for line in chosen(tmp_path, "heddle_qknorm.cu", body)]
    assert all(wide and chunk > 1 for wide, _, chunk in got)
    assert {lanes for _, lanes, _ in got} == {8, 16, 32} and {chunk for _, _, chunk in got} == {2, 4, 8}


# ------------------------------------------------------------- on the GPU

@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k,whole", [(*s, True) for s in LINEAR_WHOLE] + [(*s, False) for s in LINEAR_ODD])
def test_linear_tiles(lib, m, n, k, whole, dt):
    h, ctx = lib
    dt = TYPES[dt]
    g, x, w = product_inputs(m, n, k, dt, m + n + k)
    b, r, dy = rand(g, n, dt=dt), rand(g, m, n, dt=dt), rand(g, m, n, dt=dt)
    for name, bias, res in (("none", b, r), ("gelu", b, r), ("none", None, None)):
        y, ybuf = framed(m, n, dt)
        pre, pbuf = framed(m, n, torch.float32) if name != "none" else (None, None)
        h.heddle_linear(ctx, x, w, y, bias=bias, residual=res, act=h.ACTIVATIONS[name], pre=pre)
        z, ez, want, ey = R.linear(x, w, bias, res, name)
        R.close(y, want, ey, "y %s" % name)
        frame_kept(y, ybuf, "y")
        if pre is not None:
            R.close(pre, z, ez, "pre")
            frame_kept(pre, pbuf, "pre")
        if res is not None:  # the residual may be the output itself
            y2 = res.clone()
            h.heddle_linear(ctx, x, w, y2, bias=bias, residual=y2, act=h.ACTIVATIONS[name])
            assert torch.equal(y2, y)
        del z, ez, want, ey
    dx, xbuf = framed(m, k, dt)
    dw, wbuf = framed(n, k, dt)
    h.heddle_linear_backward(ctx, dy, x, w, dx=dx, dw=dw)
    z = torch.zeros(m, n, dtype=torch.float64, device="cuda")
    wx, ww, _ = R.linear_grads(dy, x, w, z, z, "none")
    R.close(dx, *wx, "dx")
    R.close(dw, *ww, "dw")
    frame_kept(dx, xbuf, "dx")
    frame_kept(dw, wbuf, "dw")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k,whole", [(*s, True) for s in GATED_WHOLE] + [(*s, False) for s in GATED_ODD])
def test_gated_tiles(lib, m, n, k, whole, dt):
    h, ctx = lib
    dt, name = TYPES[dt], "silu" if whole else "gelu"
    act = h.ACTIVATIONS[name]
    g, x, wg = product_inputs(m, n, k, dt, m + n + k)
    wu, dy = rand(g, n, k, dt=dt, std=k ** -0.5), rand(g, m, n, dt=dt)
    y, ybuf = framed(m, n, dt)
    (gate, gbuf), (up, ubuf) = (framed(m, n, torch.float32) for _ in range(2))
    h.heddle_gated_ffn(ctx, x, wg, wu, y, act=act, gate=gate, up=up)
    zg, eg, zu, eu, want, ey = R.gated(x, wg, wu, name)
    for got, value, bound, buf in ((y, want, ey, ybuf), (gate, zg, eg, gbuf), (up, zu, eu, ubuf)):
        R.close(got, value, bound, "gated")
        frame_kept(got, buf, "gated")
    y2 = torch.empty(m, n, dtype=dt, device="cuda")
    h.heddle_gated_ffn(ctx, x, wg, wu, y2, act=act)
    assert torch.equal(y2, y)
    (dx, xbuf), (dwg, gbuf), (dwu, ubuf) = framed(m, k, dt), framed(n, k, dt), framed(n, k, dt)
    h.heddle_gated_ffn_backward(ctx, dy, x, wg, wu, gate, up, act=act, dx=dx, dwg=dwg, dwu=dwu)
    zero = torch.zeros_like(zg)
    wants = R.gated_grads(dy, x, wg, wu, gate.double(), zero, up.double(), zero, name)
    for got, (value, bound), buf in zip((dx, dwg, dwu), wants, (xbuf, gbuf, ubuf)):
        R.close(got, value, bound, "gated grads")
        frame_kept(got, buf, "gated grads")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("b,tq,tk,hq,hk,d,window,sinks,kind", TWINS)
def test_attention_twins(lib, b, tq, tk, hq, hk, d, window, sinks, kind, dt):
    attention_test(lib, b, tq, tk, hq, hk, d, window, sinks, kind, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("t,hq,hk,rot,d,inter,dt", [(t, hq, hk, rot, d, i, dt) for t, hq, hk, d, rot, i, dt in NORMS])
def test_norms_of_several_heads(lib, t, hq, hk, rot, d, inter, dt):
    norm_test(lib, t, hq, hk, d, rot, inter, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dt,window,sinks", [(64, "bf16", 0, 0), (64, "fp16", 300, 5), (128, "bf16", 300, 5),
                                               (128, "fp16", 0, 0), (96, "bf16", 50, 130)])
def test_attention_gradients_with_scores_computed_twice(lib, d, dt, window, sinks):
    h, ctx = lib
    b, t, hq, dt = TWICE["batch"], TWICE["length"], TWICE["heads"], TYPES[dt]
    g = gen(d + window)
    q, do = (rand(g, b, t, hq, d, dt=dt) for _ in range(2))
    k, v = (rand(g, b, t, 1, d, dt=dt) for _ in range(2))
    lens = [torch.full((b,), t, dtype=torch.int32, device="cuda") for _ in range(2)]
    lens[0][b - 1], lens[1][b - 1] = 301, 333
    o, lse = torch.full_like(q, CANARY), torch.empty(b, hq, t, device="cuda")
    rest = dict(q_lens=lens[0], kv_lens=lens[1], window=window, sinks=sinks)
    h.heddle_attention(ctx, q, k, v, o, lse, **rest)
    dq, dk, dv = (torch.full_like(x, CANARY) for x in (q, k, v))
    h.heddle_attention_backward(ctx, do, q, k, v, o, lse, dq, dk, dv, **rest)
    for i in (0, b - 1):
        sums = {x: [torch.zeros(t, d, dtype=torch.float64, device="cuda") for _ in range(2)] for x in ("dk", "dv")}
        for j in range(hq):
            w = R.attention(q[i, :, j], k[i, :, 0], v[i, :, 0], int(lens[0][i]), int(lens[1][i]), window, sinks,
                            d ** -0.5, do[i, :, j])
            R.close(o[i, :, j], *w["o"], "o")
            R.close(dq[i, :, j], *w["dq"], "dq")
            for x in sums:
                sums[x][0] += w[x][0]
                sums[x][1] += w[x][1] + hq * 2.0 ** -23 * w[x][0].abs()
        R.close(dk[i, :, 0], *sums["dk"], "dk")
        R.close(dv[i, :, 0], *sums["dv"], "dv")
