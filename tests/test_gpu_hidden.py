"""Layer norm, dropout, embedding and router against their definitions in 64
bits (tests/hidden_reference.py derives the bounds), at the sizes, masks,
strides and alignments where such kernels go wrong; their refusals; gradients
against differences; a run of them together."""

import math

import pytest

torch = pytest.importorskip("torch")

import hidden_reference as H  # noqa: E402
from op_reference import close  # noqa: E402
from test_gpu_operators import TYPES, frame_kept, framed, gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(heddle_lib):
    h = heddle_lib
    ctx = h.heddle_create(0)
    yield h, ctx
    torch.cuda.synchronize()
    flags = h.heddle_device_errors(ctx)
    h.heddle_destroy(ctx)
    assert flags == 0


def laid(t, pad, skip):
    v, buf = framed(*t.shape, t.dtype, pad, skip)
    v.copy_(t)
    return v


def floats(n):
    return torch.full((n,), 77.0, device="cuda")


LAYOUTS = [(0, 0), (8, 8), (3, 1)]  # spare columns, elements before the first

# ---------------------------------------------------------------- layer norm

ROWS = [(1, 1), (1, 4096), (3, 7), (5, 64), (17, 512), (33, 513), (64, 2047), (130, 2048), (40, 4096), (9, 8192),
        (7, 8191), (3, 16384), (4, 16385), (2, 70000), (5000, 64), (2500, 600), (700, 3000)]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n", ROWS)
def test_layer_norm(lib, m, n, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for i, (pad, skip) in enumerate(LAYOUTS):
        g = gen(m + n + i)
        x = laid(rand(g, m, n, dt=dt, std=2.0) + (3 if i == 1 else 0), pad, skip)
        w = None if i == 2 else 1 + rand(g, n, dt=dt, std=0.3)
        b = None if i == 0 else rand(g, n, dt=dt)
        y, buf = framed(m, n, dt, pad, skip)
        mean, rstd = floats(m), floats(m)
        h.heddle_layer_norm(ctx, x, w, b, y, mean=mean, rstd=rstd, eps=1e-5)
        (wm, em), (wr, er), (wy, ey) = H.layer_norm(x, w, b, 1e-5)
        close(mean, wm, em, "mean")
        close(rstd, wr, er, "rstd")
        close(y, wy, ey, "y")
        frame_kept(y, buf, "y")
        h.heddle_layer_norm(ctx, x, w, b, x)  # in place, nothing saved
        assert torch.equal(x, y)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n", ROWS)
def test_layer_norm_backward(lib, m, n, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for i, (pad, skip) in enumerate(LAYOUTS):
        g = gen(m * n + i)
        x, dy = laid(rand(g, m, n, dt=dt, std=2.0), pad, skip), laid(rand(g, m, n, dt=dt), pad, skip)
        w = None if i == 2 else 1 + rand(g, n, dt=dt, std=0.3)
        dres = None if i == 1 else laid(rand(g, m, n, dt=dt), pad, skip)
        mean, rstd = x.float().mean(1), (x.float().var(1, unbiased=False) + 1e-5).rsqrt()
        dx, buf = framed(m, n, dt, pad, skip)
        dw, db = floats(n), floats(n)
        h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=dx, dw=dw, dbias=db, dres=dres)
        (wx, ex), (ww, ew), (wb, eb) = H.layer_norm_grads(dy, x, w, mean, rstd, dres)
        close(dx, wx, ex, "dx")
        close(dw, ww, ew, "dw")
        close(db, wb, eb, "dbias")
        frame_kept(dx, buf, "dx")
        # parts of it, bit for bit, also in the place of an input
        for kw in ({"dw": floats(n)}, {"dbias": floats(n)}, {"dx": torch.empty_like(dx)}):
            h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dres=dres, **kw)
            for name, t in kw.items():
                assert torch.equal(t, {"dw": dw, "dbias": db, "dx": dx}[name]), name
        if dres is not None:
            h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dres=dres, dx=dres)
            assert torch.equal(dres, dx)
        dw2 = floats(n)
        h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=dy, dw=dw2)
        assert torch.equal(dw2, dw)
        if dres is None:
            assert torch.equal(dy, dx)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n", [(20000, 520), (9000, 1031), (20000, 1032), (2000, 5121), (3000, 8192), (1200, 8190),
                                 (700, 9000), (500, 16380), (60000, 64), (90000, 9), (20000, 257), (30000, 500)])
def test_layer_norm_of_many_rows_a_block(lib, m, n, dt):
    """More rows than a block holds ahead: places of the ring are taken again
    and again."""
    h, ctx = lib
    dt = TYPES[dt]
    g = gen(m + n)
    x, dy, dres = (rand(g, m, n, dt=dt) for _ in range(3))
    w, b = 1 + rand(g, n, dt=dt, std=0.3), rand(g, n, dt=dt)
    y, dx, mean, rstd, dw, db = torch.empty_like(x), torch.empty_like(x), floats(m), floats(m), floats(n), floats(n)
    h.heddle_layer_norm(ctx, x, w, b, y, mean=mean, rstd=rstd)
    (_, _), (_, _), (wy, ey) = H.layer_norm(x, w, b, 1e-5)
    close(y, wy, ey, "y")
    del wy, ey
    h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=dx, dw=dw, dbias=db, dres=dres)
    (wx, ex), (ww, ew), (wb, eb) = H.layer_norm_grads(dy, x, w, mean, rstd, dres)
    close(dx, wx, ex, "dx")
    close(dw, ww, ew, "dw")
    close(db, wb, eb, "dbias")
    again = [torch.empty_like(dx), floats(n), floats(n)]
    h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=again[0], dw=again[1], dbias=again[2], dres=dres)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw) and torch.equal(again[2], db)


def test_layer_norm_large_means_and_values_that_are_not_finite(lib):
    h, ctx = lib
    g = gen(3)
    for n in (300, 4096, 40000):
        x = rand(g, 6, n, dt=torch.float32) + 4096.0
        x[4, n // 2], x[5, n - 1] = float("inf"), float("nan")
        y = torch.empty_like(x)
        h.heddle_layer_norm(ctx, x, None, None, y)
        _, _, (wy, ey) = H.layer_norm(x[:4], None, None, 1e-5)
        close(y[:4], wy, ey, "y")
        assert y[4:].isnan().all()
        h.heddle_layer_norm(ctx, torch.full_like(x, 7.25), None, None, y)  # no variance at all
        assert (y == 0).all()


def test_layer_norm_of_nothing(lib):
    h, ctx = lib
    x = torch.empty(0, 40, device="cuda")
    h.heddle_layer_norm(ctx, x, None, None, x)
    dw, db = floats(40), floats(40)
    h.heddle_layer_norm_backward(ctx, x, x, None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), dx=x,
                                 dw=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()
    x = torch.empty(5, 0, device="cuda", dtype=torch.bfloat16)
    h.heddle_layer_norm(ctx, x, None, None, x, mean=floats(5), rstd=floats(5))
    h.heddle_layer_norm_backward(ctx, x, x, None, floats(5), floats(5), dx=x, dw=floats(0), dbias=floats(0))


def test_layer_norm_gradients_against_differences(lib):
    h, ctx = lib
    g = gen(5)
    m, n, eps = 4, 96, 1e-5
    x, dy, w, b = (rand(g, *s, dt=torch.float32) for s in ((m, n), (m, n), (n,), (n,)))
    y, mean, rstd = torch.empty_like(x), floats(m), floats(m)
    h.heddle_layer_norm(ctx, x, w, b, y, mean=mean, rstd=rstd, eps=eps)
    dx, dw, db = torch.empty_like(x), floats(n), floats(n)
    h.heddle_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=dx, dw=dw, dbias=db)

    def value(x, w, b):
        v = x.double()
        v = (v - v.mean(1, keepdim=True)) / (v.var(1, unbiased=False, keepdim=True) + eps).sqrt()
        return ((v * w.double() + b.double()) * dy.double()).sum()

    step = 1e-4
    for t, d in ((x, dx), (w, dw), (b, db)):
        for i in (0, 17, t.numel() - 1):
            one = torch.zeros(t.numel(), dtype=torch.float64, device="cuda")
            one[i] = step
            args = [[v.double() + s * one.view(t.shape) if v is t else v for v in (x, w, b)] for s in (1, -1)]
            want = (value(*args[0]) - value(*args[1])) / (2 * step)
            assert abs(want - d.view(-1)[i].double()) < 1e-5 * (1 + want.abs())


# ------------------------------------------------------------------- dropout

@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 4099), (3, 7), (64, 1024), (33, 1000), (50, 130), (301, 2049)])
def test_dropout(lib, m, n, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for i, ((pad, skip), p, seed, offset) in enumerate(zip(
            LAYOUTS * 2, (0.1, 0.5, 0.0, 0.999, 0.35, 1 - 2.0 ** -40),
            (0, 2 ** 64 - 1, 5, 2 ** 32, 0x123456789ABCDEF, 7), (0, 2 ** 64 - 1, 3, 2 ** 32, 2 ** 63, 1))):
        g = gen(m + n + i)
        x = laid(rand(g, m, n, dt=dt, std=2.0), pad, skip)
        res = laid(rand(g, m, n, dt=dt), pad, skip) if i % 2 else None
        y, buf = framed(m, n, dt, pad, skip)
        h.heddle_dropout(ctx, x, y, p, seed, offset=offset, residual=res)
        want, bound = H.dropout(x, p, seed, offset, res)
        close(y, want, bound, "y")
        frame_kept(y, buf, "y")
        dx, buf = framed(m, n, dt, pad, skip)
        h.heddle_dropout_backward(ctx, x, dx, p, seed, offset=offset)
        want, bound = H.dropout(x, p, seed, offset, None)
        close(dx, want, bound, "dx")
        frame_kept(dx, buf, "dx")
        # the offset in two parts, and in the place of an input
        step = torch.tensor([-3], device="cuda")
        h.heddle_dropout(ctx, x, x, p, seed, offset=(offset + 3) % 2 ** 64, residual=res, step=step)
        assert torch.equal(x, y)
        if res is not None:
            before = res.clone()
            h.heddle_dropout(ctx, torch.zeros_like(res), res, 0.25, 1, residual=res)
            assert torch.equal(res, before)


def test_dropout_mask_is_of_the_elements_not_their_places(lib):
    """Strides, alignment and type do not change which elements are dropped;
    what is dropped counts for nothing."""
    h, ctx = lib
    m, n = 37, 136
    keep = None
    for dt in TYPES.values():
        for pad, skip in LAYOUTS + [(1, 0), (8, 0)]:
            x = laid(torch.ones(m, n, device="cuda", dtype=dt), pad, skip)
            y = torch.empty_like(x)
            h.heddle_dropout(ctx, x, y, 0.5, 11, offset=4)
            keep = y != 0 if keep is None else keep
            assert torch.equal(y != 0, keep)
            x = laid(torch.where(keep, 1.0, float("nan")).to(dt), pad, skip)
            h.heddle_dropout(ctx, x, y, 0.5, 11, offset=4, residual=torch.ones_like(x))
            assert torch.equal(y, torch.where(keep, 3.0, 1.0).to(dt))
    other = torch.empty(m, n, device="cuda")
    for kw in ({"seed": 12, "offset": 4}, {"seed": 11, "offset": 5}, {"seed": 11 + 2 ** 32, "offset": 4},
               {"seed": 11, "offset": 4 + 2 ** 32}):
        h.heddle_dropout(ctx, torch.ones(m, n, device="cuda"), other, 0.5, **kw)
        # independent masks agree in half of the elements, give or take five deviations
        assert abs(((other != 0) == keep).double().mean() - 0.5) < 2.5 / math.sqrt(m * n)


@pytest.mark.parametrize("p", [0.01, 0.1, 0.5, 0.9])
def test_dropout_share(lib, p):
    h, ctx = lib
    x = torch.ones(1000, 2000, device="cuda")
    y = torch.empty_like(x)
    h.heddle_dropout(ctx, x, y, p, 99)
    dropped = (y == 0).double()
    assert abs(dropped.mean() - p) < 5 * math.sqrt(p * (1 - p) / x.numel())
    assert (dropped.mean(0) - p).abs().max() < 6.5 * math.sqrt(p * (1 - p) / 1000)
    assert (dropped.mean(1) - p).abs().max() < 6.5 * math.sqrt(p * (1 - p) / 2000)


def test_dropout_of_nothing(lib):
    h, ctx = lib
    for shape in ((0, 5), (5, 0)):
        x = torch.empty(*shape, device="cuda")
        h.heddle_dropout(ctx, x, x, 0.5, 1)
        h.heddle_dropout_backward(ctx, x, x, 0.5, 1)


def test_dropout_elements_past_32_bits(lib):
    h, ctx = lib
    m, n = 3, 2 ** 31 - 8
    x = torch.ones(m, n, device="cuda", dtype=torch.float16)
    h.heddle_dropout(ctx, x, x, 0.5, 3, offset=9)
    flat = x.view(-1)
    for first in (0, 2 ** 31 - 64, 2 ** 32 - 64, m * n - 128):
        want, _ = H.dropout(torch.ones(128, device="cuda"), 0.5, 3, 9, None, first)
        assert torch.equal(flat[first:first + 128].double(), want)


# ----------------------------------------------------------------- embedding

def token_list(g, t, vocab, kind):
    if kind == "one":
        return torch.full((t,), vocab // 2, device="cuda")
    if kind == "each":
        return torch.randperm(max(t, vocab), generator=g, device="cuda")[:t] % vocab
    u = torch.rand(t, generator=g, device="cuda", dtype=torch.float64)
    return ((vocab + 1.0) ** u - 1).long().clamp(0, vocab - 1)


LOOKUPS = [  # tokens, vocabulary, shards, columns
    (1, 1, 1, 1), (1, 100, 1, 64), (16, 32000, 1, 4096), (5, 40, 4, 7), (300, 1000, 1, 136), (1000, 600, 3, 513),
    (2100, 70, 1, 1023), (4097, 5000, 2, 200), (40000, 300000, 1, 24), (33000, 4096, 1, 40), (3000, 1 << 20, 1, 8),
    (70001, 33, 1, 130), (600, 1200, 1, 5000), (600000, 50, 1, 8), (9000, 900, 1, 1040),
    (512, 30000, 1, 40), (513, 30000, 1, 40), (500, 1 << 20, 1, 4),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,vocab,shards,n", LOOKUPS)
def test_embedding(lib, t, vocab, shards, n, dt):
    h, ctx = lib
    dt = TYPES[dt]
    rows = vocab // shards
    for i, (kind, (pad, skip)) in enumerate(zip(("zipf", "one", "each"), LAYOUTS)):
        g = gen(t + vocab + i)
        tokens = token_list(g, t, vocab, kind)
        if t > 4:
            tokens[::7], tokens[3] = -1, -2 ** 31
        if i != 1:
            tokens = tokens.int()
        first = rows * (shards // 2)
        scale = (1.0, 0.75, 22.625)[i]
        table = laid(rand(g, rows, n, dt=dt), pad, skip)
        kw = dict(scale=scale, first=first, vocab=vocab)
        y, buf = framed(t, n, dt, pad, skip)
        h.heddle_embedding(ctx, tokens, table, y, **kw)
        want, bound = H.embedding(tokens, table, scale, first)
        close(y, want, bound, "y")
        frame_kept(y, buf, "y")
        dy = laid(rand(g, t, n, dt=dt), pad, skip)
        for to in {dt, torch.float32}:
            for accumulate in (False, True):
                d, buf = framed(rows, n, to, pad, skip)
                base = rand(g, rows, n, dt=to) if accumulate else None
                if accumulate:
                    d.copy_(base)
                h.heddle_embedding_backward(ctx, tokens, dy, d, accumulate=accumulate, **kw)
                want, bound = H.embedding_grad(tokens, dy, rows, scale, first, base)
                close(d, want, bound, "dtable")
                frame_kept(d, buf, "dtable")
                again = base.clone() if accumulate else torch.empty(rows, n, dtype=to, device="cuda")
                h.heddle_embedding_backward(ctx, tokens, dy, again, accumulate=accumulate, **kw)
                assert torch.equal(again, d)


def test_embedding_of_nothing(lib):
    h, ctx = lib
    none, table = torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(9, 5, device="cuda")
    h.heddle_embedding(ctx, none, table, torch.empty(0, 5, device="cuda"))
    h.heddle_embedding_backward(ctx, none, torch.empty(0, 5, device="cuda"), table, accumulate=True)
    assert (table == 1).all()
    h.heddle_embedding_backward(ctx, none, torch.empty(0, 5, device="cuda"), table)
    assert (table == 0).all()
    tokens, y = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(4, 5, device="cuda")
    h.heddle_embedding(ctx, tokens, torch.empty(0, 5, device="cuda"), y, first=3, vocab=9)  # an empty shard
    assert (y == 0).all()
    h.heddle_embedding_backward(ctx, tokens, y, torch.empty(0, 5, device="cuda"), first=3, vocab=9)
    h.heddle_embedding(ctx, tokens, torch.empty(9, 0, device="cuda"), torch.empty(4, 0, device="cuda"))
    h.heddle_embedding_backward(ctx, tokens, torch.empty(4, 0, device="cuda"), torch.empty(9, 0, device="cuda"))


def test_embedding_shards_add_up_and_padding_gives_zeros(lib):
    h, ctx = lib
    g = gen(8)
    table, tokens = rand(g, 40, 72, dt=torch.float32), torch.randint(-3, 40, (200,), generator=g, device="cuda")
    whole, part, total = torch.empty(200, 72, device="cuda"), torch.empty(200, 72, device="cuda"), 0
    h.heddle_embedding(ctx, tokens, table, whole)
    for first in range(0, 40, 10):
        h.heddle_embedding(ctx, tokens, table[first:first + 10], part, first=first, vocab=40)
        total = total + part
    assert torch.equal(total, whole)
    assert (whole[tokens < 0] == 0).all() and (whole[tokens >= 0] != 0).any()


@pytest.mark.parametrize("wide", [torch.int32, torch.int64])
def test_tokens_past_the_vocabulary_raise_the_flag(lib, wide):
    h, ctx = lib
    table = torch.ones(10, 64, device="cuda")
    y = torch.empty(3, 64, device="cuda")
    far = torch.iinfo(wide).max
    h.heddle_embedding(ctx, torch.tensor([1, 9, -far - 1], dtype=wide, device="cuda"), table, y)
    assert h.heddle_device_errors(ctx) == 0
    h.heddle_embedding(ctx, torch.tensor([1, 10, far], dtype=wide, device="cuda"), table, y)
    assert h.heddle_device_errors(ctx) == 64
    assert (y[0] == 1).all() and (y[1:] == 0).all()
    d = torch.empty(10, 64, device="cuda")
    h.heddle_embedding_backward(ctx, torch.tensor([1, 10, far], dtype=wide, device="cuda"), torch.ones_like(y), d)
    assert h.heddle_device_errors(ctx) == 64
    assert (d[1] == 1).all() and d.sum() == 64
    # of another shard: no mistake
    h.heddle_embedding(ctx, torch.tensor([1, 10, 19], dtype=wide, device="cuda"), table, y, vocab=20)
    assert h.heddle_device_errors(ctx) == 0


def test_embedding_tables_past_32_bits(lib):
    h, ctx = lib
    rows, n = 1_100_000, 4096
    table = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([0, rows - 1, rows // 2, rows - 1], device="cuda")
    table[tokens] = torch.tensor([1.0, 4.0, 2.0, 4.0], device="cuda", dtype=torch.bfloat16)[:, None]
    y = torch.empty(4, n, dtype=torch.bfloat16, device="cuda")
    h.heddle_embedding(ctx, tokens, table, y)
    assert torch.equal(y[:, 0].float(), torch.tensor([1.0, 4.0, 2.0, 4.0], device="cuda"))
    assert (y == y[:, :1]).all()
    table.fill_(3.0)
    h.heddle_embedding_backward(ctx, tokens, y, table)
    assert (table[rows - 1] == 8).all() and (table[rows // 2] == 2).all() and (table[0] == 1).all()
    table[tokens] = 0
    assert not table.any()


@pytest.mark.parametrize("n,dt", [(4, "fp32"), (3, "bf16")])
@pytest.mark.parametrize("t", [50, 70000])
def test_embedding_gradient_of_many_rows(lib, t, n, dt):
    # more rows a block than it marks at a time; with many tokens half of one row
    h, ctx = lib
    g, rows, dt = gen(t + n), 20_000_003, TYPES[dt]
    tokens = torch.randint(0, rows, (t,), generator=g, device="cuda")
    if t > 100:
        tokens[torch.rand(t, generator=g, device="cuda") < 0.5] = 8200
    dy, d = rand(g, t, n, dt=dt), torch.full((rows, n), 3.0, dtype=dt, device="cuda")
    h.heddle_embedding_backward(ctx, tokens, dy, d)
    own, at = torch.unique(tokens, return_inverse=True)
    want, bound = H.embedding_grad(at, dy, len(own), 1.0, 0, None)
    close(d[own], want, bound, "dtable")
    d[own] = 0
    assert not d.any()


# -------------------------------------------------------------------- router

def routed(h, ctx, logits, k, valid, normalize, loss=True):
    t, n = logits.shape
    out = [torch.full((t, k), 77, dtype=torch.int32, device="cuda"), torch.full((t, k), 77.0, device="cuda"),
           torch.full((n + 1,), 77, dtype=torch.int32, device="cuda"), floats(1) if loss else None]
    h.heddle_router(ctx, logits, *out[:3], loss=out[3], valid=valid, normalize=normalize)
    return out


def check_router(h, ctx, logits, k, valid, normalize, g, pad=0, skip=0):
    experts, weights, counts, loss = routed(h, ctx, logits, k, valid, normalize)
    r = H.router(logits, k, valid, normalize)
    assert torch.equal(experts, r["experts"])
    assert torch.equal(counts, r["counts"])
    near = ~r["bad"]
    close(weights[near], r["weights"][near], r["eweights"][near], "weights")
    assert weights[r["bad"]].isnan().all()
    if r["bad"].any():
        assert loss.isnan().all()
    else:
        close(loss, r["loss"], r["eloss"], "loss")
    t, n = logits.shape
    dweights, dloss = rand(g, t, k, dt=torch.float32), rand(g, 1, dt=torch.float32, std=3.0)
    for dw, dl in ((dweights, dloss), (dweights, None), (None, dloss), (None, None)):
        d, buf = framed(t, n, logits.dtype, pad, skip)
        h.heddle_router_backward(ctx, logits, experts, weights, counts, d, dweights=dw, dloss=dl, valid=valid,
                                 normalize=normalize)
        want, bound = H.router_grad(r, logits, k, normalize, dw, dl)
        close(d[near], want[near], bound[near], "dlogits")
        assert d[r["bad"]].isnan().all()
        assert (d[~r["plain"] & near] == 0).all()
        frame_kept(d, buf, "dlogits")
    return r


ROUTERS = [  # tokens, experts, chosen
    (1, 1, 1), (1, 64, 2), (5, 2, 2), (16, 64, 2), (33, 7, 3), (100, 64, 8), (70, 60, 32), (301, 65, 4), (3000, 8, 2),
    (40, 128, 8), (77, 250, 8), (64, 256, 32), (19, 512, 6), (9, 1000, 5), (6, 1024, 32), (20001, 16, 2),
    (64, 64, 2), (65, 64, 2), (200, 1024, 32), (100, 512, 6), (5000, 250, 8), (33, 100, 1),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,n,k", ROUTERS)
def test_router(lib, t, n, k, dt):
    h, ctx = lib
    dt = TYPES[dt]
    for i, (pad, skip) in enumerate(LAYOUTS):
        g = gen(t * n + i)
        logits = laid(rand(g, t, n, dt=dt, std=2.0), pad, skip)
        valid = None
        if i:
            valid = torch.rand(t, generator=g, device="cuda") < 0.7
            logits[torch.rand(t, n, generator=g, device="cuda") < 0.2] = float("-inf")
            logits[t // 2] = float("-inf")
        if i == 2:
            valid = valid.to(torch.uint8) * 200
        check_router(h, ctx, logits, k, valid, i != 1, g, pad, skip)


def test_router_equal_logits_go_by_index(lib):
    h, ctx = lib
    for n, k in ((16, 4), (64, 9), (300, 17), (1024, 32)):
        for dt in TYPES.values():
            logits = torch.zeros(3, n, device="cuda", dtype=dt)
            logits[1, n - 1] = 1.0
            logits[2, ::2] = -0.0
            experts, weights, counts, _ = routed(h, ctx, logits, k, None, True)
            assert experts[0].tolist() == list(range(k)) == experts[2].tolist()
            assert experts[1].tolist() == [n - 1] + list(range(k - 1))
            assert counts[n] == 3 and counts[:n].sum() == 3 * k


@pytest.mark.parametrize("n,k", [(60, 5), (100, 8), (250, 16), (500, 7), (1000, 32)])
def test_router_few_values(lib, n, k):
    h, ctx = lib
    for dt in TYPES.values():
        logits = torch.randint(-2, 3, (999, n), generator=gen(n), device="cuda").to(dt)
        logits[::5, 3:] = float("-inf")  # three are left
        experts, _, _, _ = routed(h, ctx, logits, k, None, True)
        want = torch.sort(logits.float(), dim=1, descending=True, stable=True).indices[:, :k]
        want[::5, 3:] = -1
        assert torch.equal(experts.long(), want)


def test_router_values_that_are_not_finite(lib):
    h, ctx = lib
    for n, k in ((8, 2), (64, 3), (200, 8)):
        g = gen(n)
        logits = rand(g, 9, n, dt=torch.float32)
        logits[1, 3] = float("nan")
        logits[2, 0] = float("inf")
        logits[3] = float("-inf")
        logits[4] = float("-inf")
        logits[4, 5] = 0.5           # one expert is left
        logits[5] = float("nan")     # padding may hold anything
        logits[6, :2] = torch.tensor([float("inf"), float("nan")])
        logits[7] = torch.finfo(torch.float32).min  # the type's lowest value is a value
        logits[8] = float("-inf")
        logits[8, 1] = float("nan")
        valid = torch.ones(9, dtype=torch.bool, device="cuda")
        valid[5] = False
        for normalize in (True, False):
            r = check_router(h, ctx, logits, k, valid, normalize, g)
            assert r["bad"].tolist() == [False, True, True, False, False, False, True, False, True]
            assert r["experts"][4].tolist() == [5] + [-1] * (k - 1)
            fine = torch.tensor([0, 3, 4, 5, 7], device="cuda")
            check_router(h, ctx, logits[fine].contiguous(), k, valid[fine].contiguous(), normalize, g)


def test_router_of_nothing(lib):
    h, ctx = lib
    logits = torch.empty(0, 12, device="cuda")
    experts, weights, counts, loss = routed(h, ctx, logits, 3, None, True)
    assert (counts == 0).all() and (loss == 0).all()
    h.heddle_router_backward(ctx, logits, experts, weights, counts, logits, dloss=loss)
    logits = torch.randn(20, 12, device="cuda")
    valid = torch.zeros(20, dtype=torch.bool, device="cuda")
    experts, weights, counts, loss = routed(h, ctx, logits, 3, valid, True)
    assert (counts == 0).all() and (loss == 0).all() and (experts == -1).all() and (weights == 0).all()
    h.heddle_router_backward(ctx, logits, experts, weights, counts, logits, dloss=torch.ones(1, device="cuda"),
                             dweights=torch.ones_like(weights), valid=valid)
    assert (logits == 0).all()


def test_router_gradients_against_differences(lib):
    h, ctx = lib
    g = gen(4)
    t, n, k = 6, 20, 3
    logits = rand(g, t, n, dt=torch.float32)
    dw, dl = rand(g, t, k, dt=torch.float32), torch.tensor([2.0], device="cuda")
    for normalize in (True, False):
        experts, weights, counts, _ = routed(h, ctx, logits, k, None, normalize)
        d = torch.empty_like(logits)
        h.heddle_router_backward(ctx, logits, experts, weights, counts, d, dweights=dw, dloss=dl, normalize=normalize)

        def value(l):
            p = torch.softmax(l, 1)
            w = p.gather(1, experts.long())
            if normalize:
                w = w / w.sum(1, keepdim=True)
            f = counts[:n].double() / (k * t)
            return (w * dw.double()).sum() + 2.0 * n * (f * p.mean(0)).sum()

        for i, j in ((0, int(experts[0, 0])), (0, int(experts[0, 2])), (3, 11), (5, 19)):
            one = torch.zeros(t, n, dtype=torch.float64, device="cuda")
            one[i, j] = 1e-4
            want = (value(logits.double() + one) - value(logits.double() - one)) / 2e-4
            assert abs(want - d[i, j].double()) < 2e-6 * (1 + want.abs())


# ---------------------------------------------------------- streams and graphs

def every_call(h, ctx, s, step):
    """A run of all of them, as a stage's first layer uses them: the embedding,
    dropout, a norm, the router on it, and back."""
    t, n, e, k = s["t"], s["n"], s["e"], s["k"]
    dt = s["table"].dtype

    def buf(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    o = {"h": buf(t, n), "x": buf(t, n), "y": buf(t, n), "mean": buf(t, dtype=torch.float32),
         "rstd": buf(t, dtype=torch.float32), "logits": buf(t, e), "experts": buf(t, k, dtype=torch.int32),
         "weights": buf(t, k, dtype=torch.float32), "counts": buf(e + 1, dtype=torch.int32),
         "loss": buf(1, dtype=torch.float32), "dlogits": buf(t, e), "dy": buf(t, n), "dx": buf(t, n), "dh": buf(t, n),
         "dw": buf(n, dtype=torch.float32), "db": buf(n, dtype=torch.float32), "dwr": buf(e, n),
         "dtable": torch.empty_like(s["table"])}

    def run():
        h.heddle_embedding(ctx, s["tokens"], s["table"], o["h"], scale=2.0)
        h.heddle_dropout(ctx, o["h"], o["x"], 0.1, 42, step=step)
        h.heddle_layer_norm(ctx, o["x"], s["w"], s["b"], o["y"], mean=o["mean"], rstd=o["rstd"])
        h.heddle_linear(ctx, o["y"], s["wr"], o["logits"])
        h.heddle_router(ctx, o["logits"], o["experts"], o["weights"], o["counts"], loss=o["loss"])
        h.heddle_router_backward(ctx, o["logits"], o["experts"], o["weights"], o["counts"], o["dlogits"],
                                 dweights=s["dweights"], dloss=s["dloss"])
        h.heddle_linear_backward(ctx, o["dlogits"], o["y"], s["wr"], dx=o["dy"], dw=o["dwr"])
        h.heddle_layer_norm_backward(ctx, o["dy"], o["x"], s["w"], o["mean"], o["rstd"], dx=o["dx"], dw=o["dw"],
                                     dbias=o["db"], dres=s["dres"])
        h.heddle_dropout_backward(ctx, o["dx"], o["dh"], 0.1, 42, step=step)
        h.heddle_embedding_backward(ctx, s["tokens"], o["dh"], o["dtable"], scale=2.0)

    return o, run


def stage(seed, t=900, n=264, e=24, k=2, vocab=500, dt=torch.bfloat16):
    g = gen(seed)
    return dict(t=t, n=n, e=e, k=k, tokens=torch.randint(0, vocab, (t,), generator=g, device="cuda"),
                table=rand(g, vocab, n, dt=dt), w=1 + rand(g, n, dt=dt, std=0.1), b=rand(g, n, dt=dt, std=0.1),
                wr=rand(g, e, n, dt=dt, std=n ** -0.5), dweights=rand(g, t, k, dt=torch.float32),
                dloss=torch.full((1,), 0.1, device="cuda"), dres=rand(g, t, n, dt=dt))


def test_a_run_of_all_against_autograd(lib):
    """The calls one after the other give what one graph of plain operations
    in 64 bits gives, up to the roundings of the values between them (each off
    by half a step of bfloat16, 2^-8: a dozen of them, whose errors mostly do
    not line up: 2 % of a gradient's norm)."""
    h, ctx = lib
    s = stage(1)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    o, run = every_call(h, ctx, s, step)
    run()
    t, n, e, k = s["t"], s["n"], s["e"], s["k"]
    leaf = {x: s[x].double().requires_grad_(True) for x in ("table", "w", "b", "wr")}
    keep = (H.numbers(0, t * n, 42, 0, "cuda") >= round(0.1 * 2 ** 32)).view(t, n).double()
    x = leaf["table"][s["tokens"]] * 2.0 * keep / 0.9
    y = torch.nn.functional.layer_norm(x, (n,), leaf["w"], leaf["b"], 1e-5)
    p = torch.softmax(y @ leaf["wr"].T, 1)
    w = p.gather(1, o["experts"].long())  # near ties may be chosen otherwise
    w = w / w.sum(1, keepdim=True)
    f = o["counts"][:e].double() / (k * t)
    loss = e * (f * p.mean(0)).sum()
    grads = torch.autograd.grad((w * s["dweights"].double()).sum() + 0.1 * loss + (x * s["dres"].double()).sum(),
                                list(leaf.values()))
    for name, want in zip(("dtable", "dw", "db", "dwr"), grads):
        off = (o[name].double() - want).norm() / want.norm()
        assert off < 0.02, "%s: %.3g" % (name, off)
    assert (o["weights"].double() - w.detach()).abs().max() < 0.05
    assert abs(o["loss"].item() - loss.item()) < 0.01 * loss.item()


def test_captured_and_replayed(lib):
    h, ctx = lib
    s = stage(2)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    o, run = every_call(h, ctx, s, step)
    run()
    first = {x: v.clone() for x, v in o.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            run()
            step.add_(1)
    torch.cuda.synchronize()
    for v in o.values():
        v.zero_()
    step.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for x, v in o.items():
        assert torch.equal(v, first[x]), x
    masks = [o["x"] != 0]
    graph.replay()  # the step has moved on: another mask
    torch.cuda.synchronize()
    masks.append(o["x"] != 0)
    assert not torch.equal(*masks)
    # beside larger calls of the same context, which let its scratch grow
    big = stage(3, t=4000, n=512, vocab=3000)
    every_call(h, ctx, big, step)[1]()
    torch.cuda.synchronize()
    step.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for x, v in o.items():
        assert torch.equal(v, first[x]), x


def test_calls_on_two_streams_take_turns_at_the_scratch(lib):
    h, ctx = lib
    sets = [stage(i, t=2000, n=512, vocab=900) for i in (5, 6)]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    want = []
    for s in sets:
        o, run = every_call(h, ctx, s, step)
        run()
        torch.cuda.synchronize()
        want.append({x: v.clone() for x, v in o.items()})
    streams = [torch.cuda.Stream() for _ in sets]
    outs = []
    for _ in range(5):
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                o, run = every_call(h, ctx, s, step)
                run()
                outs.append(o)
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        for x, v in o.items():
            assert torch.equal(v, want[i % 2][x]), x


# ------------------------------------------------------------------- refusals

def test_tensors_of_another_device_are_refused(lib):
    """A stand-in reports the context's device: no operator's function may be
    entered where it is not the tensors'; names left out stay bound."""
    import ctypes
    h, ctx = lib
    native, entered = h._op_setup(), []

    @ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p)
    def operator(c, a, s):
        entered.append(c)
        return 0

    @ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p)
    def device(c):
        return where

    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    x, v, w = torch.zeros(4, 8, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, 2, device="cuda")
    t, e, c = (torch.zeros(*n, dtype=torch.int32, device="cuda") for n in ((4,), (4, 2), (9,)))
    calls = [(h.heddle_layer_norm, (x, None, None, x)), (h.heddle_layer_norm_backward, (x, x, None, v, v, x)),
             (h.heddle_dropout, (x, x, 0.5, 1)), (h.heddle_dropout_backward, (x, x, 0.5, 1)),
             (h.heddle_embedding, (t, x, x)), (h.heddle_embedding_backward, (t, x, x)),
             (h.heddle_router, (x, e, w, c)), (h.heddle_router_backward, (x, e, w, c, x))]
    assert len(calls) == len(h._HIDDEN_NAMES)
    old = dict.fromkeys(h._OP_NAMES, address(operator))
    old["heddle_device"] = address(device)
    try:
        for names in ({**old, **dict.fromkeys(h._HIDDEN_NAMES, address(operator))}, old):
            native.bind(names, h.HeddleError, lambda index: 0)
            for where in (torch.cuda.current_device(), torch.cuda.current_device() + 1):
                for f, args in calls:
                    entered.clear()
                    if where == torch.cuda.current_device():
                        f(ctx, *args)
                        assert len(entered) == 1
                    else:
                        with pytest.raises(h.HeddleError, match="the context is of") as err:
                            f(ctx, *args)
                        assert err.value.status == h.E_ARG and not entered
    finally:
        h._op_setup()


def test_refusals(lib):
    h, ctx = lib
    x, y = torch.ones(4, 16, device="cuda"), torch.ones(4, 16, device="cuda")
    f4, f16 = floats(4), floats(16)
    tokens = torch.zeros(4, dtype=torch.int32, device="cuda")
    i2, w2, c = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"), \
        torch.zeros(17, dtype=torch.int32, device="cuda")
    calls = [
        (h.heddle_layer_norm, (x, f4, None, y), {}), (h.heddle_layer_norm, (x, None, None, y[:3]), {}),
        (h.heddle_layer_norm, (x, None, None, y), {"eps": -1.0}),
        (h.heddle_layer_norm, (x, None, None, y), {"eps": float("nan")}),
        (h.heddle_layer_norm, (x, None, None, y), {"mean": f4}),
        (h.heddle_layer_norm, (x, None, None, y.bfloat16()), {}), (h.heddle_layer_norm, (x, None, None, y.T), {}),
        (h.heddle_layer_norm, (x.expand(4, 16)[:, :1].expand(4, 16), None, None, y), {}),
        (h.heddle_layer_norm, (x, None, None, None), {}), (h.heddle_layer_norm, (x.int(), None, None, y), {}),
        (h.heddle_layer_norm, (x[0].expand(4, 16), None, None, y), {}),
        (h.heddle_layer_norm_backward, (x, x, None, None, None), {"dx": y}),
        (h.heddle_layer_norm_backward, (x, x, None, f4, f16), {"dx": y}),
        (h.heddle_layer_norm_backward, (x, x, None, f4, f4), {"dw": f4}),
        (h.heddle_layer_norm_backward, (None, x, None, f4, f4), {"dx": y}),
        (h.heddle_dropout, (x, y, 1.0, 0), {}), (h.heddle_dropout, (x, y, -0.1, 0), {}),
        (h.heddle_dropout, (x, y, float("nan"), 0), {}), (h.heddle_dropout, (x, y, 0.1, 0), {"step": c}),
        (h.heddle_dropout, (x, y, 0.1, 0), {"residual": y[:2]}), (h.heddle_dropout, (x, None, 0.1, 0), {}),
        (h.heddle_dropout_backward, (x, y, 1.5, 0), {}), (h.heddle_dropout_backward, (x, y.half(), 0.1, 0), {}),
        (h.heddle_embedding, (tokens.float(), x, y), {}), (h.heddle_embedding, (tokens[:3], x, y), {}),
        (h.heddle_embedding, (tokens, x, y), {"first": -1}), (h.heddle_embedding, (tokens, x, y), {"vocab": 3}),
        (h.heddle_embedding, (tokens, x, y), {"first": 2, "vocab": 5}),
        (h.heddle_embedding, (tokens, x, y), {"first": 2 ** 63 - 2, "vocab": 2 ** 63 - 1}),
        (h.heddle_embedding, (tokens, x, y), {"scale": float("inf")}), (h.heddle_embedding, (None, x, y), {}),
        (h.heddle_embedding, (tokens, x.half(), y), {}), (h.heddle_embedding, (tokens, None, y), {}),
        (h.heddle_embedding_backward, (tokens, x, y.bfloat16()), {}),
        (h.heddle_embedding_backward, (tokens, x.half(), y.bfloat16()), {}),
        (h.heddle_embedding_backward, (tokens, x, y[:, :8]), {}),
        (h.heddle_router, (x, i2, w2, c[:16]), {}), (h.heddle_router, (x, i2, w2, None), {}),
        (h.heddle_router, (x, i2.long(), w2, c), {}), (h.heddle_router, (x, i2, w2[:, :1], c), {}),
        (h.heddle_router, (x, i2.new_zeros(4, 17), w2.new_zeros(4, 17), c), {}),
        (h.heddle_router, (x, i2.new_zeros(4, 0), w2.new_zeros(4, 0), c), {}),
        (h.heddle_router, (x, i2, w2, c), {"valid": tokens}), (h.heddle_router, (x, i2, w2, c), {"loss": f4}),
        (h.heddle_router, (x, i2.new_zeros(2, 4).T, w2, c), {}),
        (h.heddle_router_backward, (x, i2, w2, c, None), {}), (h.heddle_router_backward, (x, i2, w2, c, y[:2]), {}),
        (h.heddle_router_backward, (x, i2, w2, c, y), {"dweights": i2}),
        (h.heddle_router_backward, (x, i2, w2, c, y), {"dloss": f4}),
    ]
    for f, args, kw in calls:
        with pytest.raises(h.HeddleError) as err:
            f(ctx, *args, **kw)
        assert err.value.status == h.E_ARG, (f.__name__, kw)
    wide = torch.ones(2, 1025, device="cuda")
    for f, args in ((h.heddle_router, (wide, i2[:2], w2[:2], torch.zeros(1026, dtype=torch.int32, device="cuda"))),
                    (h.heddle_router, (wide[:, :64], i2.new_zeros(2, 33), w2.new_zeros(2, 33),
                                       torch.zeros(65, dtype=torch.int32, device="cuda")))):
        with pytest.raises(h.HeddleError) as err:
            f(ctx, *args)
        assert err.value.status == h.E_LIMIT
    for kw in ({"seed": -1}, {"seed": 2 ** 64}, {"seed": 0, "offset": 2 ** 64}):
        with pytest.raises(OverflowError):
            h.heddle_dropout(ctx, x, y, 0.1, **kw)
    torch.cuda.synchronize()
    assert (y == 1).all()
