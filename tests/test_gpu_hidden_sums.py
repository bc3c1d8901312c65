"""Long sums of layer norm's gradients, the embedding's gradient and the
router's loss over whole numbers, which 32 bits hold exactly in any order: a
term that is lost, taken twice or added to another's place shows, whatever the
number of terms.  (A bound on a sum's rounding grows with its terms and passes
the sum itself where they are many.)"""

import pytest

torch = pytest.importorskip("torch")

import hidden_reference as H  # noqa: E402
from test_gpu_hidden import LAYOUTS, floats, laid, lib, token_list  # noqa: E402, F401
from test_gpu_operators import TYPES, frame_kept, framed, gen  # noqa: E402

pytestmark = pytest.mark.gpu


def whole(g, *shape, most=3, dt=torch.float32):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dt)


# Rows by lanes of every number, by one and two rows between a block's
# barriers, by blocks of up to 1024 threads, through memory; rows of no whole
# units; few rows and many.
ROWS = [(90000, 9), (60000, 64), (40000, 130), (20000, 257), (30000, 500), (20000, 520), (9000, 1031), (20000, 1032),
        (3000, 4096), (2000, 5121), (3000, 8192), (1200, 8190), (700, 9000), (500, 16380), (300, 20000), (31, 70001),
        (1, 264), (5, 4096)]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n", ROWS)
def test_layer_norm_sums_over_rows_are_exact(lib, m, n, dt):
    """dy, x and mean are whole numbers and rstd a power of two: every term of dw
    is a multiple of a half, and at most 3 * 4 * 2: sums of 90000 stay below
    2^23 halves."""
    h, ctx = lib
    dt = TYPES[dt]
    for i, (pad, skip) in enumerate(LAYOUTS):
        g = gen(m + n + i)
        dy, x = laid(whole(g, m, n, dt=dt), pad, skip), laid(whole(g, m, n, dt=dt), pad, skip)
        mean, rstd = whole(g, m, most=1), 2.0 ** whole(g, m, most=1)
        dw, db, dx = floats(n), floats(n), torch.empty_like(x)
        h.heddle_layer_norm_backward(ctx, dy, x, None, mean, rstd, dx=dx, dw=dw, dbias=db)
        v = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        assert torch.equal(dw.double(), (dy.double() * v).sum(0))
        assert torch.equal(db.double(), dy.double().sum(0))
        other = [floats(n), floats(n)]
        h.heddle_layer_norm_backward(ctx, dy, x, None, mean, rstd, dw=other[0], dbias=other[1])
        assert torch.equal(other[0], dw) and torch.equal(other[1], db)


EMBEDDINGS = [  # tokens, vocabulary, shards, columns
    (600000, 50, 1, 8), (70001, 33, 1, 130), (40000, 300000, 1, 24), (33000, 4096, 1, 40), (9000, 900, 1, 1040),
    (30000, 4000, 4, 513), (2100, 70, 1, 1023), (513, 30000, 1, 40), (512, 7, 1, 4), (5, 40, 4, 7), (1, 1, 1, 1),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,vocab,shards,n", EMBEDDINGS)
def test_embedding_gradient_is_exact(lib, t, vocab, shards, n, dt):
    """Sums of at most 600000 numbers of at most 3 stay below 2^21; a scale that
    is a power of two rounds nothing, and a 16-bit result once."""
    h, ctx = lib
    dt = TYPES[dt]
    rows = vocab // shards
    for i, (kind, (pad, skip)) in enumerate(zip(("zipf", "one", "each"), LAYOUTS)):
        g = gen(t + vocab + i)
        tokens = token_list(g, t, vocab, kind)
        if t > 4:
            tokens[::7] = -1
        first = rows * (shards // 2)
        dy = laid(whole(g, t, n, dt=dt), pad, skip)
        at = H.embedding_rows(tokens, first, rows)
        want = torch.zeros(rows + 1, n, dtype=torch.float64, device="cuda").index_add_(0, at, dy.double())[:rows] * 0.5
        for to in {dt, torch.float32}:
            for base in (None, whole(g, rows, n, dt=to)):
                d, buf = framed(rows, n, to, pad, skip)
                if base is not None:
                    d.copy_(base)
                h.heddle_embedding_backward(ctx, tokens, dy, d, scale=0.5, first=first, vocab=vocab,
                                            accumulate=base is not None)
                assert torch.equal(d, (want if base is None else want + base.double()).to(to))
                frame_kept(d, buf, "dtable")


@pytest.mark.parametrize("n,dt", [(4, "fp32"), (3, "bf16")])
def test_embedding_gradient_of_many_rows_is_exact(lib, n, dt):
    h, ctx = lib
    t, rows, dt = 70000, 20_000_003, TYPES[dt]
    g = gen(t + n)
    tokens = torch.randint(0, rows, (t,), generator=g, device="cuda")
    tokens[torch.rand(t, generator=g, device="cuda") < 0.5] = 8200
    dy, d = whole(g, t, n, dt=dt), torch.full((rows, n), 3.0, device="cuda")
    h.heddle_embedding_backward(ctx, tokens, dy, d)
    want = torch.zeros(rows, n, device="cuda", dtype=torch.float64).index_add_(0, tokens, dy.double())
    assert torch.equal(d.double(), want)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,n", [(1, 2), (16, 64), (64, 64), (129, 7), (20001, 16), (16384, 64), (5000, 128),
                                 (32771, 250), (3000, 512), (700, 1000)])
def test_router_loss_of_certain_choices_is_exact(lib, t, n, dt):
    """One logit of each token is so far above the others (100 or more) that its
    probability is 1 and theirs vanish beside it (below e^-100): an expert's
    probabilities add up to its choices, whole numbers.  The loss is
    n sum c^2 / t^2, off by the rounding of n sums and of a few products."""
    h, ctx = lib
    for i, (pad, skip) in enumerate(LAYOUTS):
        g = gen(t + n + i)
        one = torch.randint(0, n, (t,), generator=g, device="cuda")
        logits = laid(whole(g, t, n).scatter_(1, one[:, None], 104.0).to(TYPES[dt]), pad, skip)
        valid = torch.rand(t, generator=g, device="cuda") < 0.8 if i else None
        experts, weights = torch.empty(t, 1, dtype=torch.int32, device="cuda"), torch.empty(t, 1, device="cuda")
        counts, loss = torch.empty(n + 1, dtype=torch.int32, device="cuda"), floats(1)
        h.heddle_router(ctx, logits, experts, weights, counts, loss=loss, valid=valid)
        took = torch.ones(t, dtype=torch.bool, device="cuda") if valid is None else valid
        c = torch.bincount(one[took], minlength=n)
        assert torch.equal(counts[:n].long(), c) and counts[n] == took.sum()
        want = float(n * c.double().square().sum() / max(int(took.sum()), 1) ** 2)
        assert abs(loss.item() - want) <= (n + 8) * H.e * want
