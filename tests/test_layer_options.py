"""The layer with norms of the hidden state and dropout, against the same layer
in 64 bits; without them it is the layer that it was."""

import pytest

torch = pytest.importorskip("torch")

import hidden_reference as H  # noqa: E402

pytestmark = pytest.mark.gpu


def _reference(layer, x, dz, p, step):
    s = layer.shape
    names = [n for n in ("w_qkv", "w_o", "w_gate", "w_up", "w_down", "wq", "wk", "norm1", "norm_bias1", "norm2",
                         "norm_bias2") if n in layer.grads]
    w = {n: getattr(layer, n).double().requires_grad_() for n in names}
    xd = x.double().requires_grad_()
    b, t, d, hq, hk, n, hid = s.microbatch, s.seq, s.head_dim, layer.hq, layer.hk, x.shape[0], s.hidden
    at = layer.rope["positions"][:t].long()
    turn = torch.complex(layer.rope["cos"].double()[at], layer.rope["sin"].double()[at])[None, :, None]

    def norm(v, i):
        if not s.norms:
            return v
        return torch.nn.functional.layer_norm(v, (hid,), w["norm" + i], w["norm_bias" + i], 1e-5)

    def drop(v, mask):
        if not p:
            return v
        least = round(p * 2 ** 32)
        keep = H.numbers(0, n * hid, layer.seed, (mask << 32) + step, "cuda").view(n, hid) >= least
        return v * keep * (2 ** 32 / (2 ** 32 - least))

    def norm_rope(v, wt):
        v = v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * wt
        z = torch.complex(v[..., :d // 2], v[..., d // 2:]) * turn
        return torch.cat((z.real, z.imag), -1)

    qkv = (norm(xd, "1") @ w["w_qkv"].T).view(b, t, -1, d)
    q, k = norm_rope(qkv[:, :, :hq], w["wq"]), norm_rope(qkv[:, :, hq:hq + hk], w["wk"])
    k, v = (z.repeat_interleave(hq // hk, 2) for z in (k, qkv[:, :, hq + hk:]))
    sc = torch.einsum("bihd,bjhd->bhij", q, k) * d ** -0.5
    i, j = torch.arange(t, device="cuda")[:, None], torch.arange(t, device="cuda")[None]
    a = torch.einsum("bhij,bjhd->bihd", sc.masked_fill(j > i, -torch.inf).softmax(-1), v).reshape(n, -1)
    y = xd + drop(a @ w["w_o"].T, 0)
    m = norm(y, "2")
    z = y + drop((torch.nn.functional.silu(m @ w["w_gate"].T) * (m @ w["w_up"].T)) @ w["w_down"].T, 1)
    grads = torch.autograd.grad(z, [xd] + [w[m] for m in names], dz.double())
    return z.detach(), dict(zip(["x"] + names, grads))


@pytest.mark.parametrize("norms,p", [(True, 0.0), (False, 0.25), (True, 0.1)])
def test_layer_with_options_against_64_bits(heddle_lib, norms, p):
    """At most 20 values in a row are rounded to float16 (unit roundoff 2^-11,
    half a step) on the way from x to any gradient, each off by u of its own
    norm at most; what the branches add up stays within a factor of two: 2 % in
    norm."""
    from paper_2609_34244_gb300 import layer_profile as P
    shape = P.LayerShape(hidden=264, heads=4, kv_heads=2, ffn=320, seq=100, microbatch=2, head_dim=64,
                         dtype="float16", norms=norms, dropout=p)
    ctx = heddle_lib.heddle_create(0)
    try:
        layer = P.Layer(ctx, shape, seed=3)
        g = torch.Generator(device="cuda").manual_seed(5)
        if norms:
            for n in ("norm1", "norm_bias1", "norm2", "norm_bias2"):
                getattr(layer, n).add_(torch.randn(264, generator=g, device="cuda").half() * 0.2)
        x, dz = (torch.randn(200, 264, generator=g, device="cuda").half() for _ in range(2))
        for step in range(2 if p else 1):
            z = layer.forward(x)
            dx = layer.backward(x, dz)
            want, grads = _reference(layer, x, dz, p, step)
            for name, got, ref in [("z", z, want), ("dx", dx, grads["x"])] + \
                    [(n, layer.grads[n], grads[n]) for n in layer.grads]:
                off = (got.double() - ref).norm() / ref.norm()
                assert off < 0.02, "%s: %.3g" % (name, off)
            if p:
                layer.step.add_(1)
        assert heddle_lib.heddle_device_errors(ctx) == 0
    finally:
        heddle_lib.heddle_destroy(ctx)


def test_options_are_measured(heddle_lib):
    from paper_2609_34244_gb300 import layer_profile as P
    ctx = heddle_lib.heddle_create(0)
    try:
        shape = P.LayerShape(hidden=512, heads=4, kv_heads=2, ffn=512, seq=256, norms=True, dropout=0.1)
        assert P.measure_layer(ctx, shape, 2, reps=3) > 0
    finally:
        heddle_lib.heddle_destroy(ctx)
