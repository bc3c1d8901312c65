"""The layer that the operators make up: against the same layer in 64 bits,
and as a source of profile entries for the pricing."""

import numpy as np
import pytest


def test_profile_entries_scale_and_add_collectives():
    from paper_2609_34244_gb300 import layer_profile as P
    cluster = {"tflops": np.array([100.0, 50.0]), "intra_bw": np.array([100, 200]), "node_type": np.array([0, 1, 1]),
               "node_gpus": np.array([8, 2, 4]), "node_nic": np.array([7, 20, 10])}
    got = P.profile_entries(cluster, [8.0, 4.0, float("nan"), 1.0], 3, ar_bytes=1000, measured_type=0)
    assert got.shape == (2, 4, 3)
    assert got[0, :, 0].tolist() == [8.0, 4.0 + 4 * 1000 / 100, 4.0 + 4 * 1.5 * 1000 / 100, 1.0 + 4 * 1.75 * 1000 / 100]
    assert got[1, :, 2].tolist() == [16.0, 8.0 + 4 * 1000 / 200, 8.0 + 4 * 1.5 * 1000 / 200,
                                     2.0 + 4 * 1.75 * 1000 / 10]  # eight GPUs leave the node
    with pytest.raises(ValueError):
        P.profile_entries(cluster, [float("nan"), 1, 1, 1], 3, 0)


def test_shards():
    from paper_2609_34244_gb300 import layer_profile as P
    s = P.LayerShape(hidden=512, heads=8, kv_heads=2, ffn=96, seq=16)
    assert [s.shard(k) for k in (1, 2, 4, 8)] == [(8, 2, 96), (4, 1, 48), (2, 1, 24), (1, 1, 12)]
    with pytest.raises(ValueError):
        s.shard(3)
    with pytest.raises(ValueError):
        P.LayerShape(hidden=512, heads=12, kv_heads=3, ffn=96, seq=16).shard(4)


def _reference(layer, x, dz):
    """The layer and its gradients in 64 bits."""
    import torch
    s = layer.shape
    names = ["w_qkv", "w_o", "w_gate", "w_up", "w_down", "wq", "wk"]
    w = {n: getattr(layer, n).double().requires_grad_() for n in names}
    xd = x.double().requires_grad_()
    b, t, d, hq, hk = s.microbatch, s.seq, s.head_dim, layer.hq, layer.hk
    qkv = (xd @ w["w_qkv"].T).view(b, t, -1, d)
    p = layer.rope["positions"][:t].long()
    turn = torch.complex(layer.rope["cos"].double()[p], layer.rope["sin"].double()[p])[None, :, None]

    def norm_rope(v, wt):
        v = v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * wt
        z = torch.complex(v[..., :d // 2], v[..., d // 2:]) * turn
        return torch.cat((z.real, z.imag), -1)

    q, k = norm_rope(qkv[:, :, :hq], w["wq"]), norm_rope(qkv[:, :, hq:hq + hk], w["wk"])
    v = qkv[:, :, hq + hk:]
    k, v = (z.repeat_interleave(hq // hk, 2) for z in (k, v))
    sc = torch.einsum("bihd,bjhd->bhij", q, k) * d ** -0.5
    i, j = torch.arange(t, device="cuda")[:, None], torch.arange(t, device="cuda")[None]
    ok = j <= i
    if s.window:
        ok &= (i - j < s.window) | (j < s.sinks)
    a = torch.einsum("bhij,bjhd->bihd", sc.masked_fill(~ok, -torch.inf).softmax(-1), v).reshape(b * t, -1)
    y = a @ w["w_o"].T + xd
    f = torch.nn.functional.silu(y @ w["w_gate"].T) * (y @ w["w_up"].T)
    z = f @ w["w_down"].T + y
    grads = torch.autograd.grad(z, [xd] + [w[n] for n in names], dz.double())
    return z.detach(), dict(zip(["x"] + names, grads))


@pytest.mark.gpu
@pytest.mark.parametrize("degree", [1, 2])
def test_layer_against_64_bits(heddle_lib, degree):
    """At most 16 values in a row are rounded to float16 (unit roundoff 2^-11)
    on the way from x to any gradient, each off by u of its own norm; what the
    branches add up stays within a factor of two and a half: 2 % in norm."""
    import torch
    from paper_2609_34244_gb300 import layer_profile as P
    shape = P.LayerShape(hidden=256, heads=4, kv_heads=2, ffn=320, seq=150, microbatch=2, head_dim=64, window=70,
                         sinks=3, dtype="float16")
    ctx = heddle_lib.heddle_create(0)
    try:
        layer = P.Layer(ctx, shape, degree)
        g = torch.Generator(device="cuda").manual_seed(5)
        x, dz = (torch.randn(300, 256, generator=g, device="cuda").half() for _ in range(2))
        z = layer.forward(x)
        dx = layer.backward(x, dz)
        want, grads = _reference(layer, x, dz)
        for name, got, ref in [("z", z, want), ("dx", dx, grads["x"])] + \
                [(n, layer.grads[n], grads[n]) for n in layer.grads]:
            off = (got.double() - ref).norm() / ref.norm()
            assert off < 0.02, "%s: %.3g" % (name, off)
        assert heddle_lib.heddle_device_errors(ctx) == 0
    finally:
        heddle_lib.heddle_destroy(ctx)


@pytest.mark.gpu
def test_measured_profile_prices(heddle_lib):
    """The measured entries load as a model's profile: the tables hold them to
    the nanosecond, and candidates are priced."""
    from paper_2609_34244_gb300 import layer_profile as P
    from paper_2609_34244_gb300 import workloads as W
    h = heddle_lib
    w = W.make_workload("dense32", seed=0, n=2000)
    n_layers = len(w.model["flops"])
    shape = P.LayerShape(hidden=512, heads=4, kv_heads=2, ffn=512, seq=256)
    ctx = h.heddle_create(0)
    try:
        prof, seconds = P.measure_profile(ctx, w.cluster, shape, n_layers, reps=3)
        assert np.isfinite(seconds[:3]).all() and np.isnan(seconds[3]) and min(seconds[:3]) > 0  # eight shards of 4 heads
        h.heddle_load_cluster(ctx, w.cluster)
        h.heddle_load_model(ctx, dict(w.model, profile_s=prof))
        q, _ = h.heddle_get_tables(ctx, len(w.cluster["tflops"]), n_layers)
        want = np.floor(prof * 1e9 + 0.5)
        used = np.isin(np.arange(len(w.cluster["tflops"])), w.cluster["node_type"])
        assert np.array_equal(q[used], want[used])
        state = h.new_topk_state(4)
        h.heddle_price_topk_host(ctx, w.cands, None, state, 1 << 20, None)
        assert h.topk_state_to_dict(state)["count"] == 4
        assert h.heddle_device_errors(ctx) == 0
    finally:
        h.heddle_destroy(ctx)
