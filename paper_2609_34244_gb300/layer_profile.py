"""Measures a transformer layer on this GPU and turns it into the profile
entries that pricing takes (§5.2: seconds of one layer at each degree).

A layer is built from the library's operators at the shapes of one
tensor-parallel shard -- query heads, key heads and feed-forward columns over
the degree -- and its forward and backward passes are timed together:

  q, k, v = x w_qkv^T               heddle_linear
  q, k normed per head and rotated  heddle_qk_norm_rope
  a = attention(q, k, v)            heddle_attention
  y = a w_o^T + x                   heddle_linear, the residual in its epilogue
  f = act(y w_gate^T) (y w_up^T)    heddle_gated_ffn
  z = f w_down^T + y                heddle_linear

The norms of the hidden state that models have ahead of attention and of the
feed-forward block are not part of it, nor are experts: the entries are those
of the products, attention and norms per head of a dense layer, and too small
by two passes over the hidden state in either direction.  The backward pass
adds the two residual gradients with torch.

``python -m paper_2609_34244_gb300.layer_profile`` measures a layer, loads the
profile beside a cluster of this GPU and slower types, and prices candidates.
"""

from __future__ import annotations

import argparse
import dataclasses

import numpy as np

from . import heddle as h

DEGREES = (1, 2, 4, 8)


@dataclasses.dataclass(frozen=True)
class LayerShape:
    """A dense transformer layer and the micro-batch it runs on."""

    hidden: int
    heads: int
    kv_heads: int
    ffn: int
    seq: int
    microbatch: int = 1
    head_dim: int = 128
    window: int = 0
    sinks: int = 0
    act: str = "silu"
    dtype: str = "bfloat16"

    def shard(self, degree: int) -> tuple:
        """(query heads, key heads, feed-forward columns) of one of `degree`
        shards; key heads fewer than the degree are held by several."""
        if degree < 1 or self.heads % degree or self.ffn % degree:
            raise ValueError("%d heads and %d feed-forward columns do not divide into %d shards"
                             % (self.heads, self.ffn, degree))
        kv = self.kv_heads // degree if self.kv_heads % degree == 0 else 1
        if self.kv_heads % degree and degree % self.kv_heads:
            raise ValueError("%d key heads do not divide into %d shards" % (self.kv_heads, degree))
        return self.heads // degree, kv, self.ffn // degree


class Layer:
    """One shard of a layer: its weights, and the buffers that a training
    step of it keeps between forward and backward."""

    def __init__(self, ctx, shape: LayerShape, degree: int = 1, seed: int = 0, device="cuda"):
        import torch
        self.ctx, self.shape = ctx, shape
        self.hq, self.hk, self.ffn = shape.shard(degree)
        self.act = h.ACTIVATIONS[shape.act]
        self.dtype = getattr(torch, shape.dtype)
        d, hid, b, t = shape.head_dim, shape.hidden, shape.microbatch, shape.seq
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(*size):
            w = torch.randn(*size, generator=gen, device=device, dtype=torch.float32)
            return (w * size[-1] ** -0.5).to(self.dtype)

        self.w_qkv = weight((self.hq + 2 * self.hk) * d, hid)
        self.w_o = weight(hid, self.hq * d)
        self.w_gate, self.w_up = weight(self.ffn, hid), weight(self.ffn, hid)
        self.w_down = weight(hid, self.ffn)
        self.wq = torch.ones(d, dtype=self.dtype, device=device)
        self.wk = torch.ones(d, dtype=self.dtype, device=device)
        angle = torch.arange(t, device=device, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(d // 2, device=device, dtype=torch.float64) / (d // 2))
        self.rope = dict(positions=torch.arange(t, dtype=torch.int32, device=device).repeat(b),
                         cos=angle.cos().float(), sin=angle.sin().float())
        n = b * t

        def buf(*size, dtype=self.dtype):
            return torch.empty(*size, dtype=dtype, device=device)

        self.qkv = buf(n, self.hq + 2 * self.hk, d)
        self.q, self.k = buf(n, self.hq, d), buf(n, self.hk, d)
        self.a, self.lse = buf(n, self.hq, d), buf(b, self.hq, t, dtype=torch.float32)
        self.y, self.f, self.z = buf(n, hid), buf(n, self.ffn), buf(n, hid)
        self.gate, self.up = buf(n, self.ffn, dtype=torch.float32), buf(n, self.ffn, dtype=torch.float32)
        self.grads = {name: torch.empty_like(getattr(self, name))
                      for name in ("w_qkv", "w_o", "w_gate", "w_up", "w_down")}
        self.grads.update(wq=buf(d, dtype=torch.float32), wk=buf(d, dtype=torch.float32))
        self.d_f, self.d_y, self.d_a = buf(n, self.ffn), buf(n, hid), buf(n, self.hq, d)
        self.d_q, self.d_k = buf(n, self.hq, d), buf(n, self.hk, d)
        self.d_qkv, self.d_x = buf(n, self.hq + 2 * self.hk, d), buf(n, hid)

    def _sequences(self, t):
        return t.view(self.shape.microbatch, self.shape.seq, *t.shape[1:])

    def _attention(self):
        v = self.qkv[:, self.hq + self.hk:]
        return [self._sequences(t) for t in (self.q, self.k, v, self.a)]

    def forward(self, x):
        """z of x ([microbatch * seq][hidden]); the buffers keep what backward reads."""
        hq, hk, n = self.hq, self.hk, x.shape[0]
        h.heddle_linear(self.ctx, x, self.w_qkv, self.qkv.view(n, -1))
        h.heddle_qk_norm_rope(self.ctx, self.qkv[:, :hq], self.qkv[:, hq:hq + hk], self.wq, self.wk, self.q, self.k,
                              **self.rope)
        h.heddle_attention(self.ctx, *self._attention(), self.lse, window=self.shape.window, sinks=self.shape.sinks)
        h.heddle_linear(self.ctx, self.a.view(n, -1), self.w_o, self.y, residual=x)
        h.heddle_gated_ffn(self.ctx, self.y, self.w_gate, self.w_up, self.f, act=self.act, gate=self.gate, up=self.up)
        h.heddle_linear(self.ctx, self.f, self.w_down, self.z, residual=self.y)
        return self.z

    def backward(self, x, dz):
        """The gradient of x from that of z; the weights' are in ``grads``."""
        hq, hk, n, g = self.hq, self.hk, x.shape[0], self.grads
        h.heddle_linear_backward(self.ctx, dz, self.f, self.w_down, dx=self.d_f, dw=g["w_down"])
        h.heddle_gated_ffn_backward(self.ctx, self.d_f, self.y, self.w_gate, self.w_up, self.gate, self.up,
                                    act=self.act, dx=self.d_y, dwg=g["w_gate"], dwu=g["w_up"])
        self.d_y.add_(dz)
        h.heddle_linear_backward(self.ctx, self.d_y, self.a.view(n, -1), self.w_o, dx=self.d_a.view(n, -1),
                                 dw=g["w_o"])
        h.heddle_attention_backward(self.ctx, self._sequences(self.d_a), *self._attention(), self.lse,
                                    self._sequences(self.d_q), self._sequences(self.d_k),
                                    self._sequences(self.d_qkv[:, hq + hk:]), window=self.shape.window,
                                    sinks=self.shape.sinks)
        h.heddle_qk_norm_rope_backward(self.ctx, self.d_q, self.d_k, self.qkv[:, :hq], self.qkv[:, hq:hq + hk],
                                       self.wq, self.wk, self.d_qkv[:, :hq], self.d_qkv[:, hq:hq + hk], g["wq"],
                                       g["wk"], **self.rope)
        h.heddle_linear_backward(self.ctx, self.d_qkv.view(n, -1), x, self.w_qkv, dx=self.d_x, dw=g["w_qkv"])
        return self.d_x.add_(self.d_y)


def measure_layer(ctx, shape: LayerShape, degree: int = 1, reps: int = 5, warmup: int = 3) -> float:
    """Seconds of one forward and backward pass of a shard (the median of
    `reps`, CUDA events), its collectives not included."""
    import torch
    layer = Layer(ctx, shape, degree)
    x = torch.randn(shape.microbatch * shape.seq, shape.hidden, device="cuda").to(layer.dtype)
    dz = torch.randn_like(x)
    times = []
    for i in range(warmup + reps):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        layer.forward(x)
        layer.backward(x, dz)
        end.record()
        end.synchronize()
        if i >= warmup:
            times.append(start.elapsed_time(end) * 1e-3)
    return float(np.median(times))


def profile_entries(cluster: dict, seconds, n_layers: int, ar_bytes: int, measured_type: int = 0):
    """``profile_s`` ([n_types][4][n_layers]) from one layer's seconds at each
    of the four degrees (NaN where a degree was not measured: its entries are
    those of the next smaller degree that was).

    The types other than the measured one are taken to run the layer slower
    or faster by the ratio of their peaks.  A degree k > 1 adds the layer's
    four ring all-reduces of ar_bytes, each moving 2 (k - 1) / k of them, over
    the links between the GPUs of a node where the largest node of the type
    holds the group, else over its slowest NIC."""
    tflops = np.asarray(cluster["tflops"], dtype=np.float64)
    base = np.asarray(seconds, dtype=np.float64)
    if base.shape != (4,) or not np.isfinite(base[0]):
        raise ValueError("seconds: four degrees, the first measured")
    base = base.copy()
    for j in range(1, 4):
        if not np.isfinite(base[j]):
            base[j] = base[j - 1]
    out = np.empty((len(tflops), 4, n_layers))
    for g in range(len(tflops)):
        here = np.asarray(cluster["node_type"]) == g
        for j, k in enumerate(DEGREES):
            s = base[j] * tflops[measured_type] / tflops[g]
            if k > 1 and here.any():
                fits = k <= np.asarray(cluster["node_gpus"])[here].max()
                bw = cluster["intra_bw"][g] if fits else np.asarray(cluster["node_nic"])[here].min()
                s += 4 * (2 * (k - 1) / k) * ar_bytes / float(bw)
            out[g, j] = s
    return out


def measure_profile(ctx, cluster: dict, shape: LayerShape, n_layers: int, measured_type: int = 0, reps: int = 5):
    """Measures the layer at every degree its heads and columns divide into,
    and returns (profile_s, seconds of the four degrees)."""
    seconds = []
    for k in DEGREES:
        try:
            shape.shard(k)
        except ValueError:
            seconds.append(float("nan"))
            continue
        seconds.append(measure_layer(ctx, shape, k, reps=reps))
    ar_bytes = shape.microbatch * shape.seq * shape.hidden * 2
    return profile_entries(cluster, seconds, n_layers, ar_bytes, measured_type), seconds


def main(argv=None):
    from . import workloads as W
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--ffn", type=int, default=14336)
    ap.add_argument("--seq", type=int, default=2048)
    ap.add_argument("--microbatch", type=int, default=1)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--candidates", type=int, default=100_000)
    a = ap.parse_args(argv)
    shape = LayerShape(a.hidden, a.heads, a.kv_heads, a.ffn, a.seq, a.microbatch, window=a.window, sinks=a.sinks)
    w = W.make_workload("dense32", seed=0, n=a.candidates)
    n_layers = len(w.model["flops"])
    ctx = h.heddle_create(0)
    try:
        fastest = int(np.argmax(w.cluster["tflops"]))  # stands for this GPU
        prof, seconds = measure_profile(ctx, w.cluster, shape, n_layers, fastest)
        for k, s in zip(DEGREES, seconds):
            print("degree %d: %s" % (k, "not divisible" if s != s else "%.3f ms a layer" % (s * 1e3)))
        h.heddle_load_cluster(ctx, w.cluster)
        h.heddle_load_model(ctx, dict(w.model, profile_s=prof))
        state = h.new_topk_state(4)
        h.heddle_price_topk_host(ctx, w.cands, None, state, 1 << 20, None)
        best = h.topk_state_to_dict(state)
        for i, t in zip(best["idx"], best["T"]):
            print("candidate %d: %.3f ms an iteration" % (i, t * 1e-6))
    finally:
        h.heddle_destroy(ctx)


if __name__ == "__main__":
    main()
