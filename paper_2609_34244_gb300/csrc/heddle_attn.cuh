// heddle_attn.cuh -- what the attention kernels share: a sequence's span of
// positions, and the launchers of the tensor-core kernels.
#pragma once

#include "heddle_ops.cuh"

namespace hd {

// Queries and keys of a sequence; a query's position is its index plus off.
struct Span {
    int64_t ql, kl, off;
};
__device__ __forceinline__ Span span_of(const heddle_attention_args& a, int64_t b) {
    Span s{a.q_len, a.kv_len, 0};
    if (a.q_lens) s.ql = max((int64_t)0, min((int64_t)a.q_lens[b], a.q_len));
    if (a.kv_lens) s.kl = max((int64_t)0, min((int64_t)a.kv_lens[b], a.kv_len));
    s.off = s.kl - s.ql;
    return s;
}

// Whether the tensor-core kernels take a call; their scratch; their launches.
bool attn_tc_takes(const heddle_attention_args& a);
bool attn_tc_takes_grad(const heddle_attention_grad_args& g);
size_t attn_tc_scratch(const OpContext& x, const heddle_attention_args& a);
cudaError_t launch_attn_tc(const OpContext& x, const heddle_attention_args& a, unsigned char* ws, cudaStream_t st);
// keep: with room for the scores' gradients between the backward's passes
size_t attn_tc_grad_scratch(const OpContext& x, const heddle_attention_args& a, bool keep);
cudaError_t launch_attn_tc_grad(const OpContext& x, const heddle_attention_grad_args& g, const float* delta,
                                unsigned char* ws, bool keep, cudaStream_t st);

}  // namespace hd
