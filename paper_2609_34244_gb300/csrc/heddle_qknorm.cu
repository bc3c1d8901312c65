// heddle_qknorm.cu -- norms of queries and keys per head with the position
// rotation in the same pass, and their gradients.

#include "heddle_ops.cuh"

namespace hd {
namespace {

constexpr int kWarps = 8;
constexpr int kMaxDim = 256;

struct Row {
    const void* x;
    void* y;
    const void* w;
    int64_t token;
    bool is_q;
};

__device__ __forceinline__ int partner(int i, int rot, bool inter) {
    return inter ? i ^ 1 : i < rot / 2 ? i + rot / 2 : i - rot / 2;
}

// One warp per head and token.
template <class T, bool GRAD>
__global__ void __launch_bounds__(kWarps * 32) qk_norm_rope_kernel(heddle_qk_norm_rope_grad_args ga, float* partial,
                                                                  uint32_t* err) {
    const heddle_qk_norm_rope_args& a = ga.fwd;
    __shared__ float row[kWarps][kMaxDim];
    __shared__ float grad[kWarps][kMaxDim];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int D = a.head_dim, rot = a.rot_dim, half = rot / 2;
    const int heads = a.q_heads + a.k_heads;
    const int64_t rows = a.tokens * heads;
    float dw[2][kMaxDim / 32] = {};
    for (int64_t r = (int64_t)blockIdx.x * kWarps + warp; r < rows; r += (int64_t)gridDim.x * kWarps) {
        const int64_t t = r / heads;
        const int h = (int)(r - t * heads);
        const bool is_q = h < a.q_heads;
        const int hh = is_q ? h : h - a.q_heads;
        const heddle_heads& in = is_q ? a.q : a.k;
        const heddle_heads& out = is_q ? a.q_out : a.k_out;
        const T* x = static_cast<const T*>(in.data) + t * in.token_stride + hh * in.head_stride;
        T* y = static_cast<T*>(out.data) + t * out.token_stride + hh * out.head_stride;
        const T* w = static_cast<const T*>(is_q ? a.wq : a.wk);
        const float *cs = nullptr, *sn = nullptr;
        bool bad = false;
        if (rot) {
            const int64_t p = a.positions[t];
            bad = p < 0 || p >= a.table_len;
            cs = a.cos + (bad ? 0 : p) * half;
            sn = a.sin + (bad ? 0 : p) * half;
        }
        if (bad && lane == 0) atomicOr(err, kErrOpPosition);
        float v[kMaxDim / 32], ss = 0.0f;
#pragma unroll
        for (int j = 0; j < kMaxDim / 32; ++j) {
            const int i = lane + 32 * j;
            v[j] = i < D ? to_float(x[i]) : 0.0f;
            ss += v[j] * v[j];
        }
        ss = warp_sum(ss);
        const float rstd = 1.0f / sqrtf(ss / D + a.eps);
        if (!GRAD) {
#pragma unroll
            for (int j = 0; j < kMaxDim / 32; ++j) {
                const int i = lane + 32 * j;
                if (i < D) row[warp][i] = v[j] * rstd * to_float(w[i]);
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kMaxDim / 32; ++j) {
                const int i = lane + 32 * j;
                if (i >= D) break;
                float o = row[warp][i];
                if (i < rot && !bad) {
                    const int pi = a.interleaved ? i / 2 : i % half;
                    const bool second = a.interleaved ? i & 1 : i >= half;
                    const float other = row[warp][partner(i, rot, a.interleaved)];
                    o = second ? o * cs[pi] + other * sn[pi] : o * cs[pi] - other * sn[pi];
                }
                y[i] = from_float<T>(bad ? 0.0f : o);
            }
            __syncwarp();
        } else {
            const heddle_heads& dst = is_q ? ga.dq : ga.dk;
            T* dx = static_cast<T*>(dst.data) + t * dst.token_stride + hh * dst.head_stride;
#pragma unroll
            for (int j = 0; j < kMaxDim / 32; ++j) {
                const int i = lane + 32 * j;
                if (i < D) grad[warp][i] = bad ? 0.0f : to_float(y[i]);
            }
            __syncwarp();
            float tv[kMaxDim / 32], dot = 0.0f;
#pragma unroll
            for (int j = 0; j < kMaxDim / 32; ++j) {
                const int i = lane + 32 * j;
                tv[j] = 0.0f;
                if (i >= D) continue;
                float d = grad[warp][i];
                if (i < rot && !bad) {
                    const int pi = a.interleaved ? i / 2 : i % half;
                    const bool second = a.interleaved ? i & 1 : i >= half;
                    const float other = grad[warp][partner(i, rot, a.interleaved)];
                    d = second ? d * cs[pi] - other * sn[pi] : d * cs[pi] + other * sn[pi];
                }
                const float xh = v[j] * rstd;
                dw[is_q ? 0 : 1][j] += bad ? 0.0f : d * xh;
                tv[j] = d * to_float(w[i]);
                dot += tv[j] * xh;
            }
            dot = warp_sum(dot) / D;
#pragma unroll
            for (int j = 0; j < kMaxDim / 32; ++j) {
                const int i = lane + 32 * j;
                if (i < D) dx[i] = from_float<T>(bad ? 0.0f : rstd * (tv[j] - v[j] * rstd * dot));
            }
            __syncwarp();
        }
    }
    if (GRAD) {
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kMaxDim / 32; ++j) row[warp][lane + 32 * j] = dw[s][j];
            __syncthreads();
            for (int i = threadIdx.x; i < D; i += kWarps * 32) {
                float v = 0.0f;
                for (int k = 0; k < kWarps; ++k) v += row[k][i];
                partial[((int64_t)s * gridDim.x + blockIdx.x) * D + i] = v;
            }
        }
    }
}

// Sums the blocks' partial weight gradients, one block per 32 columns of dwq or dwk.
__global__ void __launch_bounds__(256) weight_grad_kernel(const float* partial, int blocks, int D, float* dwq,
                                                          float* dwk) {
    __shared__ float s[8][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int i = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (i < D)
        for (int b = warp; b < blocks; b += 8) v += partial[((int64_t)blockIdx.y * blocks + b) * D + i];
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < D) {
        for (int k = 1; k < 8; ++k) v += s[k][lane];
        (blockIdx.y ? dwk : dwq)[i] = v;
    }
}

int norm_blocks(const OpContext& x, const heddle_qk_norm_rope_args& a) {
    const int64_t rows = a.tokens * ((int64_t)a.q_heads + a.k_heads);
    const int64_t want = ceil_div(rows, kWarps), most = (int64_t)x.num_sms * 8;
    return (int)(want < 1 ? 1 : want < most ? want : most);
}

template <bool GRAD>
void launch_rows(const OpContext& x, const heddle_qk_norm_rope_grad_args& a, float* partial, cudaStream_t st) {
    const int blocks = norm_blocks(x, a.fwd);
    if (a.fwd.dtype == HEDDLE_BF16)
        qk_norm_rope_kernel<__nv_bfloat16, GRAD><<<blocks, kWarps * 32, 0, st>>>(a, partial, x.err);
    else if (a.fwd.dtype == HEDDLE_FP16)
        qk_norm_rope_kernel<__half, GRAD><<<blocks, kWarps * 32, 0, st>>>(a, partial, x.err);
    else
        qk_norm_rope_kernel<float, GRAD><<<blocks, kWarps * 32, 0, st>>>(a, partial, x.err);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const OpContext& x, const heddle_qk_norm_rope_args& a, cudaStream_t st) {
    heddle_qk_norm_rope_grad_args ga{};
    ga.fwd = a;
    launch_rows<false>(x, ga, nullptr, st);
    return cudaGetLastError();
}

size_t qk_norm_rope_grad_scratch(const OpContext& x, const heddle_qk_norm_rope_grad_args& a) {
    return align256(sizeof(float) * 2 * (size_t)norm_blocks(x, a.fwd) * a.fwd.head_dim);
}

cudaError_t launch_qk_norm_rope_grad(const OpContext& x, const heddle_qk_norm_rope_grad_args& a, unsigned char* ws,
                                     cudaStream_t st) {
    float* partial = reinterpret_cast<float*>(ws);
    launch_rows<true>(x, a, partial, st);
    const int D = a.fwd.head_dim;
    weight_grad_kernel<<<dim3((unsigned)ceil_div(D, 32), 2), 256, 0, st>>>(partial, norm_blocks(x, a.fwd), D, a.dwq,
                                                                           a.dwk);
    return cudaGetLastError();
}

}  // namespace hd
