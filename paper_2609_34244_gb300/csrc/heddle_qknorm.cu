// heddle_qknorm.cu -- norms of queries and keys per head with the position
// rotation in the same pass, and their gradients.
//
// Bound by memory: a head is read and written once, everything between stays
// in registers.  Where heads are whole 16-byte units, a group of lanes holds
// a head, 16 bytes a lane, and walks over several heads of one token, whose
// cosines and sines it keeps; what lies at other addresses is read and written
// value by value, with the same results.  A head of any other size takes the
// kernel of one warp a head, its values dealt out one by one.

#include "heddle_ops.cuh"

namespace hd {
namespace {

constexpr int kWarps = 8;
constexpr int kMaxDim = 256;

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
                const float add = bad ? 0.0f : d * xh;
                dw[0][j] += is_q ? add : 0.0f;
                dw[1][j] += is_q ? 0.0f : add;
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
#pragma unroll
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

// V values of 16 bytes, at once or one by one.
template <class T>
__device__ __forceinline__ uint4 load_unit(const T* p, bool whole) {
    if (whole) return *reinterpret_cast<const uint4*>(p);
    uint4 u;
    T* t = reinterpret_cast<T*>(&u);
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) t[i] = p[i];
    return u;
}
template <class T>
__device__ __forceinline__ void store_unit(T* p, const uint4& u, bool whole) {
    if (whole) {
        *reinterpret_cast<uint4*>(p) = u;
        return;
    }
    const T* t = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) p[i] = t[i];
}

// A head of whole 16-byte units in a group of GL lanes, V values a lane, the
// last lanes idle where head_dim / V is not GL.  A group takes `chunk`
// heads of one token at a time.
template <class T, int GL, bool GRAD>
__global__ void __launch_bounds__(256) qk_norm_rope_wide_kernel(const __grid_constant__ heddle_qk_norm_rope_grad_args ga,
                                                                float* partial, uint32_t* err, int chunk, bool whole) {
    constexpr int V = 16 / sizeof(T), kGroups = 256 / GL, kDepth = GRAD ? 2 : 4;
    const heddle_qk_norm_rope_args& a = ga.fwd;
    const int lane = threadIdx.x % GL, group = threadIdx.x / GL;
    const int D = a.head_dim, rot = a.rot_dim, half = rot / 2, i0 = lane * V;
    const int heads = a.q_heads + a.k_heads, chunks = (heads + chunk - 1) / chunk;
    const int64_t units = a.tokens * chunks;
    const bool live = i0 < D, turns = i0 < rot;
    // the group's lanes, as a mask and where the pair's other half is
    const uint32_t mask = GL == 32 ? ~0u : ((1u << GL) - 1) << (threadIdx.x % 32 / GL * GL);
    const bool second = !a.interleaved && i0 >= half;
    const int other = a.interleaved ? lane : turns ? (second ? lane - half / V : lane + half / V) : lane;
    const float inv_d = 1.0f / D;
    float wq[V], wk[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        wq[v] = live && a.q_heads ? to_float(static_cast<const T*>(a.wq)[i0 + v]) : 0.0f;
        wk[v] = live && a.k_heads ? to_float(static_cast<const T*>(a.wk)[i0 + v]) : 0.0f;
    }
    float dwq[V] = {}, dwk[V] = {};

    // (p, q) -> turned by the lane's angles; back: by their negatives
    auto turn = [&](float (&v)[V], const float (&cs)[V], const float (&sn)[V], float sign) {
        if (a.interleaved) {
            if (turns)
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float p = v[i], q = v[i + 1], s = sign * sn[i / 2];
                    v[i] = p * cs[i / 2] - q * s;
                    v[i + 1] = q * cs[i / 2] + p * s;
                }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float o = __shfl_sync(mask, v[i], other, GL);
                const float s = second ? sign * sn[i] : -sign * sn[i];
                if (turns) v[i] = v[i] * cs[i] + o * s;
            }
        }
    };

    for (int64_t u = (int64_t)blockIdx.x * kGroups + group; u < units; u += (int64_t)gridDim.x * kGroups) {
        const int64_t t = u / chunks;
        const int h0 = (int)(u - t * chunks) * chunk, h1 = min(heads, h0 + chunk);
        bool bad = false;
        float cs[V], sn[V];
        if (rot) {
            const int64_t p = a.positions[t];
            bad = p < 0 || p >= a.table_len;
            if (bad && lane == 0) atomicOr(err, kErrOpPosition);
            if (turns) {
                if (!bad) {
                    const int64_t at = p * half + (a.interleaved ? i0 / 2 : second ? i0 - half : i0);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (v < (a.interleaved ? V / 2 : V)) cs[v] = a.cos[at + v], sn[v] = a.sin[at + v];
                }
            }
        }
        if (bad) {
#pragma unroll
            for (int v = 0; v < V; ++v) cs[v] = sn[v] = 0.0f;
        }
        for (int h = h0; h < h1; h += kDepth) {
            uint4 x[kDepth], g[kDepth];
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const int hh = min(h + k, h1 - 1);
                const bool is_q = hh < a.q_heads;
                const int at = is_q ? hh : hh - a.q_heads;
                const heddle_heads& in = is_q ? a.q : a.k;
                const heddle_heads& out = is_q ? a.q_out : a.k_out;
                x[k] = g[k] = make_uint4(0, 0, 0, 0);
                if (live) {
                    x[k] = load_unit(static_cast<const T*>(in.data) + t * in.token_stride + at * in.head_stride + i0,
                                     whole);
                    if (GRAD)
                        g[k] = load_unit(
                            static_cast<const T*>(out.data) + t * out.token_stride + at * out.head_stride + i0, whole);
                }
            }
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const int hh = h + k;
                if (hh >= h1) break;
                const bool is_q = hh < a.q_heads;
                const int at = is_q ? hh : hh - a.q_heads;
                const heddle_heads& dst = GRAD ? (is_q ? ga.dq : ga.dk) : (is_q ? a.q_out : a.k_out);
                const T* xt = reinterpret_cast<const T*>(&x[k]);
                float v[V], ss = 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[i] = to_float(xt[i]);
                    ss += v[i] * v[i];
                }
#pragma unroll
                for (int o = GL / 2; o; o >>= 1) ss += __shfl_xor_sync(mask, ss, o, GL);
                const float rstd = 1.0f / sqrtf(ss * inv_d + a.eps);
                float r[V];
                if (!GRAD) {
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] = v[i] * rstd * (is_q ? wq[i] : wk[i]);
                    turn(r, cs, sn, 1.0f);
                } else {
                    const T* gt = reinterpret_cast<const T*>(&g[k]);
                    float dot = 0.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] = to_float(gt[i]);
                    turn(r, cs, sn, -1.0f);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        v[i] *= rstd;
                        const float dw = bad ? 0.0f : r[i] * v[i];
                        dwq[i] += is_q ? dw : 0.0f;
                        dwk[i] += is_q ? 0.0f : dw;
                        r[i] *= is_q ? wq[i] : wk[i];
                        dot += r[i] * v[i];
                    }
#pragma unroll
                    for (int o = GL / 2; o; o >>= 1) dot += __shfl_xor_sync(mask, dot, o, GL);
                    dot *= inv_d;
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] = rstd * (r[i] - v[i] * dot);
                }
                if (live) {
                    uint4 y;
                    T* yt = reinterpret_cast<T*>(&y);
#pragma unroll
                    for (int i = 0; i < V; ++i) yt[i] = from_float<T>(bad ? 0.0f : r[i]);
                    store_unit(static_cast<T*>(dst.data) + t * dst.token_stride + at * dst.head_stride + i0, y, whole);
                }
            }
        }
    }
    if (GRAD) {  // the block's groups, in order
        __shared__ float s[kGroups][GL * V];
        for (int side = 0; side < 2; ++side) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v) s[group][i0 + v] = side ? dwk[v] : dwq[v];
            __syncthreads();
            for (int i = threadIdx.x; i < D; i += 256) {
                float sum = 0.0f;
#pragma unroll
                for (int k = 0; k < kGroups; ++k) sum += s[k][i];
                partial[((int64_t)side * gridDim.x + blockIdx.x) * D + i] = sum;
            }
        }
    }
}

// Sums the blocks' partial weight gradients, one block per 32 columns of dwq or dwk.
__global__ void __launch_bounds__(1024) weight_grad_kernel(const float* partial, int blocks, int D, float* dwq,
                                                           float* dwk) {
    __shared__ float s[32][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int i = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (i < D)
#pragma unroll 4
        for (int b = warp; b < blocks; b += 32) v += partial[((int64_t)blockIdx.y * blocks + b) * D + i];
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < D) {
        for (int k = 1; k < 32; ++k) v += s[k][lane];
        (blockIdx.y ? dwk : dwq)[i] = v;
    }
}

int elem_bytes(int32_t dtype) { return dtype == HEDDLE_FP32 ? 4 : 2; }

bool units16(const heddle_heads& t, int heads, int size) {
    return heads == 0 || ((uintptr_t)t.data % 16 == 0 && t.token_stride * size % 16 == 0 && t.head_stride * size % 16 == 0);
}

// Heads of whole 16-byte units in at most 32 lanes, pairs that lie in one
// lane or in the same places of two: by sizes alone, so that results do not
// depend on where the tensors lie.
bool wide_takes(const heddle_qk_norm_rope_args& a) {
    const int V = 16 / elem_bytes(a.dtype);
    return a.head_dim % V == 0 && a.head_dim / V <= 32 && a.rot_dim % (a.interleaved ? V : 2 * V) == 0;
}
bool whole_units(const heddle_qk_norm_rope_grad_args& g, bool grad) {
    const heddle_qk_norm_rope_args& a = g.fwd;
    const int size = elem_bytes(a.dtype);
    return units16(a.q, a.q_heads, size) && units16(a.k, a.k_heads, size) && units16(a.q_out, a.q_heads, size) &&
           units16(a.k_out, a.k_heads, size) &&
           (!grad || (units16(g.dq, a.q_heads, size) && units16(g.dk, a.k_heads, size)));
}

struct Launch {
    bool wide, whole;
    int lanes, chunk, blocks;
};
Launch plan_rows(const OpContext& x, const heddle_qk_norm_rope_grad_args& g, bool grad) {
    const heddle_qk_norm_rope_args& a = g.fwd;
    Launch l{wide_takes(a), whole_units(g, grad), 32, 1, 1};
    const int64_t heads = (int64_t)a.q_heads + a.k_heads;
    int64_t want;
    if (l.wide) {
        const int need = a.head_dim * elem_bytes(a.dtype) / 16;
        l.lanes = need <= 8 ? 8 : need <= 16 ? 16 : 32;
        const int groups = 256 / l.lanes;
        // several heads a group once every SM has groups enough without
        l.chunk = a.tokens * ceil_div(heads, 8) >= (int64_t)x.num_sms * groups * 4 ? 8 : 1;
        want = ceil_div(a.tokens * ceil_div(heads, l.chunk), groups);
    } else {
        want = ceil_div(a.tokens * heads, kWarps);
    }
    const int64_t most = (int64_t)x.num_sms * 8;
    l.blocks = (int)(want < 1 ? 1 : want < most ? want : most);
    return l;
}

template <class T, bool GRAD>
void launch_typed(const Launch& l, const OpContext& x, const heddle_qk_norm_rope_grad_args& a, float* partial,
                  cudaStream_t st) {
    if (!l.wide)
        qk_norm_rope_kernel<T, GRAD><<<l.blocks, kWarps * 32, 0, st>>>(a, partial, x.err);
    else if (l.lanes == 8)
        qk_norm_rope_wide_kernel<T, 8, GRAD><<<l.blocks, 256, 0, st>>>(a, partial, x.err, l.chunk, l.whole);
    else if (l.lanes == 16)
        qk_norm_rope_wide_kernel<T, 16, GRAD><<<l.blocks, 256, 0, st>>>(a, partial, x.err, l.chunk, l.whole);
    else
        qk_norm_rope_wide_kernel<T, 32, GRAD><<<l.blocks, 256, 0, st>>>(a, partial, x.err, l.chunk, l.whole);
}

template <bool GRAD>
void launch_rows(const Launch& l, const OpContext& x, const heddle_qk_norm_rope_grad_args& a, float* partial,
                 cudaStream_t st) {
    if (a.fwd.dtype == HEDDLE_BF16)
        launch_typed<__nv_bfloat16, GRAD>(l, x, a, partial, st);
    else if (a.fwd.dtype == HEDDLE_FP16)
        launch_typed<__half, GRAD>(l, x, a, partial, st);
    else
        launch_typed<float, GRAD>(l, x, a, partial, st);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const OpContext& x, const heddle_qk_norm_rope_args& a, cudaStream_t st) {
    heddle_qk_norm_rope_grad_args ga{};
    ga.fwd = a;
    launch_rows<false>(plan_rows(x, ga, false), x, ga, nullptr, st);
    return cudaGetLastError();
}

size_t qk_norm_rope_grad_scratch(const OpContext& x, const heddle_qk_norm_rope_grad_args& a) {
    return align256(sizeof(float) * 2 * (size_t)plan_rows(x, a, true).blocks * a.fwd.head_dim);
}

cudaError_t launch_qk_norm_rope_grad(const OpContext& x, const heddle_qk_norm_rope_grad_args& a, unsigned char* ws,
                                     cudaStream_t st) {
    float* partial = reinterpret_cast<float*>(ws);
    const Launch l = plan_rows(x, a, true);
    launch_rows<true>(l, x, a, partial, st);
    const int D = a.fwd.head_dim;
    weight_grad_kernel<<<dim3((unsigned)ceil_div(D, 32), 2), 1024, 0, st>>>(partial, l.blocks, D, a.dwq, a.dwk);
    return cudaGetLastError();
}

}  // namespace hd
