// heddle_qknorm.cu -- norms of queries and keys per head with the position
// rotation in the same pass, and their gradients.
//
// Bound by memory: a head is read and written once, everything between stays
// in registers (16384 tokens of 72 heads of 128 bfloat16: forward 108 us for
// 606 MB, backward 168 us for 910 MB, 5.6e12 and 5.4e12 bytes a second).
// Where heads are whole 16-byte units, a group of lanes holds a head, 16
// bytes a lane, and walks over several heads of one token, whose cosines and
// sines it keeps; what lies at other addresses is read and written value by
// value, with the same results.  A head of any other size takes the kernel of
// one warp a head, its values dealt out one by one.

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
    allow_dependents();
    await_previous();
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

// Half of a lane's values: 8 bytes, at once or one by one.
template <class T>
__device__ __forceinline__ uint2 load_half(const T* p, bool whole) {
    if (whole) return *reinterpret_cast<const uint2*>(p);
    uint2 u;
    T* t = reinterpret_cast<T*>(&u);
#pragma unroll
    for (int i = 0; i < (int)(8 / sizeof(T)); ++i) t[i] = p[i];
    return u;
}
template <class T>
__device__ __forceinline__ void store_half(T* p, const uint2& u, bool whole) {
    if (whole) {
        *reinterpret_cast<uint2*>(p) = u;
        return;
    }
    const T* t = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < (int)(8 / sizeof(T)); ++i) p[i] = t[i];
}

// 1 / sqrt(v), the approximation and one step of Newton's iteration for it.
__device__ __forceinline__ float inv_sqrt(float v) {
    const float r = rsqrtf(v);
    return v > 0.0f && v < INFINITY ? r * fmaf(-0.5f * v * r, r, 1.5f) : r;
}

// What the kernel knows of a call beforehand.  kAny: nothing.  kHalves and
// kPairs: the layout of the pairs, and that all lies at whole units; two
// thirds of the instructions then (16384 tokens of 72 heads of 128 bfloat16,
// forward: 186 us as kAny, 114 us).  kAllHalves and kAllPairs: also that every
// lane has values and turns them, as most models' heads do (108 us).
enum RotaryCase { kAny, kHalves, kPairs, kAllHalves, kAllPairs };

// A head of whole 16-byte units in a group of GL lanes, V values a lane, the
// last lanes idle where head_dim / V is not GL.  A lane's values are two runs
// of V / 2 that hold both values of every pair they turn: places i.. and
// i + rot_dim / 2.., or 2i.., so that no value changes lanes.  A block takes
// queries or keys alone (the first q_blocks queries); a group takes `chunk`
// heads of one token at a time and keeps its angles.  Sums and differences of
// products are spelled out, so that every case rounds alike.
template <class T, int GL, bool GRAD, RotaryCase CASE>
__global__ void __launch_bounds__(256, 3)
    qk_norm_rope_wide_kernel(const __grid_constant__ heddle_qk_norm_rope_grad_args ga, float* partial, uint32_t* err,
                             int q_blocks, int chunk, bool whole_units) {
    allow_dependents();
    await_previous();
    constexpr int V = 16 / sizeof(T), H = V / 2, kGroups = 256 / GL, kDepth = GRAD ? 2 : 4;
    const heddle_qk_norm_rope_args& a = ga.fwd;
    const bool is_q = blockIdx.x < q_blocks;
    const int block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : gridDim.x - q_blocks;
    const int heads = is_q ? a.q_heads : a.k_heads, chunks = (heads + chunk - 1) / chunk;
    const heddle_heads in = is_q ? a.q : a.k, out = is_q ? a.q_out : a.k_out, dst = is_q ? ga.dq : ga.dk;
    const int lane = threadIdx.x % GL, group = threadIdx.x / GL;
    constexpr bool kAll = CASE == kAllHalves || CASE == kAllPairs;
    const int D = kAll ? GL * V : a.head_dim, rot = kAll ? D : a.rot_dim;
    const bool live = kAll || lane * V < D, turns = kAll || lane * V < rot;
    const bool inter = CASE == kAny ? a.interleaved : CASE == kPairs || CASE == kAllPairs;
    const bool whole = CASE != kAny || whole_units;
    // the lane's two runs; lanes past the turned part hold V values in a row,
    // those past the head read its first ones and count for nothing
    const int at0 = !live ? 0 : turns && !inter ? lane * H : lane * V;
    const int at1 = turns && !inter ? at0 + rot / 2 : at0 + H;
    const uint32_t mask = GL == 32 ? ~0u : ((1u << (GL & 31)) - 1) << (threadIdx.x % 32 / GL * GL);
    const float inv_d = 1.0f / D;
    float w[V], dw[V] = {};
    {
        const T* wt = static_cast<const T*>(is_q ? a.wq : a.wk);
#pragma unroll
        for (int v = 0; v < H; ++v) {
            w[v] = to_float(wt[at0 + v]);
            w[H + v] = to_float(wt[at1 + v]);
        }
    }

    const int64_t units = a.tokens * chunks;
    for (int64_t u = (int64_t)block * kGroups + group; u < units; u += (int64_t)blocks * kGroups) {
        const int64_t t = u / chunks;
        const int h0 = (int)(u - t * chunks) * chunk, count = min(heads - h0, chunk);
        float cs[H], sn[H];
        bool bad = false;
        if (rot) {
            const int64_t p = a.positions[t];
            bad = p < 0 || p >= a.table_len;
            const int64_t at = (bad ? 0 : p) * (rot / 2) + (turns ? lane * H : 0);
            if (bad) {
                if (lane == 0) atomicOr(err, kErrOpPosition);
            } else if (CASE != kAny) {
#pragma unroll
                for (int v = 0; v < H; v += 2) {
                    const float2 c = *reinterpret_cast<const float2*>(a.cos + at + v),
                                 s = *reinterpret_cast<const float2*>(a.sin + at + v);
                    cs[v] = c.x, cs[v + 1] = c.y, sn[v] = s.x, sn[v + 1] = s.y;
                }
            } else {
#pragma unroll
                for (int v = 0; v < H; ++v) cs[v] = a.cos[at + v], sn[v] = a.sin[at + v];
            }
        }
        const T* x_at = static_cast<const T*>(in.data) + t * in.token_stride + h0 * in.head_stride;
        const T* g_at = static_cast<const T*>(out.data) + t * out.token_stride + h0 * out.head_stride;
        T* y_at = GRAD ? static_cast<T*>(dst.data) + t * dst.token_stride + h0 * dst.head_stride
                       : static_cast<T*>(out.data) + t * out.token_stride + h0 * out.head_stride;
        const int64_t y_step = GRAD ? dst.head_stride : out.head_stride;
        if (bad) {  // no such position: zeros
            for (int h = 0; h < count; ++h)
                if (live) {
                    store_half(y_at + h * y_step + at0, make_uint2(0, 0), whole);
                    store_half(y_at + h * y_step + at1, make_uint2(0, 0), whole);
                }
            continue;
        }
        // the lane's pairs turned by the angles, back by their negatives
        auto turn = [&](float (&v)[V], bool back) {
            if (!rot) return;
            auto pair = [&](float& x, float& y, int k) {
                const float s = back ? -sn[k] : sn[k];
                const float tx = fmaf(x, cs[k], -__fmul_rn(y, s)), ty = fmaf(y, cs[k], __fmul_rn(x, s));
                x = turns ? tx : x;
                y = turns ? ty : y;
            };
            if (inter) {
#pragma unroll
                for (int k = 0; k < H; ++k) pair(v[2 * k], v[2 * k + 1], k);
            } else {
#pragma unroll
                for (int k = 0; k < H; ++k) pair(v[k], v[H + k], k);
            }
        };
        for (int h = 0; h < count; h += kDepth) {
            // heads past the last are the last again, not stored
            uint2 x[kDepth][2], g[kDepth][2];
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const int at = min(k, count - 1 - h);
                x[k][0] = load_half(x_at + at * in.head_stride + at0, whole);
                x[k][1] = load_half(x_at + at * in.head_stride + at1, whole);
                if (GRAD) {
                    g[k][0] = load_half(g_at + at * out.head_stride + at0, whole);
                    g[k][1] = load_half(g_at + at * out.head_stride + at1, whole);
                }
            }
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const bool stored = h + k < count;
                float v[V], ss = 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[i] = to_float(reinterpret_cast<const T*>(&x[k][i / H])[i % H]);
                    ss = fmaf(v[i], v[i], ss);
                }
                ss = live ? ss : 0.0f;
#pragma unroll
                for (int o = GL / 2; o; o >>= 1) ss += __shfl_xor_sync(mask, ss, o, GL);
                const float rstd = inv_sqrt(fmaf(ss, inv_d, a.eps));
                float r[V];
                if (!GRAD) {
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] = v[i] * rstd * w[i];
                    turn(r, false);
                } else {
                    float dot = 0.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] = to_float(reinterpret_cast<const T*>(&g[k][i / H])[i % H]);
                    turn(r, true);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float d = r[i];
                        v[i] *= rstd;
                        if (stored) dw[i] = fmaf(d, v[i], dw[i]);
                        r[i] = d * w[i];
                        dot = fmaf(r[i], v[i], dot);
                    }
                    dot = live ? dot : 0.0f;
#pragma unroll
                    for (int o = GL / 2; o; o >>= 1) dot += __shfl_xor_sync(mask, dot, o, GL);
                    dot *= inv_d;
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] = rstd * fmaf(-v[i], dot, r[i]);
                }
                if (live && stored) {
                    uint2 y[2];
#pragma unroll
                    for (int i = 0; i < V; ++i) reinterpret_cast<T*>(&y[i / H])[i % H] = from_float<T>(r[i]);
                    store_half(y_at + k * y_step + at0, y[0], whole);
                    store_half(y_at + k * y_step + at1, y[1], whole);
                }
            }
            x_at += kDepth * in.head_stride;
            g_at += kDepth * out.head_stride;
            y_at += kDepth * y_step;
        }
    }
    if (GRAD) {  // the block's groups, in order
        __shared__ float s[kGroups][GL * V];
#pragma unroll
        for (int v = 0; v < H; ++v)
            if (live) s[group][at0 + v] = dw[v], s[group][at1 + v] = dw[H + v];
        __syncthreads();
        for (int i = threadIdx.x; i < D; i += 256) {
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kGroups; ++k) sum += s[k][i];
            partial[(int64_t)blockIdx.x * D + i] = sum;
        }
    }
}

// Sums the blocks' partial weight gradients, one block per 32 columns of dwq
// (the first q_blocks blocks) or dwk (the next k_blocks).
__global__ void __launch_bounds__(1024) weight_grad_kernel(const float* partial, int q_blocks, int k_blocks, int D,
                                                           float* dwq, float* dwk) {
    allow_dependents();
    await_previous();
    __shared__ float s[32][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int i = blockIdx.x * 32 + lane;
    float v = 0.0f;
    const int first = blockIdx.y ? q_blocks : 0, blocks = blockIdx.y ? k_blocks : q_blocks;
    if (i < D)
#pragma unroll 8
        for (int b = warp; b < blocks; b += 32) v += partial[(int64_t)(first + b) * D + i];
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < D) {
        for (int k = 1; k < 32; ++k) v += s[k][lane];
        (blockIdx.y ? dwk : dwq)[i] = v;
    }
}

int elem_bytes(int32_t dtype) { return dtype == HEDDLE_FP32 ? 4 : 2; }

bool units8(const heddle_heads& t, int heads, int size) {
    return heads == 0 ||
           ((uintptr_t)t.data % 8 == 0 && t.token_stride * size % 8 == 0 && t.head_stride * size % 8 == 0);
}

// Heads of whole 16-byte units in at most 32 lanes, whole lanes of turned
// values: by sizes alone, so that results do not depend on where the tensors
// lie.
bool wide_takes(const heddle_qk_norm_rope_args& a) {
    const int V = 16 / elem_bytes(a.dtype);
    return a.head_dim % V == 0 && a.head_dim / V <= 32 && a.rot_dim % V == 0;
}
bool whole_units(const heddle_qk_norm_rope_grad_args& g, bool grad) {
    const heddle_qk_norm_rope_args& a = g.fwd;
    const int size = elem_bytes(a.dtype);
    return (uintptr_t)a.cos % 8 == 0 && (uintptr_t)a.sin % 8 == 0 && units8(a.q, a.q_heads, size) &&
           units8(a.k, a.k_heads, size) && units8(a.q_out, a.q_heads, size) &&
           units8(a.k_out, a.k_heads, size) &&
           (!grad || (units8(g.dq, a.q_heads, size) && units8(g.dk, a.k_heads, size)));
}

struct Launch {
    bool wide, whole;
    int lanes, chunk, q_blocks, k_blocks;
};
Launch plan_rows(const OpContext& x, const heddle_qk_norm_rope_grad_args& g, bool grad) {
    const heddle_qk_norm_rope_args& a = g.fwd;
    Launch l{wide_takes(a), whole_units(g, grad), 32, 1, 0, 0};
    const int64_t heads = (int64_t)a.q_heads + a.k_heads;
    if (!l.wide) {  // rows of queries and keys by turns: both sums over all blocks
        const int64_t want = ceil_div(a.tokens * heads, kWarps), most = (int64_t)x.num_sms * 8;
        l.q_blocks = l.k_blocks = (int)(want < 1 ? 1 : want < most ? want : most);
        return l;
    }
    const int need = a.head_dim * elem_bytes(a.dtype) / 16;
    l.lanes = need <= 8 ? 8 : need <= 16 ? 16 : 32;
    const int groups = 256 / l.lanes;
    // as many heads a group, up to eight, as leave every group that runs at a
    // time four units of them
    for (l.chunk = 8; l.chunk > 1; l.chunk /= 2)
        if (a.tokens * (ceil_div(a.q_heads, l.chunk) + ceil_div(a.k_heads, l.chunk)) >=
            (int64_t)x.num_sms * groups * 12)
            break;
    const int64_t q_want = ceil_div(a.tokens * ceil_div(a.q_heads, l.chunk), groups),
                  k_want = ceil_div(a.tokens * ceil_div(a.k_heads, l.chunk), groups);
    const int64_t most = (int64_t)x.num_sms * 6;  // two rounds of three blocks an SM
    if (q_want + k_want <= most) {
        l.q_blocks = (int)q_want, l.k_blocks = (int)k_want;
    } else {  // shared by heads, one block at least where there are any
        int64_t kb = most * a.k_heads / heads;
        kb = a.k_heads && kb < 1 ? 1 : kb;
        const int64_t qb = a.q_heads ? (most - kb < 1 ? 1 : most - kb) : 0;
        l.q_blocks = (int)(qb < q_want ? qb : q_want);
        l.k_blocks = (int)(kb < k_want ? kb : k_want);
    }
    return l;
}

template <class T, int GL, bool GRAD>
void launch_wide(const Launch& l, const OpContext& x, const heddle_qk_norm_rope_grad_args& a, float* partial,
                 cudaStream_t st) {
    const int blocks = l.q_blocks + l.k_blocks;
    const bool all = a.fwd.rot_dim == a.fwd.head_dim && a.fwd.head_dim == GL * (int)(16 / sizeof(T));
    auto* kernel = !l.whole            ? qk_norm_rope_wide_kernel<T, GL, GRAD, kAny>
                   : a.fwd.interleaved ? (all ? qk_norm_rope_wide_kernel<T, GL, GRAD, kAllPairs>
                                              : qk_norm_rope_wide_kernel<T, GL, GRAD, kPairs>)
                                       : (all ? qk_norm_rope_wide_kernel<T, GL, GRAD, kAllHalves>
                                              : qk_norm_rope_wide_kernel<T, GL, GRAD, kHalves>);
    launch(x, kernel, dim3(blocks), 256, 0, st, a, partial, x.err, l.q_blocks, l.chunk, l.whole);
}

template <class T, bool GRAD>
void launch_typed(const Launch& l, const OpContext& x, const heddle_qk_norm_rope_grad_args& a, float* partial,
                  cudaStream_t st) {
    const int blocks = l.q_blocks + l.k_blocks;
    if (!l.wide)
        launch(x, qk_norm_rope_kernel<T, GRAD>, dim3(l.q_blocks), kWarps * 32, 0, st, a, partial, x.err);
    else if (blocks == 0)
        return;
    else if (l.lanes == 8)
        launch_wide<T, 8, GRAD>(l, x, a, partial, st);
    else if (l.lanes == 16)
        launch_wide<T, 16, GRAD>(l, x, a, partial, st);
    else
        launch_wide<T, 32, GRAD>(l, x, a, partial, st);
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
    const Launch l = plan_rows(x, a, true);
    return align256(sizeof(float) * (size_t)(l.q_blocks + l.k_blocks) * a.fwd.head_dim);
}

cudaError_t launch_qk_norm_rope_grad(const OpContext& x, const heddle_qk_norm_rope_grad_args& a, unsigned char* ws,
                                     cudaStream_t st) {
    float* partial = reinterpret_cast<float*>(ws);
    const Launch l = plan_rows(x, a, true);
    launch_rows<true>(l, x, a, partial, st);
    const int D = a.fwd.head_dim;
    launch(x, weight_grad_kernel, dim3((unsigned)ceil_div(D, 32), 2), 1024, 0, st, partial, l.q_blocks, l.k_blocks, D,
           a.dwq, a.dwk);
    return cudaGetLastError();
}

}  // namespace hd
