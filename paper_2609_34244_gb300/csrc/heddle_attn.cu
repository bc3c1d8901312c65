// heddle_attn.cu -- attention with a sliding window and first tokens that
// stay visible, one warp per row: any head_dim, stride and alignment.

#include <type_traits>

#include "heddle_attn.cuh"

namespace hd {
namespace {

constexpr int kWarps = 8;
constexpr int kVals = 8;  // values of a head a lane holds: head_dim <= 256

template <class T>
__device__ __forceinline__ const T* at(const heddle_heads& t, int64_t b, int64_t i, int64_t h) {
    return static_cast<const T*>(t.data) + b * t.batch_stride + i * t.token_stride + h * t.head_stride;
}
template <class T>
__device__ __forceinline__ T* out_at(const heddle_heads& t, int64_t b, int64_t i, int64_t h) {
    return static_cast<T*>(t.data) + b * t.batch_stride + i * t.token_stride + h * t.head_stride;
}

template <class T>
__device__ __forceinline__ void load_row(const T* p, int D, int lane, float (&v)[kVals]) {
#pragma unroll
    for (int j = 0; j < kVals; ++j) v[j] = lane + 32 * j < D ? to_float(p[lane + 32 * j]) : 0.0f;
}
template <class T>
__device__ __forceinline__ void store_row(T* p, int D, int lane, const float (&v)[kVals], float f) {
#pragma unroll
    for (int j = 0; j < kVals; ++j)
        if (lane + 32 * j < D) p[lane + 32 * j] = from_float<T>(v[j] * f);
}
__device__ __forceinline__ float dot_rows(const float (&a)[kVals], const float (&b)[kVals]) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < kVals; ++j) s += a[j] * b[j];
    return warp_sum(s);
}

template <class T>
__global__ void __launch_bounds__(kWarps * 32) attn_row_kernel(heddle_attention_args a) {
    const int lane = threadIdx.x % 32, D = a.head_dim;
    const int64_t rows = a.batch * a.q_heads * a.q_len;
    for (int64_t r = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; r < rows; r += (int64_t)gridDim.x * kWarps) {
        const int64_t b = r / (a.q_heads * a.q_len), h = r / a.q_len % a.q_heads, i = r % a.q_len;
        const int64_t hk = h / (a.q_heads / a.kv_heads);
        const Span s = span_of(a, b);
        const int64_t p = i < s.ql ? s.off + i : -1;
        float q[kVals], o[kVals] = {}, m = -INFINITY, l = 0.0f;
        load_row(at<T>(a.q, b, i, h), D, lane, q);
        const int64_t low = a.window && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
        for (int64_t j = 0; j <= p; ++j) {
            if (j < low && j >= a.sinks) j = low;
            float k[kVals], v[kVals];
            load_row(at<T>(a.k, b, j, hk), D, lane, k);
            load_row(at<T>(a.v, b, j, hk), D, lane, v);
            const float sc = dot_rows(q, k) * a.scale;
            const float top = fmaxf(m, sc);
            const float keep = m == -INFINITY ? 0.0f : expf(m - top), w = sc == -INFINITY ? 0.0f : expf(sc - top);
            l = l * keep + w;
#pragma unroll
            for (int x = 0; x < kVals; ++x) o[x] = o[x] * keep + w * v[x];
            m = top;
        }
        store_row(out_at<T>(a.o, b, i, h), D, lane, o, l == 0.0f ? 0.0f : 1.0f / l);
        if (a.lse && lane == 0) a.lse[r] = l == 0.0f ? -INFINITY : m + logf(l);
    }
}

// The counters of kernels that hand out work, zero at the start of every call's
// gradients: whatever calls that overlapped against the rule left in them would
// make all later ones leave out query tiles.  The maxima start from zero too.
__device__ __forceinline__ void start_pieces(int32_t* sched) {
    if (blockIdx.x == 0 && threadIdx.x < kSched) sched[threadIdx.x] = 0;
}

// delta_i = do_i . o_i for heads of whole 16-byte units: GL lanes a row, 16
// bytes a lane, rows in the order of memory.  Bound by memory: 67 MB in 14 us
// with its launch (4096 tokens of 32 heads of 128; a warp a row took 33).
template <class T, int GL>
__global__ void __launch_bounds__(256) attn_delta_wide_kernel(const __grid_constant__ heddle_attention_grad_args g,
                                                              float* delta, int32_t* sched) {
    allow_dependents();
    await_previous();
    start_pieces(sched);
    const heddle_attention_args& a = g.fwd;
    const int lane = threadIdx.x % GL;
    const uint32_t r = blockIdx.x * (256 / GL) + threadIdx.x / GL;  // (b, i, h)
    const uint32_t heads = a.q_heads, n = (uint32_t)a.q_len;
    if (r >= a.batch * heads * n) return;
    const uint32_t h = r % heads, bi = r / heads, i = bi % n, b = bi / n;
    float s = 0.0f;
    if (lane * 8 < a.head_dim) {
        const uint4 u = *reinterpret_cast<const uint4*>(at<T>(a.o, b, i, h) + lane * 8);
        const uint4 w = *reinterpret_cast<const uint4*>(at<T>(g.d_o, b, i, h) + lane * 8);
        const T *x = reinterpret_cast<const T*>(&u), *y = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += to_float(x[j]) * to_float(y[j]);
    }
    const uint32_t mask = ((1ull << GL) - 1) << (threadIdx.x % 32 / GL * GL);
#pragma unroll
    for (int o = GL / 2; o; o >>= 1) s += __shfl_xor_sync(mask, s, o, GL);
    if (lane == 0) delta[((int64_t)b * heads + h) * n + i] = s;
}

// Queries that see at most this many keys take delta from the weights
// instead, sum_j P_ij (do_i . v_j): o is rounded to the element type, which is
// as large an error of dS there as the rounding of dS itself, and fades with
// more keys.  They are the first kFewKeys positions of a sequence, or every
// query of a call whose window and sinks together are no more.
constexpr int kFewKeys = 16;

// 16 lanes a row, a key each; `per` rows a head: the queries of the first
// `per` positions, or (all) the first `per` queries.  The row, or -1.
template <class T>
__device__ __forceinline__ int64_t few_delta(const heddle_attention_grad_args& g, int64_t per, bool all, float* value) {
    const heddle_attention_args& a = g.fwd;
    const int lane = threadIdx.x % kFewKeys, D = a.head_dim;
    const int64_t r = (int64_t)blockIdx.x * (256 / kFewKeys) + threadIdx.x / kFewKeys;  // (b, h, e)
    if (r >= a.batch * a.q_heads * per) return -1;
    const int64_t e = r % per, h = r / per % a.q_heads, b = r / (per * a.q_heads);
    const Span sp = span_of(a, b);
    const int64_t i = all ? e : e - sp.off, pos = sp.off + i;
    if (i < 0 || i >= sp.ql || pos < 0) return -1;
    const int64_t low = a.window && pos + 1 > a.window ? pos + 1 - a.window : 0;
    const int64_t first = min(a.sinks, low), keys = first + pos + 1 - low;
    if (keys > kFewKeys) return -1;
    const int64_t hk = h / (a.q_heads / a.kv_heads), row = (b * a.q_heads + h) * a.q_len + i;
    const uint32_t mask = 0xffffu << (threadIdx.x % 32 / kFewKeys * kFewKeys);
    float s = 0.0f, total = 0.0f;
    if (lane < keys) {
        const int64_t key = lane < first ? lane : low + lane - first;
        const T *q = at<T>(a.q, b, i, h), *d_o = at<T>(g.d_o, b, i, h);
        const T *k = at<T>(a.k, b, key, hk), *v = at<T>(a.v, b, key, hk);
        float qk = 0.0f, dv = 0.0f;
#pragma unroll 4
        for (int c = 0; c < D; c += 8) {
            const uint4 uq = *reinterpret_cast<const uint4*>(q + c), uk = *reinterpret_cast<const uint4*>(k + c);
            const uint4 ud = *reinterpret_cast<const uint4*>(d_o + c), uv = *reinterpret_cast<const uint4*>(v + c);
            const T *tq = reinterpret_cast<const T*>(&uq), *tk = reinterpret_cast<const T*>(&uk);
            const T *td = reinterpret_cast<const T*>(&ud), *tv = reinterpret_cast<const T*>(&uv);
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                qk += to_float(tq[x]) * to_float(tk[x]);
                dv += to_float(td[x]) * to_float(tv[x]);
            }
        }
        total = expf(qk * a.scale - a.lse[row]);
        s = total * dv;
    }
#pragma unroll
    for (int o = kFewKeys / 2; o; o >>= 1) {
        s += __shfl_xor_sync(mask, s, o, kFewKeys);
        total += __shfl_xor_sync(mask, total, o, kFewKeys);
    }
    *value = s / total;
    return row;
}

// The largest square of a gradient's row (which 0) or of a value's (1), of those
// that count and are finite, GL lanes a row: what dS of float16 is kept in range
// by (ds_factor).  `block` of `blocks`; to sched[2 + which], the same in any
// order.
template <class T, int GL>
__device__ __forceinline__ void row_squares(const heddle_attention_grad_args& g, int which, int block, int blocks,
                                            int32_t* sched) {
    const heddle_attention_args& a = g.fwd;
    constexpr int kAhead = 4;
    const int lane = threadIdx.x % GL;
    const int64_t step = (int64_t)blocks * (256 / GL);
    const uint32_t mask = ((1ull << GL) - 1) << (threadIdx.x % 32 / GL * GL);
    const heddle_heads& t = which ? a.v : g.d_o;
    const uint32_t n = (uint32_t)(which ? a.kv_len : a.q_len), heads = which ? a.kv_heads : a.q_heads;
    const int64_t rows = a.batch * heads * n;
    float most = 0.0f;
    for (int64_t r0 = (int64_t)block * (256 / GL) + threadIdx.x / GL; r0 < rows; r0 += kAhead * step) {
        uint4 u[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            u[k] = make_uint4(0, 0, 0, 0);
            if (r0 + k * step >= rows || lane * 8 >= a.head_dim) continue;
            const uint32_t r = (uint32_t)(r0 + k * step), h = r % heads, bi = r / heads, i = bi % n, b = bi / n;
            const Span s = span_of(a, b);
            if (i < (which ? s.kl : s.ql)) u[k] = *reinterpret_cast<const uint4*>(at<T>(t, b, i, h) + lane * 8);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const T* x = reinterpret_cast<const T*>(&u[k]);
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += to_float(x[j]) * to_float(x[j]);
#pragma unroll
            for (int o = GL / 2; o; o >>= 1) s += __shfl_xor_sync(mask, s, o, GL);
            if (s < INFINITY) most = fmaxf(most, s);
        }
    }
    __shared__ float parts[8];
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < 8; ++k) most = fmaxf(most, parts[k]);
        await_previous();  // which sets it to zero
        if (most > 0.0f) atomicMax(sched + 2 + which, __float_as_int(most));
    }
}

// Blocks from `few` on, of float16 alone: row_squares, `squares` of them of the
// gradients' rows and the others of the values'.
template <class T, int GL>
__global__ void __launch_bounds__(256) attn_few_delta_kernel(const __grid_constant__ heddle_attention_grad_args g,
                                                             float* delta, int64_t per, bool all, int few,
                                                             int squares, int32_t* sched) {
    allow_dependents();
    if (std::is_same<T, __half>::value && (int)blockIdx.x >= few) {
        const int block = (int)blockIdx.x - few, others = (int)gridDim.x - few - squares;
        const int which = block >= squares;
        row_squares<T, GL>(g, which, which ? block - squares : block, which ? others : squares, sched);
        return;
    }
    float value = 0.0f;
    const int64_t row = few_delta<T>(g, per, all, &value);
    await_previous();  // which writes these rows as well
    if (row >= 0 && threadIdx.x % kFewKeys == 0) delta[row] = value;
}

bool units16(const heddle_heads& t) {
    return (uintptr_t)t.data % 16 == 0 && t.batch_stride % 8 == 0 && t.token_stride % 8 == 0 && t.head_stride % 8 == 0;
}

// delta_i = do_i . o_i
template <class T>
__global__ void __launch_bounds__(kWarps * 32) attn_delta_kernel(heddle_attention_grad_args g, float* delta,
                                                                 int32_t* sched) {
    allow_dependents();
    await_previous();
    start_pieces(sched);
    const heddle_attention_args& a = g.fwd;
    const int lane = threadIdx.x % 32, D = a.head_dim;
    const int64_t rows = a.batch * a.q_heads * a.q_len;
    for (int64_t r = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; r < rows; r += (int64_t)gridDim.x * kWarps) {
        const int64_t b = r / (a.q_heads * a.q_len), h = r / a.q_len % a.q_heads, i = r % a.q_len;
        float o[kVals], d[kVals];
        load_row(at<T>(a.o, b, i, h), D, lane, o);
        load_row(at<T>(g.d_o, b, i, h), D, lane, d);
        const float s = dot_rows(o, d);
        if (lane == 0) delta[r] = s;
    }
}

template <class T>
__global__ void __launch_bounds__(kWarps * 32) attn_dq_row_kernel(heddle_attention_grad_args g, const float* delta) {
    const heddle_attention_args& a = g.fwd;
    const int lane = threadIdx.x % 32, D = a.head_dim;
    const int64_t rows = a.batch * a.q_heads * a.q_len;
    for (int64_t r = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; r < rows; r += (int64_t)gridDim.x * kWarps) {
        const int64_t b = r / (a.q_heads * a.q_len), h = r / a.q_len % a.q_heads, i = r % a.q_len;
        const int64_t hk = h / (a.q_heads / a.kv_heads);
        const Span s = span_of(a, b);
        const int64_t p = i < s.ql ? s.off + i : -1;
        float q[kVals], d[kVals], dq[kVals] = {};
        load_row(at<T>(a.q, b, i, h), D, lane, q);
        load_row(at<T>(g.d_o, b, i, h), D, lane, d);
        const float lse = a.lse[r], dl = delta[r];
        const int64_t low = a.window && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
        for (int64_t j = 0; j <= p; ++j) {
            if (j < low && j >= a.sinks) j = low;
            float k[kVals], v[kVals];
            load_row(at<T>(a.k, b, j, hk), D, lane, k);
            load_row(at<T>(a.v, b, j, hk), D, lane, v);
            const float w = expf(dot_rows(q, k) * a.scale - lse);
            const float ds = w * (dot_rows(d, v) - dl) * a.scale;
#pragma unroll
            for (int x = 0; x < kVals; ++x) dq[x] += ds * k[x];
        }
        store_row(out_at<T>(g.dq, b, i, h), D, lane, dq, 1.0f);
    }
}

template <class T>
__global__ void __launch_bounds__(kWarps * 32) attn_dkv_row_kernel(heddle_attention_grad_args g, const float* delta) {
    const heddle_attention_args& a = g.fwd;
    const int lane = threadIdx.x % 32, D = a.head_dim;
    const int64_t rows = a.batch * a.kv_heads * a.kv_len, group = a.q_heads / a.kv_heads;
    for (int64_t r = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; r < rows; r += (int64_t)gridDim.x * kWarps) {
        const int64_t b = r / (a.kv_heads * a.kv_len), hk = r / a.kv_len % a.kv_heads, j = r % a.kv_len;
        const Span s = span_of(a, b);
        float k[kVals], v[kVals], dk[kVals] = {}, dv[kVals] = {};
        load_row(at<T>(a.k, b, j, hk), D, lane, k);
        load_row(at<T>(a.v, b, j, hk), D, lane, v);
        const int64_t first = max((int64_t)0, j - s.off);
        int64_t last = j < s.kl ? s.ql : 0;
        if (a.window && j >= a.sinks) last = min(last, j + a.window - s.off);
        for (int64_t h = hk * group; h < (hk + 1) * group; ++h)
            for (int64_t i = first; i < last; ++i) {
                float q[kVals], d[kVals];
                load_row(at<T>(a.q, b, i, h), D, lane, q);
                load_row(at<T>(g.d_o, b, i, h), D, lane, d);
                const int64_t at_row = (b * a.q_heads + h) * a.q_len + i;
                const float w = expf(dot_rows(q, k) * a.scale - a.lse[at_row]);
                const float ds = w * (dot_rows(d, v) - delta[at_row]) * a.scale;
#pragma unroll
                for (int x = 0; x < kVals; ++x) {
                    dv[x] += w * d[x];
                    dk[x] += ds * q[x];
                }
            }
        store_row(out_at<T>(g.dk, b, j, hk), D, lane, dk, 1.0f);
        store_row(out_at<T>(g.dv, b, j, hk), D, lane, dv, 1.0f);
    }
}

unsigned row_blocks(const OpContext& x, int64_t rows) {
    const int64_t most = (int64_t)x.num_sms * 64;
    return (unsigned)(ceil_div(rows, kWarps) < most ? ceil_div(rows, kWarps) : most);
}

template <class T>
cudaError_t attention_grad(const OpContext& x, const heddle_attention_grad_args& g, float* delta, unsigned char* rest,
                           bool keep, cudaStream_t st) {
    const heddle_attention_args& a = g.fwd;
    const int64_t rows = a.batch * a.q_heads * a.q_len, keys = a.batch * a.kv_heads * a.kv_len;
    const bool tc = attn_tc_takes_grad(g);
    if (rows && a.head_dim % 8 == 0 && a.head_dim <= 128 && units16(a.o) && units16(g.d_o)) {
        if (a.head_dim <= 64)
            launch(x, attn_delta_wide_kernel<T, 8>, dim3((unsigned)ceil_div(rows, 32)), 256, 0, st, g, delta,
                   x.sched);
        else
            launch(x, attn_delta_wide_kernel<T, 16>, dim3((unsigned)ceil_div(rows, 16)), 256, 0, st, g, delta,
                   x.sched);
    } else if (rows) {
        launch(x, attn_delta_kernel<T>, dim3(row_blocks(x, rows)), kWarps * 32, 0, st, g, delta, x.sched);
    }
    if (tc) {
        const bool all = a.window && a.window + a.sinks <= kFewKeys;
        const int64_t per = all || a.q_len < kFewKeys ? a.q_len : kFewKeys;
        const int64_t few = ceil_div(a.batch * a.q_heads * per, 256 / kFewKeys);
        const int group = a.head_dim <= 64 ? 8 : 16;
        auto blocks_of = [&](int64_t n) {
            const int64_t want = ceil_div(n, 4 * 256 / group), most = 4 * (int64_t)x.num_sms;
            return !std::is_same<T, __half>::value ? 0 : want < most ? want : most;
        };
        const int64_t squares = blocks_of(rows), others = blocks_of(keys);
        launch(x, group == 8 ? attn_few_delta_kernel<T, 8> : attn_few_delta_kernel<T, 16>,
               dim3((unsigned)(few + squares + others)), 256, 0, st, g, delta, per, all || a.q_len < kFewKeys, (int)few,
               (int)squares, x.sched);
        const cudaError_t e = cudaGetLastError();
        return e == cudaSuccess ? launch_attn_tc_grad(x, g, delta, rest, keep, st) : e;
    }
    if (rows) {
        attn_dq_row_kernel<T><<<row_blocks(x, rows), kWarps * 32, 0, st>>>(g, delta);
    }
    if (keys) attn_dkv_row_kernel<T><<<row_blocks(x, keys), kWarps * 32, 0, st>>>(g, delta);
    return cudaGetLastError();
}

}  // namespace

size_t attention_scratch(const OpContext& x, const heddle_attention_args& a) {
    return attn_tc_takes(a) ? attn_tc_scratch(x, a) : 0;
}

cudaError_t launch_attention(const OpContext& x, const heddle_attention_args& a, unsigned char* ws, cudaStream_t st) {
    if (attn_tc_takes(a)) return launch_attn_tc(x, a, ws, st);
    const unsigned grid = row_blocks(x, a.batch * a.q_heads * a.q_len);
    if (a.dtype == HEDDLE_BF16)
        attn_row_kernel<__nv_bfloat16><<<grid, kWarps * 32, 0, st>>>(a);
    else
        attn_row_kernel<__half><<<grid, kWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}

static size_t delta_bytes(const heddle_attention_args& a) {
    return align256(sizeof(float) * (size_t)(a.batch * a.q_heads * a.q_len));
}

size_t attention_grad_scratch(const OpContext& x, const heddle_attention_grad_args& g, bool keep) {
    return delta_bytes(g.fwd) + (attn_tc_takes_grad(g) ? attn_tc_grad_scratch(x, g.fwd, keep) : 0);
}

cudaError_t launch_attention_grad(const OpContext& x, const heddle_attention_grad_args& g, unsigned char* ws,
                                  bool keep, cudaStream_t st) {
    float* delta = reinterpret_cast<float*>(ws);
    unsigned char* rest = ws + delta_bytes(g.fwd);
    return g.fwd.dtype == HEDDLE_BF16 ? attention_grad<__nv_bfloat16>(x, g, delta, rest, keep, st)
                                      : attention_grad<__half>(x, g, delta, rest, keep, st);
}

}  // namespace hd
