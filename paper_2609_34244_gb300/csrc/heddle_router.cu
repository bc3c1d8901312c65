// heddle_router.cu -- the router of an expert layer: softmax over the experts,
// the chosen ones, their counts, the balance loss, and the gradient.
//
// A few megabytes in and out: bound by latency.  A group of lanes holds a
// token's logits in registers; the largest are found one after the other, by
// value and then by index.  What a lane's experts get, probability and
// choices, is summed in its registers over all tokens of its group, then over
// the block's groups, then over blocks by a second kernel, always in order.
// The backward pass computes the probabilities again.

#include "heddle_ops.cuh"

namespace hd {
namespace {

constexpr int kThreads = 256;
constexpr int kMostChosen = 32;

// The larger one; NaN where either is.
__device__ __forceinline__ float max_nan(float a, float b) { return a != a || a > b ? a : b; }

// A token's experts in L lanes, N a lane: lane, lane + L, ..
template <class T, int L, int N>
struct Token {
    float p[N];   // exp(logit - top), zeros past the last
    float top, total;
    __device__ __forceinline__ bool takes_part() const { return top != -INFINITY; }
    __device__ __forceinline__ bool sound() const { return top < INFINITY; }  // false for NaN

    static __device__ __forceinline__ uint32_t mask() {
        return L == 32 ? ~0u : ((1u << (L & 31)) - 1) << (threadIdx.x % 32 / L * L);
    }
    static __device__ __forceinline__ float sum(float v) {
#pragma unroll
        for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(mask(), v, o, L);
        return v;
    }
    __device__ __forceinline__ void read(const T* l, int experts, bool valid, float (&v)[N]) {
        const int lane = threadIdx.x % L;
        top = -INFINITY;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            v[j] = valid && lane + j * L < experts ? to_float(l[lane + j * L]) : -INFINITY;
            top = max_nan(top, v[j]);
        }
#pragma unroll
        for (int o = L / 2; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(mask(), top, o, L));
        total = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            p[j] = takes_part() ? expf(v[j] - top) : 0.0f;
            if (!sound() && lane + j * L < experts) p[j] = NAN;
            total += p[j];
        }
        total = sum(total);
    }
};

// Probabilities' sums and choices of a block: probs[block][experts],
// choices[block][experts + 1].
template <class T, int L, int N>
__global__ void __launch_bounds__(kThreads)
    router_kernel(const __grid_constant__ heddle_router_args a, float* probs, int32_t* choices) {
    allow_dependents();
    await_previous();
    constexpr int kGroups = kThreads / L;
    __shared__ float psum[kGroups][L * N];
    __shared__ int32_t csum[L * N + 1];
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const uint32_t mask = Token<T, L, N>::mask();
    float sums[N] = {};
    int32_t chose[N] = {}, tokens = 0;
    for (int i = threadIdx.x; i <= L * N; i += kThreads) csum[i] = 0;
    for (int64_t t = (int64_t)blockIdx.x * kGroups + group; t < a.tokens; t += (int64_t)gridDim.x * kGroups) {
        Token<T, L, N> k;
        float v[N];
        k.read(static_cast<const T*>(a.logits) + t * a.ldl, a.experts, !a.valid || a.valid[t], v);
        const bool some = k.takes_part(), sound = k.sound();
        tokens += some;
        const float inv = some ? 1.0f / k.total : 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) sums[j] += k.p[j] * inv;
        // the chosen ones: lane j % L keeps the j-th
        constexpr int kRounds = kMostChosen / L;
        uint32_t taken = 0;
        float mine_p[kRounds] = {}, chosen = 0.0f;
        int mine[kRounds];
#pragma unroll
        for (int q = 0; q < kRounds; ++q) {
            mine[q] = -1;
            for (int j = 0; j < L && q * L + j < a.top_k; ++j) {
                float best = -INFINITY, best_p = 0.0f;
                int at = INT32_MAX;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (!(taken >> i & 1) && v[i] > best) best = v[i], at = lane + i * L, best_p = k.p[i];
#pragma unroll
                for (int o = L / 2; o; o >>= 1) {
                    const float b = __shfl_xor_sync(mask, best, o, L), bp = __shfl_xor_sync(mask, best_p, o, L);
                    const int i = __shfl_xor_sync(mask, at, o, L);
                    if (b > best || (b == best && i < at)) best = b, at = i, best_p = bp;
                }
                if (!some || !sound || at == INT32_MAX) at = -1, best_p = 0.0f;
                chosen += best_p;
                if (at >= 0 && at % L == lane) {
                    taken |= 1u << (at / L);
#pragma unroll
                    for (int i = 0; i < N; ++i) chose[i] += i == at / L;
                }
                if (j == lane) mine[q] = at, mine_p[q] = best_p;
            }
        }
        const float over = !a.normalize ? inv : chosen > 0.0f ? 1.0f / chosen : 0.0f;
#pragma unroll
        for (int q = 0; q < kRounds; ++q) {
            if (q * L + lane >= a.top_k) break;
            a.expert[t * a.top_k + q * L + lane] = mine[q];
            a.weight[t * a.top_k + q * L + lane] = some && !sound ? NAN : mine_p[q] * over;
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) psum[group][lane + j * L] = sums[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (chose[j]) atomicAdd(&csum[lane + j * L], chose[j]);  // whole numbers
    if (lane == 0 && tokens) atomicAdd(&csum[L * N], tokens);
    __syncthreads();
    for (int i = threadIdx.x; i < a.experts; i += kThreads) {
        float s = 0.0f;
        for (int g = 0; g < kGroups; ++g) s += psum[g][i];
        probs[(int64_t)blockIdx.x * a.experts + i] = s;
        choices[(int64_t)blockIdx.x * (a.experts + 1) + i] = csum[i];
    }
    if (threadIdx.x == 0) choices[(int64_t)blockIdx.x * (a.experts + 1) + a.experts] = csum[L * N];
}

// One block: counts and loss from the blocks' sums.
__global__ void __launch_bounds__(1024)
    router_join_kernel(const __grid_constant__ heddle_router_args a, const float* probs, const int32_t* choices,
                       int blocks) {
    allow_dependents();
    await_previous();
    __shared__ float part[32];
    const int E = a.experts;
    float loss = 0.0f;
    for (int e = threadIdx.x; e <= E; e += 1024) {
        int32_t c = 0;
        float p = 0.0f;
        for (int b = 0; b < blocks; ++b) {
            c += choices[(int64_t)b * (E + 1) + e];
            if (e < E) p += probs[(int64_t)b * E + e];
        }
        a.count[e] = c;
        if (e < E) loss += (float)c * p;
    }
    loss = warp_sum(loss);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = loss;
    __syncthreads();
    if (threadIdx.x < 32 && a.loss) {
        loss = warp_sum(part[threadIdx.x]);
        int32_t n = 0;
        for (int b = 0; b < blocks; ++b) n += choices[(int64_t)b * (E + 1) + E];
        if (threadIdx.x == 0) *a.loss = n ? loss * ((float)E / (float)a.top_k) / (float)n / (float)n : 0.0f;
    }
}

template <class T, int L, int N>
__global__ void __launch_bounds__(kThreads)
    router_grad_kernel(const __grid_constant__ heddle_router_grad_args g) {
    allow_dependents();
    await_previous();
    const heddle_router_args& a = g.fwd;
    constexpr int kGroups = kThreads / L;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    float even[N];  // the loss's part of dp
    {
        const float n = (float)a.count[a.experts], d = g.d_loss ? *g.d_loss : 0.0f;
        const float per = n > 0.0f ? d * ((float)a.experts / (float)a.top_k) / n / n : 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j)
            even[j] = g.d_loss && lane + j * L < a.experts ? per * (float)a.count[lane + j * L] : 0.0f;
    }
    for (int64_t t = (int64_t)blockIdx.x * kGroups + group; t < a.tokens; t += (int64_t)gridDim.x * kGroups) {
        Token<T, L, N> k;
        float v[N];
        k.read(static_cast<const T*>(a.logits) + t * a.ldl, a.experts, !a.valid || a.valid[t], v);
        const bool some = k.takes_part();
        const float inv = some ? 1.0f / k.total : 0.0f;
        float dp[N];
#pragma unroll
        for (int j = 0; j < N; ++j) dp[j] = even[j], k.p[j] *= inv;
        if (g.d_weight && some) {
            float mean = 0.0f, over = 1.0f;
            if (a.normalize) {  // of the chosen ones: their gradients' mean, their probabilities' sum
                over = 0.0f;
                for (int j = 0; j < a.top_k; ++j) {
                    const int64_t at = t * a.top_k + j;
                    const int e = a.expert[at];
                    mean = fmaf(g.d_weight[at], a.weight[at], mean);
#pragma unroll
                    for (int i = 0; i < N; ++i) over += e == lane + i * L ? k.p[i] : 0.0f;
                }
                over = Token<T, L, N>::sum(over);
                over = over > 0.0f ? 1.0f / over : 0.0f;
            }
            for (int j = 0; j < a.top_k; ++j) {
                const int64_t at = t * a.top_k + j;
                const int e = a.expert[at];
                const float d = (g.d_weight[at] - mean) * over;
#pragma unroll
                for (int i = 0; i < N; ++i) dp[i] += e == lane + i * L ? d : 0.0f;
            }
        }
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) s = fmaf(k.p[j], dp[j], s);
        s = Token<T, L, N>::sum(s);
        T* out = static_cast<T*>(g.dlogits) + t * g.ldd;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (lane + j * L < a.experts) out[lane + j * L] = from_float<T>(some ? k.p[j] * (dp[j] - s) : 0.0f);
    }
}

// Lanes a token, and its experts a lane.
struct Split {
    int lanes, each;
};
Split split_of(int experts) {
    if (experts <= 64) return {8, 8};
    return {32, experts <= 128 ? 4 : experts <= 256 ? 8 : experts <= 512 ? 16 : 32};
}

int64_t blocks_of(const OpContext& x, const heddle_router_args& a) {
    const int64_t want = ceil_div(a.tokens, kThreads / split_of(a.experts).lanes), most = (int64_t)x.num_sms * 2;
    return want < most ? want : most;
}

template <class T, class F>
cudaError_t with_split(int experts, F f) {
    const Split s = split_of(experts);
    if (s.lanes == 8) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 8>());
    if (s.each == 4) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 4>());
    if (s.each == 8) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
    if (s.each == 16) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>(), std::integral_constant<int, 32>());
}

template <class T>
cudaError_t forward(const OpContext& x, const heddle_router_args& a, unsigned char* ws, cudaStream_t st) {
    const int64_t blocks = blocks_of(x, a);
    float* probs = reinterpret_cast<float*>(ws);
    int32_t* choices = reinterpret_cast<int32_t*>(ws + align256(sizeof(float) * blocks * a.experts));
    cudaError_t e = cudaSuccess;
    if (blocks)
        e = with_split<T>(a.experts, [&](auto l, auto n) {
            return launch(x, router_kernel<T, l.value, n.value>, dim3((unsigned)blocks), kThreads, 0, st, a, probs,
                          choices);
        });
    if (e == cudaSuccess)
        e = launch(x, router_join_kernel, dim3(1), 1024, 0, st, a, (const float*)probs, (const int32_t*)choices,
                   (int)blocks);
    return e;
}

template <class T>
cudaError_t backward(const OpContext& x, const heddle_router_grad_args& g, cudaStream_t st) {
    return with_split<T>(g.fwd.experts, [&](auto l, auto n) {
        return launch(x, router_grad_kernel<T, l.value, n.value>, dim3((unsigned)blocks_of(x, g.fwd)), kThreads, 0, st,
                      g);
    });
}

}  // namespace

size_t router_scratch(const OpContext& x, const heddle_router_args& a) {
    const size_t blocks = (size_t)blocks_of(x, a);
    return align256(sizeof(float) * blocks * a.experts) + align256(sizeof(int32_t) * blocks * (a.experts + 1));
}

cudaError_t launch_router(const OpContext& x, const heddle_router_args& a, unsigned char* ws, cudaStream_t st) {
    if (a.dtype == HEDDLE_BF16) return forward<__nv_bfloat16>(x, a, ws, st);
    if (a.dtype == HEDDLE_FP16) return forward<__half>(x, a, ws, st);
    return forward<float>(x, a, ws, st);
}

cudaError_t launch_router_grad(const OpContext& x, const heddle_router_grad_args& g, cudaStream_t st) {
    if (g.fwd.dtype == HEDDLE_BF16) return backward<__nv_bfloat16>(x, g, st);
    if (g.fwd.dtype == HEDDLE_FP16) return backward<__half>(x, g, st);
    return backward<float>(x, g, st);
}

}  // namespace hd
