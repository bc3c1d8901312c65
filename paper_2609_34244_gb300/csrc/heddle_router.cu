// heddle_router.cu -- the router of an expert layer: softmax over the experts,
// the chosen ones, their counts, the balance loss, and the gradient.
//
// A few megabytes in and out: bound by latency and, with many choices, by
// instructions.  A group of lanes holds a token's logits in registers, the next
// token's on their way.  The largest are found one after the other as ordered
// whole numbers, by value and then by index, whole warps with their reduction
// instructions.  What a lane's experts get, probability and choices, is summed
// in its registers over all tokens of its group, then over the block's groups,
// then over blocks by a second kernel, always in order.  The backward pass
// computes the probabilities again.

#include <string.h>

#include "heddle_tc.cuh"

namespace hd {
namespace {

constexpr int kMostChosen = 32;

// Whole numbers in the order of the floats; equal for both zeros, and none is 0.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ ((uint32_t)((int32_t)~key >> 31) | 0x80000000u));
}
// Those of 16-bit floats, in the upper half, with the expert's complement below:
// the first of equal ones is the largest, and one reduction finds value and expert.
template <class T>
__device__ __forceinline__ uint32_t packed_key(float v, int expert) {
    uint16_t u;
    const T t = from_float<T>(v + 0.0f);
    memcpy(&u, &t, 2);
    const uint32_t k = u & 0x8000u ? ~(uint32_t)u & 0xffffu : u | 0x8000u;
    return k << 16 | (0xffffu - expert);
}
template <class T>
__device__ __forceinline__ float packed_value(uint32_t key) {
    const uint32_t k = key >> 16;
    const uint16_t u = (uint16_t)(k & 0x8000u ? k & 0x7fffu : ~k);
    T t;
    memcpy(&t, &u, 2);
    return to_float(t);
}
// The largest key of -infinity.
template <class T>
constexpr uint32_t kLowest = 0x007fffffu;
template <>
constexpr uint32_t kLowest<__half> = 0x03ffffffu;

// L lanes of a warp.
template <int L>
struct Group {
    uint32_t mask;
    int lane;
    __device__ __forceinline__ Group()
        : mask(L == 32 ? ~0u : ((1u << (L & 31)) - 1) << (threadIdx.x % 32 / L * L)), lane(threadIdx.x % L) {}
    __device__ __forceinline__ uint32_t largest(uint32_t v) const {
        if constexpr (L == 32) {
            return __reduce_max_sync(~0u, v);
        } else {
#pragma unroll
            for (int o = L / 2; o; o >>= 1) {
                const uint32_t w = __shfl_xor_sync(mask, v, o, L);
                v = w > v ? w : v;
            }
            return v;
        }
    }
    __device__ __forceinline__ int least(int v) const {
        if constexpr (L == 32) {
            return __reduce_min_sync(~0u, v);
        } else {
#pragma unroll
            for (int o = L / 2; o; o >>= 1) {
                const int w = __shfl_xor_sync(mask, v, o, L);
                v = w < v ? w : v;
            }
            return v;
        }
    }
    __device__ __forceinline__ float sum(float v) const {
#pragma unroll
        for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(mask, v, o, L);
        return v;
    }
    __device__ __forceinline__ bool any(bool v) const { return __ballot_sync(mask, v) & mask; }
};

// A token's logits, N a lane: experts lane, lane + L, ..; -infinity past the
// last one and for a token that takes no part.
template <class T, int L, int N>
__device__ __forceinline__ void load_logits(const heddle_router_args& a, int64_t t, int lane, float (&v)[N]) {
    const bool valid = t < a.tokens && (!a.valid || a.valid[t]);
    const T* l = static_cast<const T*>(a.logits) + t * a.ldl;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = valid && lane + j * L < a.experts ? to_float(l[lane + j * L]) : -INFINITY;
}

// Their exponentials over the largest one's, in p; `inv` over their sum.
template <int L, int N>
struct Softmax {
    float top, inv;
    bool some, sound;  // takes part; no NaN and no +infinity
    __device__ __forceinline__ Softmax(const Group<L>& g, const float (&v)[N], int experts, float (&p)[N]) {
        uint32_t most = 0;
        bool nan = false;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t k = key_of(v[j]);
            most = k > most ? k : most;
            nan |= v[j] != v[j];
        }
        top = value_of(g.largest(most));
        nan = g.any(nan);
        sound = !nan && top < INFINITY;
        some = nan || top > -INFINITY;
        float total = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            p[j] = some ? expf(v[j] - top) : 0.0f;
            if (!sound && g.lane + j * L < experts) p[j] = NAN;
            total += p[j];
        }
        total = g.sum(total);
        inv = some ? 1.0f / total : 0.0f;
    }
};

// Threads a block: those that the registers allow.
template <int L, int N>
constexpr int kThreads = N > 8 || L == 8 ? 256 : N == 8 ? 768 : 1024;
template <int L, int N>
constexpr int kResident = L == 8 ? 4 : 1;  // blocks an SM

// The loss from its sum over experts of choices times probabilities.
__device__ __forceinline__ float balance(const heddle_router_args& a, float sum, int32_t tokens) {
    const float n = (float)tokens;
    return tokens ? sum * ((float)a.experts / (float)a.top_k) / n / n : 0.0f;
}

// Sums of a block: of probabilities and choices, sums[experts + 1][block], the
// last of the tokens.  With ONE block they are all, and it gives the results: a
// second kernel would cost a few tokens as much as the first.
template <class T, int L, int N, bool ONE>
__global__ void __launch_bounds__(kThreads<L, N>, kResident<L, N>)
    router_kernel(const __grid_constant__ heddle_router_args a, float2* sums) {
    allow_dependents();
    await_previous();
    constexpr int kBlock = kThreads<L, N>, kGroups = kBlock / L, kRounds = kMostChosen / L;
    __shared__ float psum[kBlock / 32][L * N];
    __shared__ int32_t csum[L * N + 1];
    const Group<L> g;
    const int lane = g.lane;
    float psums[N] = {}, v[N], next[N];
    int32_t tokens = 0;
    for (int i = threadIdx.x; i <= L * N; i += kBlock) csum[i] = 0;
    __syncthreads();
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t t = (int64_t)blockIdx.x * kGroups + threadIdx.x / L;
    load_logits<T, L, N>(a, t, lane, next);
    for (; t < a.tokens; t += step) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = next[j];
        load_logits<T, L, N>(a, t + step, lane, next);
        float p[N];
        const Softmax<L, N> s(g, v, a.experts, p);
        tokens += s.some;
        constexpr bool kPacked = sizeof(T) == 2;
        uint32_t key[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            psums[j] = fmaf(p[j], s.inv, psums[j]);
            if constexpr (kPacked)
                key[j] = packed_key<T>(v[j], lane + j * L);
            else
                key[j] = key_of(v[j]);
            if (!s.sound) key[j] = 0;
        }
        // the chosen ones: lane j % L keeps the j-th
        float value[kRounds] = {}, chosen = 0.0f;
        int mine[kRounds];
#pragma unroll
        for (int q = 0; q < kRounds; ++q) {
            mine[q] = -1;
            for (int j = 0; j < L && q * L + j < a.top_k; ++j) {
                uint32_t best = key[0];
#pragma unroll
                for (int i = 1; i < N; ++i) best = key[i] > best ? key[i] : best;
                best = g.largest(best);
                if (best <= kLowest<T>) break;  // none is left
                int at;
                if constexpr (kPacked) {
                    at = 0xffff - (int)(best & 0xffffu);
#pragma unroll
                    for (int i = 0; i < N; ++i) key[i] = key[i] == best ? 0 : key[i];
                } else {
                    at = INT32_MAX;
#pragma unroll
                    for (int i = N - 1; i >= 0; --i) at = key[i] == best ? lane + i * L : at;
                    at = g.least(at);
#pragma unroll
                    for (int i = 0; i < N; ++i) key[i] = at == lane + i * L ? 0 : key[i];
                }
                if (j == lane) mine[q] = at, value[q] = __uint_as_float(best);
            }
        }
#pragma unroll
        for (int q = 0; q < kRounds; ++q) {
            const uint32_t key_q = __float_as_uint(value[q]);
            float v_q;
            if constexpr (kPacked)
                v_q = packed_value<T>(key_q);
            else
                v_q = value_of(key_q);
            value[q] = mine[q] >= 0 ? expf(v_q - s.top) : 0.0f;
            chosen += value[q];
        }
        chosen = g.sum(chosen);
        const float over = !a.normalize ? s.inv : chosen > 0.0f ? 1.0f / chosen : 0.0f;
#pragma unroll
        for (int q = 0; q < kRounds; ++q) {
            if (q * L + lane >= a.top_k) break;
            if (mine[q] >= 0) atomicAdd(&csum[mine[q]], 1);  // whole numbers
            a.expert[t * a.top_k + q * L + lane] = mine[q];
            a.weight[t * a.top_k + q * L + lane] = s.sound ? value[q] * over : NAN;
        }
    }
    // a warp's groups, then the block's warps
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
        for (int o = L; o < 32; o <<= 1) psums[j] += __shfl_xor_sync(~0u, psums[j], o);
        if (threadIdx.x % 32 < L) psum[threadIdx.x / 32][lane + j * L] = psums[j];
    }
    if (lane == 0 && tokens) atomicAdd(&csum[L * N], tokens);
    __syncthreads();
    float loss = 0.0f;
    for (int i = threadIdx.x; i <= a.experts; i += kBlock) {
        float p = 0.0f;
        if (i < a.experts) {
#pragma unroll 16
            for (int k = 0; k < kBlock / 32; ++k) p += psum[k][i];
        }
        const int32_t c = csum[i < a.experts ? i : L * N];
        if (ONE) {
            a.count[i] = c;
            if (i < a.experts) loss = fmaf((float)c, p, loss);
        } else {
            sums[(int64_t)i * gridDim.x + blockIdx.x] = make_float2(p, __int_as_float(c));
        }
    }
    if (ONE && a.loss) {
        __shared__ float part[kBlock / 32];
        loss = warp_sum(loss);
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = loss;
        __syncthreads();
        if (threadIdx.x < 32) {
            loss = warp_sum(threadIdx.x < kBlock / 32 ? part[threadIdx.x] : 0.0f);
            if (threadIdx.x == 0) *a.loss = balance(a, loss, csum[L * N]);
        }
    }
}

// Counts and loss from the blocks' sums: a warp a column, its lanes over the
// blocks; one block, or a cluster where there is much to read, whose parts of
// the loss its first block adds in order.
constexpr int kJoin = 1024, kJoinCluster = 8;
constexpr int kAtOnce = 8;  // loads that are waited for together
__global__ void __launch_bounds__(kJoin)
    router_join_kernel(const __grid_constant__ heddle_router_args a, const float2* sums, int blocks) {
    allow_dependents();
    await_previous();
    __shared__ float part[kJoin / 32];
    __shared__ float mine;
    __shared__ int32_t tokens;
    const int cols = a.experts + 1, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t rank = gridDim.x > 1 ? tc::cluster_rank() : 0;
    float loss = 0.0f;
    for (int c = rank * (kJoin / 32) + warp; c < cols; c += gridDim.x * (kJoin / 32)) {
        float p = 0.0f;
        int32_t n = 0;
        for (int b0 = lane; b0 < blocks; b0 += 32 * kAtOnce) {
            float2 s[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                s[k] = b0 + 32 * k < blocks ? sums[(int64_t)c * blocks + b0 + 32 * k] : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) p += s[k].x, n += __float_as_int(s[k].y);
        }
        p = warp_sum(p), n = __reduce_add_sync(~0u, n);
        if (lane == 0) a.count[c] = n;
        loss = c < a.experts ? fmaf((float)n, p, loss) : loss;
    }
    if (!a.loss) return;
    if (lane == 0) part[warp] = loss;
    // the tokens' column, again, by the block that ends the sum
    if (rank == 0 && warp == kJoin / 32 - 1) {
        int32_t n = 0;
        for (int b0 = lane; b0 < blocks; b0 += 32 * kAtOnce) {
            float2 s[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                s[k] = b0 + 32 * k < blocks ? sums[(int64_t)a.experts * blocks + b0 + 32 * k] : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) n += __float_as_int(s[k].y);
        }
        n = __reduce_add_sync(~0u, n);
        if (lane == 0) tokens = n;
    }
    __syncthreads();
    if (warp == 0) {
        loss = warp_sum(part[lane]);
        if (lane == 0) mine = loss;
    }
    if (gridDim.x > 1) {
        tc::cluster_sync();
        if (rank == 0 && threadIdx.x == 0) {
            for (uint32_t r = 1; r < gridDim.x; ++r) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];"
                             : "=f"(v)
                             : "r"(tc::cluster_at(tc::smem_u32(&mine), r))
                             : "memory");
                loss += v;
            }
        }
        tc::cluster_sync();  // the others' memory is read
    }
    if (rank == 0 && threadIdx.x == 0) *a.loss = balance(a, loss, tokens);
}

template <class T, int L, int N>
__global__ void __launch_bounds__(kThreads<L, N>, kResident<L, N>)
    router_grad_kernel(const __grid_constant__ heddle_router_grad_args ga) {
    allow_dependents();
    await_previous();
    const heddle_router_args& a = ga.fwd;
    constexpr int kGroups = kThreads<L, N> / L, kRounds = kMostChosen / L;
    __shared__ float all[kGroups][L * N];
    const Group<L> g;
    const int lane = g.lane;
    float* given = all[threadIdx.x / L];  // zeros between tokens
#pragma unroll
    for (int j = 0; j < N; ++j) given[lane + j * L] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t t = (int64_t)blockIdx.x * kGroups + threadIdx.x / L;
    float v[N], next[N];
    load_logits<T, L, N>(a, t, lane, next);
    float even[N];  // the loss's part of dp
    {
        const float n = (float)a.count[a.experts], d = ga.d_loss ? *ga.d_loss : 0.0f;
        const float per = n > 0.0f ? d * ((float)a.experts / (float)a.top_k) / n / n : 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j)
            even[j] = ga.d_loss && lane + j * L < a.experts ? per * (float)a.count[lane + j * L] : 0.0f;
    }
    for (; t < a.tokens; t += step) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = next[j];
        load_logits<T, L, N>(a, t + step, lane, next);
        // the chosen ones' gradients, choice j in lane j % L
        float d[kRounds] = {};
        int expert[kRounds];
        float mean = 0.0f, first = 0.0f;
#pragma unroll
        for (int q = 0; q < kRounds; ++q) {
            expert[q] = -1;
            const int64_t at = t * a.top_k + q * L + lane;
            if (ga.d_weight && q * L + lane < a.top_k) expert[q] = a.expert[at];
            if (expert[q] >= a.experts) expert[q] = -1;  // not a result of the forward call
            if (expert[q] >= 0) {
                d[q] = ga.d_weight[at];
                if (a.normalize) {
                    const float w = a.weight[at];
                    mean = fmaf(d[q], w, mean);
                    if (q == 0) first = w;
                }
            }
        }
        float p[N], dp[N];
        const Softmax<L, N> s(g, v, a.experts, p);
#pragma unroll
        for (int j = 0; j < N; ++j) dp[j] = even[j], p[j] *= s.inv;
        if (ga.d_weight) {
            float over = 1.0f;
            if (a.normalize) {
                // over the chosen ones' probabilities: the first one's is `inv`
                // itself, and `first` of their sum
                mean = g.sum(mean);
                over = __shfl_sync(g.mask, first, 0, L) / s.inv;
                over = s.some ? over : 0.0f;
            }
            // to the lanes that hold them
            __syncwarp(g.mask);
#pragma unroll
            for (int q = 0; q < kRounds; ++q)
                if (expert[q] >= 0) given[expert[q]] = (d[q] - mean) * over;
            __syncwarp(g.mask);
#pragma unroll
            for (int j = 0; j < N; ++j) dp[j] += given[lane + j * L];
            __syncwarp(g.mask);
#pragma unroll
            for (int q = 0; q < kRounds; ++q)
                if (expert[q] >= 0) given[expert[q]] = 0.0f;
        }
        float mix = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) mix = fmaf(p[j], dp[j], mix);
        mix = g.sum(mix);
        T* out = static_cast<T*>(ga.dlogits) + t * ga.ldd;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (lane + j * L < a.experts) out[lane + j * L] = from_float<T>(s.some ? p[j] * (dp[j] - mix) : 0.0f);
    }
}

// Lanes a token, and its experts a lane.
template <class F>
auto with_split(int experts, F f) {
    if (experts <= 64) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 8>());
    if (experts <= 128) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 4>());
    if (experts <= 256) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
    if (experts <= 512) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>(), std::integral_constant<int, 32>());
}

int64_t blocks_of(const OpContext& x, const heddle_router_args& a) {
    return with_split(a.experts, [&](auto l, auto n) {
        constexpr int threads = kThreads<l.value, n.value>;
        const int64_t want = ceil_div(a.tokens, threads / l.value);
        const int64_t most = (int64_t)x.num_sms * kResident<l.value, n.value>;
        return want < most ? want : most;
    });
}

// Whether one block does it all: for up to two rounds of its groups.
bool one_block(const heddle_router_args& a) {
    return with_split(a.experts, [&](auto l, auto n) {
        return a.tokens <= 2 * kThreads<l.value, n.value> / l.value;
    });
}

template <class T>
cudaError_t forward(const OpContext& x, const heddle_router_args& a, unsigned char* ws, cudaStream_t st) {
    float2* sums = reinterpret_cast<float2*>(ws);
    const bool one = one_block(a);
    const int64_t blocks = one ? 1 : blocks_of(x, a);
    const cudaError_t e = with_split(a.experts, [&](auto l, auto n) {
        constexpr int threads = kThreads<l.value, n.value>;
        auto* kernel = one ? router_kernel<T, l.value, n.value, true> : router_kernel<T, l.value, n.value, false>;
        return launch(x, kernel, dim3((unsigned)blocks), threads, 0, st, a, sums);
    });
    if (e != cudaSuccess || one) return e;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {kJoinCluster, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    const bool many = blocks * (a.experts + 1) > 2048;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(many ? kJoinCluster : 1);
    cfg.blockDim = dim3(kJoin);
    cfg.stream = st;
    cfg.attrs = many ? attr : attr + 1;
    cfg.numAttrs = (many ? 1 : 0) + (x.chained ? 1 : 0);
    x.chained = true;
    return cudaLaunchKernelEx(&cfg, router_join_kernel, a, (const float2*)sums, (int)blocks);
}

template <class T>
cudaError_t backward(const OpContext& x, const heddle_router_grad_args& g, cudaStream_t st) {
    return with_split(g.fwd.experts, [&](auto l, auto n) {
        constexpr int threads = kThreads<l.value, n.value>;
        return launch(x, router_grad_kernel<T, l.value, n.value>, dim3((unsigned)blocks_of(x, g.fwd)), threads, 0, st,
                      g);
    });
}

}  // namespace

size_t router_scratch(const OpContext& x, const heddle_router_args& a) {
    return one_block(a) ? 0 : align256(sizeof(float2) * (size_t)blocks_of(x, a) * (a.experts + 1));
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
