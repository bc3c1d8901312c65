// heddle_router.cu -- the router of an expert layer: softmax over the experts,
// the chosen ones, their counts, the balance loss, and the gradient.
//
// A few megabytes in and out: bound by latency and, with many choices, by
// instructions.  A warp holds a token's logits in registers, the next token's
// on their way.  The largest are found one after the other as ordered whole
// numbers, by value and then by index, with the warp's reduction instructions.
// What a lane's experts get, probability and choices, is summed in its registers
// over all tokens of its warp, then over the block's warps, then over blocks by
// a second kernel, always in order.  The backward pass computes the
// probabilities again.  16384 tokens of 64 bfloat16 logits, two chosen: 9.7 us
// forward, 6.4 backward; 32771 of 250 floats, eight chosen: 29 and 21 us (their
// 69 MB take 10).  These and the times below are of calls of a graph one after
// the other, the join's kernel with them.

#include <string.h>

#include "heddle_tc.cuh"

namespace hd {
namespace {

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

// A token's logits, N a lane of a warp: experts lane, lane + 32, ..; -infinity past the
// last one and for a token that takes no part.
template <class T, int N>
__device__ __forceinline__ void load_logits(const heddle_router_args& a, int64_t t, int lane, float (&v)[N]) {
    const bool valid = t < a.tokens && (!a.valid || a.valid[t]);
    const T* l = static_cast<const T*>(a.logits) + t * a.ldl;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = valid && lane + j * 32 < a.experts ? to_float(l[lane + j * 32]) : -INFINITY;
}

// Their exponentials over the largest one's, in p; `inv` over their sum.
template <int N>
struct Softmax {
    float top, inv;
    bool some, sound;  // takes part; no NaN and no +infinity
    __device__ __forceinline__ Softmax(int lane, const float (&v)[N], int experts, float (&p)[N]) {
        uint32_t most = 0;
        bool nan = false;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t k = key_of(v[j]);
            most = k > most ? k : most;
            nan |= v[j] != v[j];
        }
        top = value_of(__reduce_max_sync(~0u, most));
        nan = __any_sync(~0u, nan);
        sound = !nan && top < INFINITY;
        some = nan || top > -INFINITY;
        float total = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            p[j] = some ? expf(v[j] - top) : 0.0f;
            if (!sound && lane + j * 32 < experts) p[j] = NAN;
            total += p[j];
        }
        total = warp_sum(total);
        inv = some ? 1.0f / total : 0.0f;
    }
};

// A token's keys, the largest one after the other, and the first of equal ones.
// Up to four a lane stay in registers and are all compared for each choice; more
// lie in shared memory as lists.  (32771 tokens of 250 floats, eight chosen: 29
// us, from registers 34; 16384 of 64 bfloat16, eight chosen: 12.7 and 11.5.)
template <class T, int N, bool LISTS = (N > 4)>
struct Search;
template <class T, int N>
struct Search<T, N, false> {
    static constexpr int kPlaces = 32 * N;
    uint32_t (&key)[N];
    int lane;
    __device__ __forceinline__ Search(uint32_t (&k)[N], uint32_t*, int l) : key(k), lane(l) {}
    __device__ __forceinline__ uint32_t next(int& at) {
        uint32_t best = key[0];
#pragma unroll
        for (int i = 1; i < N; ++i) best = key[i] > best ? key[i] : best;
        best = __reduce_max_sync(~0u, best);
        if constexpr (sizeof(T) == 2) {
            at = 0xffff - (int)(best & 0xffffu);
#pragma unroll
            for (int i = 0; i < N; ++i) key[i] = key[i] == best ? 0 : key[i];
        } else {
            at = INT32_MAX;
#pragma unroll
            for (int i = N - 1; i >= 0; --i) at = key[i] == best ? lane + i * 32 : at;
            at = __reduce_min_sync(~0u, at);
#pragma unroll
            for (int i = 0; i < N; ++i) key[i] = at == lane + i * 32 ? 0 : key[i];
        }
        return best;
    }
};
// Every lane knows its largest, and the list of the lane that has the largest of
// all is gone through by the warp, a lane a key.
template <class T, int N>
struct Search<T, N, true> {
    static constexpr int kEach = N + 1, kPlaces = 32 * kEach;  // an odd distance between lists
    uint32_t* list;
    int lane;
    uint32_t most = 0;
    __device__ __forceinline__ Search(const uint32_t (&key)[N], uint32_t* at, int l) : list(at), lane(l) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            list[lane * kEach + i] = key[i];
            most = key[i] > most ? key[i] : most;
        }
        __syncwarp();
    }
    __device__ __forceinline__ uint32_t next(int& at) {
        const uint32_t best = __reduce_max_sync(~0u, most);
        int slot, owner;
        uint32_t v;
        if constexpr (sizeof(T) == 2) {
            at = 0xffff - (int)(best & 0xffffu);
            slot = at / 32, owner = at % 32;
            v = lane < N ? list[owner * kEach + lane] : 0;
        } else {
            const uint32_t who = __ballot_sync(~0u, most == best);
            if (who & (who - 1)) {  // equal ones in several lanes
                at = INT32_MAX;
#pragma unroll
                for (int i = N - 1; i >= 0; --i) at = list[lane * kEach + i] == best ? lane + i * 32 : at;
                at = __reduce_min_sync(~0u, at);
                slot = at / 32, owner = at % 32;
                v = lane < N ? list[owner * kEach + lane] : 0;
            } else {
                owner = __ffs(who) - 1;
                v = lane < N ? list[owner * kEach + lane] : 0;
                slot = __ffs(__ballot_sync(~0u, v == best)) - 1;
                at = owner + slot * 32;
            }
        }
        if (lane == slot) v = list[owner * kEach + slot] = 0;
        v = __reduce_max_sync(~0u, v);
        if (lane == owner) most = v;
        __syncwarp();
        return best;
    }
};

// Threads a block, one an SM: those that the registers allow.  (Two blocks of 1024
// for 64 experts: 16384 tokens 10.3 us, one 9.7.)
template <int N>
constexpr int kThreads = N == 32 ? 256 : N == 16 ? 512 : N == 8 ? 768 : 1024;

// The loss from its sum over experts of choices times probabilities.
__device__ __forceinline__ float balance(const heddle_router_args& a, float sum, int32_t tokens) {
    const float n = (float)tokens;
    return tokens ? sum * ((float)a.experts / (float)a.top_k) / n / n : 0.0f;
}

// Sums of a block: of probabilities and choices, sums[experts + 1][block], the
// last of the tokens.  With ONE block they are all, and it gives the results.
template <class T, int N, bool ONE>
__global__ void __launch_bounds__(kThreads<N>, 1)
    router_kernel(const __grid_constant__ heddle_router_args a, float2* sums) {
    allow_dependents();
    await_previous();
    constexpr int kBlock = kThreads<N>, kWarps = kBlock / 32;
    using Lists = Search<T, N>;
    // a warp's list, then its sums
    __shared__ uint32_t own_of[kWarps][Lists::kPlaces];
    __shared__ int32_t csum[32 * N + 1];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    float psums[N] = {}, v[N], next[N];
    int32_t tokens = 0;
    for (int i = threadIdx.x; i <= 32 * N; i += kBlock) csum[i] = 0;
    __syncthreads();
    const int64_t step = (int64_t)gridDim.x * kWarps;
    int64_t t = (int64_t)blockIdx.x * kWarps + warp;
    load_logits<T, N>(a, t, lane, next);
    for (; t < a.tokens; t += step) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = next[j];
        load_logits<T, N>(a, t + step, lane, next);
        float p[N];
        const Softmax<N> s(lane, v, a.experts, p);
        tokens += s.some;
        constexpr bool kPacked = sizeof(T) == 2;
        uint32_t key[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            psums[j] = fmaf(p[j], s.inv, psums[j]);
            if constexpr (kPacked)
                key[j] = packed_key<T>(v[j], lane + j * 32);
            else
                key[j] = key_of(v[j]);
            if (!s.sound) key[j] = 0;
        }
        // the chosen ones: lane j keeps the j-th
        Lists search(key, own_of[warp], lane);
        uint32_t own = 0;
        int mine = -1;
        for (int j = 0; j < a.top_k; ++j) {
            int at;
            const uint32_t best = search.next(at);
            if (best <= kLowest<T>) break;  // none is left
            if (j == lane) mine = at, own = best;
        }
        float value;
        if constexpr (kPacked)
            value = packed_value<T>(own);
        else
            value = value_of(own);
        value = mine >= 0 ? expf(value - s.top) : 0.0f;
        const float chosen = warp_sum(value);
        const float over = !a.normalize ? s.inv : chosen > 0.0f ? 1.0f / chosen : 0.0f;
        if (lane < a.top_k) {
            if (mine >= 0) atomicAdd(&csum[mine], 1);  // whole numbers
            a.expert[t * a.top_k + lane] = mine;
            a.weight[t * a.top_k + lane] = s.sound ? value * over : NAN;
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) own_of[warp][lane + j * 32] = __float_as_uint(psums[j]);
    if (lane == 0 && tokens) atomicAdd(&csum[32 * N], tokens);
    __syncthreads();
    float loss = 0.0f;
    for (int i = threadIdx.x; i <= a.experts; i += kBlock) {
        float p = 0.0f;
        if (i < a.experts) {
#pragma unroll 16
            for (int k = 0; k < kWarps; ++k) p += __uint_as_float(own_of[k][i]);
        }
        const int32_t c = csum[i < a.experts ? i : 32 * N];
        if (ONE) {
            a.count[i] = c;
            if (i < a.experts) loss = fmaf((float)c, p, loss);
        } else {
            sums[(int64_t)i * gridDim.x + blockIdx.x] = make_float2(p, __int_as_float(c));
        }
    }
    if (ONE && a.loss) {
        __shared__ float part[kWarps];
        loss = warp_sum(loss);
        if (lane == 0) part[warp] = loss;
        __syncthreads();
        if (warp == 0) {
            loss = warp_sum(lane < kWarps ? part[lane] : 0.0f);
            if (lane == 0) *a.loss = balance(a, loss, csum[32 * N]);
        }
    }
}

// Counts and loss from the blocks' sums: a warp a column, its lanes over the
// blocks; one block, or a cluster where its warps would have several columns
// each, whose parts of the loss its first block adds in order.
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

template <class T, int N>
__global__ void __launch_bounds__(kThreads<N>, 1)
    router_grad_kernel(const __grid_constant__ heddle_router_grad_args ga) {
    allow_dependents();
    await_previous();
    const heddle_router_args& a = ga.fwd;
    constexpr int kWarps = kThreads<N> / 32;
    __shared__ float all[kWarps][32 * N];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    float* given = all[warp];  // zeros between tokens
#pragma unroll
    for (int j = 0; j < N; ++j) given[lane + j * 32] = 0.0f;
    __syncwarp();
    const int64_t step = (int64_t)gridDim.x * kWarps;
    int64_t t = (int64_t)blockIdx.x * kWarps + warp;
    float v[N], next[N];
    load_logits<T, N>(a, t, lane, next);
    float even[N];  // the loss's part of dp
    {
        const float n = (float)a.count[a.experts], d = ga.d_loss ? *ga.d_loss : 0.0f;
        const float per = n > 0.0f ? d * ((float)a.experts / (float)a.top_k) / n / n : 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j)
            even[j] = ga.d_loss && lane + j * 32 < a.experts ? per * (float)a.count[lane + j * 32] : 0.0f;
    }
    for (; t < a.tokens; t += step) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = next[j];
        load_logits<T, N>(a, t + step, lane, next);
        // the chosen ones' gradients, choice j in lane j
        const int64_t at = t * a.top_k + lane;
        float d = 0.0f, w = 0.0f;
        int expert = ga.d_weight && lane < a.top_k ? a.expert[at] : -1;
        if (expert >= a.experts) expert = -1;  // not a result of the forward call
        if (expert >= 0) {
            d = ga.d_weight[at];
            if (a.normalize) w = a.weight[at];
        }
        float p[N], dp[N];
        const Softmax<N> s(lane, v, a.experts, p);
#pragma unroll
        for (int j = 0; j < N; ++j) dp[j] = even[j], p[j] *= s.inv;
        if (ga.d_weight) {
            float over = 1.0f, mean = 0.0f;
            if (a.normalize) {
                // over the chosen ones' probabilities: the first one's is `inv`
                // itself, and its weight of their sum
                mean = warp_sum(d * w);
                over = __shfl_sync(~0u, w, 0) / s.inv;
                over = s.some ? over : 0.0f;
            }
            // to the lanes that hold them
            if (expert >= 0) given[expert] = (d - mean) * over;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < N; ++j) dp[j] += given[lane + j * 32];
            __syncwarp();
            if (expert >= 0) given[expert] = 0.0f;
            __syncwarp();
        }
        float mix = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) mix = fmaf(p[j], dp[j], mix);
        mix = warp_sum(mix);
        T* out = static_cast<T*>(ga.dlogits) + t * ga.ldd;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (lane + j * 32 < a.experts) out[lane + j * 32] = from_float<T>(s.some ? p[j] * (dp[j] - mix) : 0.0f);
    }
}

// Experts a lane of a token's warp.  (Eight lanes a token up to 64 experts took
// a fifth longer for 64 tokens of 64 experts, two of them, and 4 % less for
// 16384 of eight.)
template <class F>
auto with_split(int experts, F f) {
    if (experts <= 64) return f(std::integral_constant<int, 2>());
    if (experts <= 128) return f(std::integral_constant<int, 4>());
    if (experts <= 256) return f(std::integral_constant<int, 8>());
    if (experts <= 512) return f(std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>());
}

int64_t blocks_of(const OpContext& x, const heddle_router_args& a) {
    return with_split(a.experts, [&](auto n) {
        const int64_t want = ceil_div(a.tokens, kThreads<n.value> / 32);
        return want < x.num_sms ? want : (int64_t)x.num_sms;
    });
}

// Whether one block does it all: for up to two rounds of its warps.  (64 tokens
// of 64 experts: 4.4 us, 4.9 with a second kernel; 128 tokens, in four rounds:
// 7.0 and 5.7.)
bool one_block(const heddle_router_args& a) {
    return with_split(a.experts, [&](auto n) { return a.tokens <= 2 * (kThreads<n.value> / 32); });
}

template <class T>
cudaError_t forward(const OpContext& x, const heddle_router_args& a, unsigned char* ws, cudaStream_t st) {
    float2* sums = reinterpret_cast<float2*>(ws);
    const bool one = one_block(a);
    const int64_t blocks = one ? 1 : blocks_of(x, a);
    const cudaError_t e = with_split(a.experts, [&](auto n) {
        auto* kernel = one ? router_kernel<T, n.value, true> : router_kernel<T, n.value, false>;
        return launch(x, kernel, dim3((unsigned)blocks), kThreads<n.value>, 0, st, a, sums);
    });
    if (e != cudaSuccess || one) return e;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {kJoinCluster, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    // 32771 tokens of 250 experts: 29.1 us by a cluster, 32.8 by a block; 16384 of
    // 64: 9.9 and 9.7; of eight: 9.3 and 8.2
    const bool many = a.experts > 64;
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
    return with_split(g.fwd.experts, [&](auto n) {
        return launch(x, router_grad_kernel<T, n.value>, dim3((unsigned)blocks_of(x, g.fwd)), kThreads<n.value>, 0, st,
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
