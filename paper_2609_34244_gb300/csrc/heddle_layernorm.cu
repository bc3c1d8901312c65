// heddle_layernorm.cu -- layer norm and its gradients.
//
// Bound by memory.  A row is held by a group of threads, a few 16-byte units
// each: its mean first, in two floats, then the squares of its deviations from
// it, so that a large mean costs no digits and nothing is read from memory
// twice.  Short rows take 4 to 32 lanes of a warp, others a block, which walks
// over rows.  Gradients of such rows are read through a ring in shared memory
// that bulk copies fill ahead; the weights' sums over rows stay in registers,
// one set a block, and a second kernel adds the sets in order.  Arithmetic runs
// on two values at a time, and 16-bit values are used as they lie in their
// words: 16384 x 8192 bfloat16 takes 87 us forward (6.2 TB/s) and 168 backward
// (6.4, with the join); taken out one by one they were bound by instructions,
// 149 and 350.

#include <atomic>

#include "heddle_rows.cuh"

namespace hd {
namespace {

// The block's sum, the same in every thread.  `turn` alternates between calls:
// one barrier each.
struct BlockSum {
    float* part;  // [2][32], of a block's shared memory
    int lanes;    // a power of two that has the warps' sums
    int turn = 0;
    __device__ __forceinline__ BlockSum() {
        __shared__ float all[2][32];
        part = all[0];
        const int warps = blockDim.x / 32;
        lanes = 1 << (32 - __clz(warps - 1));
        if (threadIdx.x < 64) part[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    __device__ __forceinline__ float operator()(float v) {
        float* at = part + turn;
        v = warp_sum(v);
        if (threadIdx.x % 32 == 0) at[threadIdx.x / 32] = v;
        __syncthreads();
        v = at[threadIdx.x % lanes];
#pragma unroll
        for (int o = 16; o; o >>= 1)
            if (o < lanes) v += __shfl_xor_sync(~0u, v, o);
        turn ^= 32;
        return v;
    }
};
// Two sums: the lower half of a warp's lanes goes on with the first, the upper
// half with the second.
__device__ __forceinline__ void block_sums(float& v0, float& v1, int& turn) {
    __shared__ float part[2][2][32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32, half = lane / 16;
    float v = (half ? v1 : v0) + __shfl_xor_sync(~0u, half ? v0 : v1, 16);
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if (lane % 16 == 0) part[turn][half][warp] = v;
    __syncthreads();
    const int i = lane % 16;
    v = (i < warps ? part[turn][half][i] : 0.0f) + (i + 16 < warps ? part[turn][half][i + 16] : 0.0f);
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    v0 = __shfl_sync(~0u, v, 0), v1 = __shfl_sync(~0u, v, 16);
    turn ^= 1;
}

// Four sums: a quarter of a warp's lanes for each.
__device__ __forceinline__ void block_sums(float (&v)[4], int& turn) {
    __shared__ float part[2][4][32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
    const bool up = lane & 16, odd = lane & 8;
    const float a = (up ? v[2] : v[0]) + __shfl_xor_sync(~0u, up ? v[0] : v[2], 16),
                b = (up ? v[3] : v[1]) + __shfl_xor_sync(~0u, up ? v[1] : v[3], 16);
    float c = (odd ? b : a) + __shfl_xor_sync(~0u, odd ? a : b, 8);
#pragma unroll
    for (int o = 4; o; o >>= 1) c += __shfl_xor_sync(~0u, c, o);
    if (lane % 8 == 0) part[turn][lane / 8][warp] = c;
    __syncthreads();
    c = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        if (i + lane % 8 < warps) c += part[turn][lane / 8][i + lane % 8];
#pragma unroll
    for (int o = 4; o; o >>= 1) c += __shfl_xor_sync(~0u, c, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __shfl_sync(~0u, c, 8 * i);
    turn ^= 1;
}

// sum / cols in two floats, inv = 1 / cols: the product, corrected by its
// remainder (exact where the quotient is a float: a row of one value has no
// variance), and what then remains.  A division would take a dozen
// instructions of every thread.
struct Mean {
    float value, left;
    __device__ __forceinline__ Mean(float sum, float cols, float inv) {
        const float q = sum * inv;
        value = fmaf(fmaf(-q, cols, sum), inv, q);
        left = fmaf(-value, cols, sum) * inv;
    }
};

// Of GL lanes of a warp, all of which take part.
template <int GL, int N>
__device__ __forceinline__ void lanes_sum(float (&v)[N]) {
#pragma unroll
    for (int o = GL / 2; o; o >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(~0u, v[i], o);
    }
}

// A vector of the row's length in registers, or `none`.
template <class T, class R>
__device__ __forceinline__ void load_vector(const R& part, uint32_t (&w)[R::kWords], const void* p, float none) {
    if (p) {
        part.load(w, static_cast<const T*>(p), (uintptr_t)p % 16 == 0 && part.cols % R::V == 0);
    } else {
#pragma unroll
        for (int i = 0; i < R::N / 2; ++i) set_pair<T>(w, i, both(none));
    }
}

// The sum of a row's values, zeros past its end.
template <class T, class R>
__device__ __forceinline__ float sum_of(const R&, const uint32_t (&r)[R::kWords]) {
    float2 s[2] = {both(0.0f), both(0.0f)};
#pragma unroll
    for (int p = 0; p < R::N / 2; ++p) s[p % 2] = plus<T>(r, p, s[p % 2]);
    s[0] = add2(s[0], s[1]);
    return s[0].x + s[0].y;
}
// Their deviations from the mean's first part, and the sum of these' squares.
// ENDS: the row's end may lie in a unit.
//
// What a mean is off by reaches every y times rstd, and beside large means it is
// not small: its rounding is taken out as its second part, `left`.  Sums of
// 16-bit values around a large mean are exact for thousands of them; those of
// 32 bits are not, so the deviations are added up as well and tell what is left
// (32768 x 2048 floats: 87.3 us, 86.5 without; 8192 x 8192: 98.2 and 94.6; 16384
// x 8192 bfloat16 would take 106 for 87).
template <class T>
constexpr bool kLeft = sizeof(T) == 4;
template <class T, bool ENDS, class R>
__device__ __forceinline__ float2 deviations_of(const R& part, const uint32_t (&r)[R::kWords], float2 (&v)[R::N / 2],
                                                float mean) {
    float2 d = both(0.0f), s = both(0.0f);
    const float2 m = both(-mean);
#pragma unroll
    for (int p = 0; p < R::N / 2; ++p) {
        v[p] = plus<T>(r, p, m);
        if (ENDS) {
            const float2 f = make_float2(part.in(2 * p) ? v[p].x : 0.0f, part.in(2 * p + 1) ? v[p].y : 0.0f);
            if (kLeft<T>) d = add2(d, f);
            s = fma2(f, f, s);
        } else if (part.in(2 * p / R::V * R::V)) {  // a unit is in or out as a whole
            if (kLeft<T>) d = add2(d, v[p]);
            s = fma2(v[p], v[p], s);
        }
    }
    return make_float2(d.x + d.y, s.x + s.y);
}
// What is left of the mean, and 1 / sqrt(variance + eps).
struct Spread {
    float left, rstd;
    // Of the two sums: the variance is the squares' mean less the square of what
    // is left.
    __device__ __forceinline__ Spread(float2 sums, float inv, float eps) : left(sums.x * inv) {
        const float var = fmaf(-left, left, sums.y * inv);
        rstd = inv_sqrt((var < 0.0f ? 0.0f : var) + eps);
    }
    // Of the mean and the squares: half a unit of the mean's last place, whose
    // square is nothing beside a variance of 16-bit values.
    __device__ __forceinline__ Spread(const Mean& mean, float squares, float inv, float eps)
        : left(mean.left), rstd(inv_sqrt(fmaf(squares, inv, eps))) {}
};
template <class T, class S>
__device__ __forceinline__ Spread spread_of(S& total, const Mean& mean, float2 sums, float inv, float eps) {
    if constexpr (kLeft<T>)
        return Spread(total(sums), inv, eps);
    else
        return Spread(mean, total(sums.y), inv, eps);
}

// Weight and bias of a lane as floats in its registers.
template <class T, class R>
struct Held {
    float2 w[R::N / 2], b[R::N / 2];
    __device__ __forceinline__ Held(const R& part, const heddle_layer_norm_args& a, float4*) {
        uint32_t r[R::kWords];
        load_vector<T>(part, r, a.weight, 1.0f);
#pragma unroll
        for (int p = 0; p < R::N / 2; ++p) w[p] = pair_of<T>(r, p);
        load_vector<T>(part, r, a.bias, 0.0f);
#pragma unroll
        for (int p = 0; p < R::N / 2; ++p) b[p] = pair_of<T>(r, p);
    }
    __device__ __forceinline__ void scale(const R&, uint32_t (&out)[R::kWords], const float2 (&v)[R::N / 2],
                                          const Spread& spread) const {
        const float2 s = both(spread.rstd), o = both(-spread.left * spread.rstd);
#pragma unroll
        for (int p = 0; p < R::N / 2; ++p) set_pair<T>(out, p, fma2(fma2(v[p], s, o), w[p], b[p]));
    }
};
// Those of a block as floats in shared memory, each thread its own, four values
// after four: taking 16-bit ones out of their words for every row cost more.
template <class T, class R>
struct Shared {
    const float4 *w, *b;
    int threads;
    __device__ __forceinline__ Shared(const R& part, const heddle_layer_norm_args& a, float4* at)
        : w(at), b(at + blockDim.x * (R::N / 4)), threads(blockDim.x) {
        uint32_t r[R::kWords];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            load_vector<T>(part, r, k ? a.bias : a.weight, k ? 0.0f : 1.0f);
#pragma unroll
            for (int q = 0; q < R::N / 4; ++q) {
                const float2 x = pair_of<T>(r, 2 * q), y = pair_of<T>(r, 2 * q + 1);
                at[(k * (R::N / 4) + q) * threads + threadIdx.x] = make_float4(x.x, x.y, y.x, y.y);
            }
        }
    }
    __device__ __forceinline__ void scale(const R&, uint32_t (&out)[R::kWords], const float2 (&v)[R::N / 2],
                                          const Spread& spread) const {
        const float2 s = both(spread.rstd), o = both(-spread.left * spread.rstd);
#pragma unroll
        for (int q = 0; q < R::N / 4; ++q) {
            const float4 wv = w[q * threads + threadIdx.x], bv = b[q * threads + threadIdx.x];
            set_pair<T>(out, 2 * q, fma2(fma2(v[2 * q], s, o), make_float2(wv.x, wv.y), make_float2(bv.x, bv.y)));
            set_pair<T>(out, 2 * q + 1,
                        fma2(fma2(v[2 * q + 1], s, o), make_float2(wv.z, wv.w), make_float2(bv.z, bv.w)));
        }
    }
};
// 16-bit ones as they lie in their words, beside a ring: taking them out costs
// less than the second block an SM that the floats leave no room for (16384 x
// 8192 bfloat16 one element off 16 bytes: 143 us, floats 209; the same bits).
template <class T, class R>
struct Packed {
    const uint4 *w, *b;
    int threads;
    __device__ __forceinline__ Packed(const R& part, const heddle_layer_norm_args& a, float4* place)
        : threads(blockDim.x) {
        uint4* at = reinterpret_cast<uint4*>(place);
        w = at, b = at + threads * (R::N / R::V);
        uint32_t r[R::kWords];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            load_vector<T>(part, r, k ? a.bias : a.weight, k ? 0.0f : 1.0f);
#pragma unroll
            for (int u = 0; u < R::N / R::V; ++u)
                at[(k * (R::N / R::V) + u) * threads + threadIdx.x] =
                    make_uint4(r[4 * u], r[4 * u + 1], r[4 * u + 2], r[4 * u + 3]);
        }
    }
    __device__ __forceinline__ void scale(const R&, uint32_t (&out)[R::kWords], const float2 (&v)[R::N / 2],
                                          const Spread& spread) const {
        const float2 s = both(spread.rstd), o = both(-spread.left * spread.rstd);
#pragma unroll
        for (int u = 0; u < R::N / R::V; ++u) {
            const uint4 wv = w[u * threads + threadIdx.x], bv = b[u * threads + threadIdx.x];
            const uint32_t wr[4] = {wv.x, wv.y, wv.z, wv.w}, br[4] = {bv.x, bv.y, bv.z, bv.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int p = 4 * u + i;
                set_pair<T>(out, p, fma2(fma2(v[p], s, o), pair_of<T>(wr, i), pair_of<T>(br, i)));
            }
        }
    }
};
// 32-bit ones need no taking out and stay in registers.
template <class T, class R, int GL>
using Affine = typename std::conditional<GL != 0 || sizeof(T) == 4, Held<T, R>, Shared<T, R>>::type;
template <class T>
int affine_bytes(int threads, int units, bool packed) {
    return sizeof(T) == 4 ? 0 : 2 * threads * units * 16 * (packed ? 1 : 2);
}

// A row's sums over GL lanes, GL 0: over the block.
template <int GL>
struct Total {
    __device__ __forceinline__ float operator()(float v) const {
        float one[1] = {v};
        lanes_sum<GL>(one);
        return one[0];
    }
    __device__ __forceinline__ float2 operator()(float2 v) const {
        float two[2] = {v.x, v.y};
        lanes_sum<GL>(two);
        return make_float2(two[0], two[1]);
    }
};
template <>
struct Total<0> : BlockSum {};
// Two of a block at once: the lower half of a warp's lanes goes on with the
// first, the upper half with the second.  Only where they are asked for: with
// 512 bytes more, 16-bit rows' blocks would not fit three an SM.
struct BlockPairs : BlockSum {
    float* pairs;  // [2][2][32], by the same turns
    __device__ __forceinline__ BlockPairs() {
        __shared__ float all[2][2][32];
        pairs = all[0][0];
        if (threadIdx.x < 64) pairs[threadIdx.x] = pairs[64 + threadIdx.x] = 0.0f;
        __syncthreads();
    }
    using BlockSum::operator();
    __device__ __forceinline__ float2 operator()(float2 f) {
        const bool up = threadIdx.x & 16;
        float* at = pairs + 2 * turn + (threadIdx.x & 16) * 2;
        float v = (up ? f.y : f.x) + __shfl_xor_sync(~0u, up ? f.x : f.y, 16);
#pragma unroll
        for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
        if (threadIdx.x % 16 == 0) at[threadIdx.x / 32] = v;
        __syncthreads();
        v = at[threadIdx.x & 15 & (lanes - 1)];
        if (lanes == 32) v += at[16 + threadIdx.x % 16];
#pragma unroll
        for (int o = 8; o; o >>= 1)
            if (o < lanes) v += __shfl_xor_sync(~0u, v, o);
        const float w = __shfl_xor_sync(~0u, v, 16);
        return up ? make_float2(w, v) : make_float2(v, w);
    }
};
template <class T, int GL>
using RowTotal = typename std::conditional<GL == 0 && kLeft<T>, BlockPairs, Total<GL>>::type;

constexpr int kShort = 256;  // threads a block of short rows
// Its blocks an SM, by the registers of U units a thread.  (2^20 x 64 floats
// forward: 89 us by six, 102 by four; 262144 x 512 bfloat16: 88 by three, 91 by
// four, 166 by six.  2^20 x 128 bfloat16 backward: 174 by four, 230 by two, 272
// by five.)
template <class T, int U>
constexpr int kShortResident = U == 1 ? (sizeof(T) == 4 ? 6 : 4) : sizeof(T) == 4 ? 4 : 3;
template <int U>
constexpr int kShortGradResident = U == 1 ? 4 : 2;

// GL lanes a row; GL 0: the block.
template <class T, int GL, int U, bool STRIDED, int MOST>
__global__ void __launch_bounds__(MOST, GL ? kShortResident<T, U> : MOST == 256 ? 3 : 1024 / MOST)
    layer_norm_kernel(const __grid_constant__ heddle_layer_norm_args a, bool whole) {
    extern __shared__ __align__(128) unsigned char shared[];
    allow_dependents();
    await_previous();
    using R = RowPart<T, U, STRIDED>;
    const int group = GL ? GL : blockDim.x, groups = GL ? MOST / GL : 1;
    const R part{GL ? (int)threadIdx.x % GL : (int)threadIdx.x, group, (int)a.cols};
    const float cols = (float)a.cols, inv = 1.0f / cols;
    const T* x = static_cast<const T*>(a.x);
    uint32_t now[R::kWords], next[R::kWords];
    const int64_t step = (int64_t)gridDim.x * groups;
    int64_t r = (int64_t)blockIdx.x * groups + (GL ? threadIdx.x / GL : 0);
    T* y = static_cast<T*>(a.y) + r * a.ldy;
    // rows past the last are the last again, not stored
    x += (r < a.rows ? r : a.rows - 1) * a.ldx;
    part.load(next, x, whole);
    const Affine<T, R, GL> affine(part, a, reinterpret_cast<float4*>(shared));
    RowTotal<T, GL> total;
    // a warp's groups go round together
    for (int64_t first = (int64_t)blockIdx.x * groups; first < a.rows; first += step, r += step, y += step * a.ldy) {
        float2 v[R::N / 2];
#pragma unroll
        for (int i = 0; i < R::kWords; ++i) now[i] = next[i];
        if (r + step < a.rows) x += step * a.ldx;
        if (first + step < a.rows) part.load(next, x, whole);
        const Mean mean(total(sum_of<T>(part, now)), cols, inv);
        const Spread spread =
            spread_of<T>(total, mean, deviations_of<T, STRIDED>(part, now, v, mean.value), inv, a.eps);
        if (r >= a.rows) continue;
        if (a.mean && part.lane == 0) a.mean[r] = mean.value + spread.left, a.rstd[r] = spread.rstd;
        affine.scale(part, now, v, spread);
        part.store(y, now, whole);
    }
}

// The same by a block for rows that do not lie at 16 bytes: through the ring,
// read from and written to memory in units all the same.
template <class T, int U, bool STRIDED, int MOST>
__global__ void __launch_bounds__(MOST, MOST == 256 ? 2 : 1024 / MOST)
    layer_norm_ring_kernel(const __grid_constant__ heddle_layer_norm_args a, int stages, bool staged, uint32_t* err) {
    extern __shared__ __align__(128) unsigned char shared[];
    allow_dependents();
    await_previous();
    using R = RowPart<T, U, STRIDED>;
    const R part{(int)threadIdx.x, (int)blockDim.x, (int)a.cols};
    const float cols = (float)a.cols, inv = 1.0f / cols;
    const T* x = static_cast<const T*>(a.x);
    Ring ring(shared + sizeof(RingBars), reinterpret_cast<RingBars*>(shared), 1, stages,
              (int)(a.cols * (int64_t)sizeof(T)));
    unsigned char* out = shared + sizeof(RingBars) + stages * ring.place;
    const int rows = (int)((a.rows - blockIdx.x + gridDim.x - 1) / gridDim.x);
    const int64_t step = gridDim.x * a.ldx;
    x += blockIdx.x * a.ldx;
    const T* ahead = x;
    auto fetch = [&](int k) {
        if (k < rows) ring.fetch(ahead, nullptr, nullptr);
        ahead += step;
    };
    for (int k = 0; k < stages - 1; ++k) fetch(k);
    using Vectors = typename std::conditional<U == 4, Packed<T, R>, Affine<T, R, 0>>::type;
    const Vectors affine(part, a, reinterpret_cast<float4*>(out + (staged ? ring.place : 0)));
    T* y = static_cast<T*>(a.y) + blockIdx.x * a.ldy;
    RowTotal<T, 0> total;
    for (int k = 0; k < rows; ++k, x += step, y += gridDim.x * a.ldy) {
        uint32_t words[R::kWords];
        float2 v[R::N / 2];
        ring.wait(0);
        load_units<false>(words, part, ring.row(0, 0), low_of(x) & 15);
        const Mean mean(total(sum_of<T>(part, words)), cols, inv);
        fetch(k + stages - 1);  // all have read the row before this one
        ring.advance(1);
        const Spread spread =
            spread_of<T>(total, mean, deviations_of<T, true>(part, words, v, mean.value), inv, a.eps);
        if (a.mean && threadIdx.x == 0) {
            const int64_t r = blockIdx.x + (int64_t)k * gridDim.x;
            a.mean[r] = mean.value + spread.left, a.rstd[r] = spread.rstd;
        }
        affine.scale(part, words, v, spread);
        store_units<false>(y, part, words, staged ? out : nullptr);
    }
    ring.leave(err);
}

// --------------------------------------------------------------- gradients

// A row's part in the two sums, and in those over rows.
template <class T, class R>
__device__ __forceinline__ void add_row(const R&, const uint32_t (&x)[R::kWords], const uint32_t (&g)[R::kWords],
                                        const uint32_t (&w)[R::kWords], float mean, float rstd, bool live, float& sum0,
                                        float& sum1, float2 (&dw)[R::N / 2], float2 (&db)[R::N / 2]) {
    float2 s0 = both(0.0f), s1 = both(0.0f);
    const float2 m = both(-mean), s = both(rstd);
#pragma unroll
    for (int p = 0; p < R::N / 2; ++p) {
        // past the row's end dy is zero
        const float2 n = mul2(plus<T>(x, p, m), s), f = pair_of<T>(g, p), t = times<T>(g, w, p);
        s0 = add2(s0, t);
        s1 = fma2(t, n, s1);
        if (live) {
            dw[p] = fma2(f, n, dw[p]);
            db[p] = add2(db[p], f);
        }
    }
    sum0 = s0.x + s0.y, sum1 = s1.x + s1.y;
}
// dx = rstd t - rstd mean(t) - ((x - mean) rstd mean(t n)) rstd + dres.  No factor
// is rstd^2, which is past a float's range where rstd is not: a product a pair
// more (300000 x 401 bfloat16 with the weights': 187 us, by n once more 211, by
// rstd^2 186).
template <class T, class R>
__device__ __forceinline__ void grad_row(const R&, uint32_t (&out)[R::kWords], const uint32_t (&x)[R::kWords],
                                         const uint32_t (&g)[R::kWords], const uint32_t (&w)[R::kWords],
                                         const uint32_t (&res)[R::kWords], float mean, float rstd, float mean0,
                                         float mean1) {
    const float2 m = both(-mean), s = both(rstd), c = both(-rstd * mean0), d = both(-rstd * mean1);
#pragma unroll
    for (int p = 0; p < R::N / 2; ++p) {
        const float2 v = mul2(plus<T>(x, p, m), d);
        set_pair<T>(out, p, plus<T>(res, p, fma2(times<T>(g, w, p), s, fma2(v, s, c))));
    }
}

// With the sums over rows, partial[dw, db][block][cols].
template <class T, int GL, int U, bool STRIDED>
__global__ void __launch_bounds__(kShort, kShortGradResident<U>)
    layer_norm_grad_kernel(const __grid_constant__ heddle_layer_norm_grad_args a, float* partial, bool whole) {
    allow_dependents();
    await_previous();
    using R = RowPart<T, U, STRIDED>;
    constexpr int kGroups = kShort / GL;
    const R part{(int)threadIdx.x % GL, GL, (int)a.cols};
    const float cols = (float)a.cols, inv = 1.0f / cols;
    const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy), *dres = static_cast<const T*>(a.dres);
    uint32_t w[R::kWords], xv[R::kWords], gv[R::kWords], rv[R::kWords] = {};
    float2 dw[R::N / 2], db[R::N / 2];
#pragma unroll
    for (int p = 0; p < R::N / 2; ++p) dw[p] = db[p] = both(0.0f);
    load_vector<T>(part, w, a.weight, 1.0f);
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / GL;
    for (int64_t first = (int64_t)blockIdx.x * kGroups; first < a.rows; first += step, r += step) {
        const bool live = r < a.rows;
        const int64_t at = live ? r : a.rows - 1;
        part.load(xv, x + at * a.ldx, whole);
        part.load(gv, dy + at * a.lddy, whole);
        if (dres && a.dx) part.load(rv, dres + at * a.ldr, whole);
        const float mean = a.mean[at], rstd = a.rstd[at];
        float v[2];
        add_row<T>(part, xv, gv, w, mean, rstd, live, v[0], v[1], dw, db);
        lanes_sum<GL>(v);
        if (!a.dx || !live) continue;
        grad_row<T>(part, gv, xv, gv, w, rv, mean, rstd, v[0] * inv, v[1] * inv);
        part.store(static_cast<T*>(a.dx) + r * a.lddx, gv, whole);
    }
    // the block's groups, in order
    __shared__ float sums[kGroups][GL * R::N];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int p = 0; p < R::N / 2; ++p) {
            const float2 v = k ? db[p] : dw[p];
            sums[threadIdx.x / GL][part.at(2 * p)] = v.x, sums[threadIdx.x / GL][part.at(2 * p + 1)] = v.y;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.cols; i += kShort) {
            float v = 0.0f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) v += sums[g][i];
            partial[((int64_t)k * gridDim.x + blockIdx.x) * a.cols + i] = v;
        }
    }
}

// A block a row, x, dy and dres through the ring; they are read from it once
// for the sums and once more for dx.  ROWS at a time between two barriers: two
// where that leaves four ahead (26214 x 5120 bfloat16: 165 us, one at a time
// 182), one where the slots are few (16384 x 8192: 168 us, two 189).
template <class T, int U, bool WHOLE, bool STRIDED, int ROWS, int MOST>
__global__ void __launch_bounds__(MOST)
    layer_norm_grad_ring_kernel(const __grid_constant__ heddle_layer_norm_grad_args a, float* partial, int stages,
                                int arrays, bool staged, uint32_t* err) {
    extern __shared__ __align__(128) unsigned char shared[];
    allow_dependents();
    await_previous();
    using R = RowPart<T, U, STRIDED>;
    const R part{(int)threadIdx.x, (int)blockDim.x, (int)a.cols};
    const float inv = 1.0f / (float)a.cols;
    const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy),
            *dres = a.dx ? static_cast<const T*>(a.dres) : nullptr;
    Ring ring(shared + sizeof(RingBars), reinterpret_cast<RingBars*>(shared), arrays, stages,
              (int)(a.cols * (int64_t)sizeof(T)));
    unsigned char* out = shared + sizeof(RingBars) + stages * arrays * ring.place;
    const int rows = (int)((a.rows - blockIdx.x + gridDim.x - 1) / gridDim.x);
    const int64_t xs = gridDim.x * a.ldx, gs = gridDim.x * a.lddy, rs = gridDim.x * a.ldr, ds = gridDim.x * a.lddx;
    x += blockIdx.x * a.ldx, dy += blockIdx.x * a.lddy;
    if (dres) dres += blockIdx.x * a.ldr;
    T* dx = a.dx ? static_cast<T*>(a.dx) + blockIdx.x * a.lddx : nullptr;
    // where rows lie modulo 16 bytes: those at hand, and their steps
    uint32_t xl = low_of(x), gl = low_of(dy), rl = low_of(dres);
    const uint32_t xd = (uint32_t)(xs * sizeof(T)), gd = (uint32_t)(gs * sizeof(T)), rd = (uint32_t)(rs * sizeof(T));
    auto fetch = [&](int k) {
        if (k < rows) ring.fetch(x, dy, dres);
        x += xs, dy += gs;
        if (dres) dres += rs;
    };
    for (int k = 0; k < stages - ROWS; ++k) fetch(k);
    uint32_t w[R::kWords];
    float2 dw[R::N / 2], db[R::N / 2];
#pragma unroll
    for (int p = 0; p < R::N / 2; ++p) dw[p] = db[p] = both(0.0f);
    load_vector<T>(part, w, a.weight, 1.0f);
    float mean[ROWS], rstd[ROWS];
    auto statistics = [&](int k) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int64_t r = blockIdx.x + (int64_t)(k + i < rows ? k + i : rows - 1) * gridDim.x;
            mean[i] = a.mean[r], rstd[i] = a.rstd[r];
        }
    };
    statistics(0);
    // one row at a time stays in registers where there are enough
    constexpr bool kKeep = ROWS == 1 && MOST <= 512;
    uint32_t xv[R::kWords], gv[R::kWords];
    int turn = 0;
    for (int k = 0; k < rows; k += ROWS) {
        float v[2 * ROWS] = {}, m[ROWS], s[ROWS];
        const unsigned char* at[ROWS][3];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            m[i] = mean[i], s[i] = rstd[i];
#pragma unroll
            for (int j = 0; j < 3; ++j) at[i][j] = ring.row(i, j);
        }
        statistics(k + ROWS);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (k + i >= rows) break;
            ring.wait(i);
            load_units<WHOLE>(xv, part, at[i][0], xl + i * xd & 15);
            load_units<WHOLE>(gv, part, at[i][1], gl + i * gd & 15);
            add_row<T>(part, xv, gv, w, m[i], s[i], true, v[2 * i], v[2 * i + 1], dw, db);
        }
        if constexpr (ROWS == 1)
            block_sums(v[0], v[1], turn);
        else
            block_sums(v, turn);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) fetch(k + stages - ROWS + i);  // in the place of rows that all have left
        ring.advance(ROWS);
        if (dx) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i, dx += ds) {
                if (k + i >= rows) break;
                uint32_t rv[R::kWords] = {};
                if (!kKeep) {
                    load_units<WHOLE>(xv, part, at[i][0], xl + i * xd & 15);
                    load_units<WHOLE>(gv, part, at[i][1], gl + i * gd & 15);
                }
                if (dres) load_units<WHOLE>(rv, part, at[i][2], rl + i * rd & 15);
                grad_row<T>(part, gv, xv, gv, w, rv, m[i], s[i], v[2 * i] * inv, v[2 * i + 1] * inv);
                store_units<WHOLE>(dx, part, gv, staged ? out : nullptr);
            }
        }
        xl += ROWS * xd, gl += ROWS * gd, rl += ROWS * rd;
    }
    if (partial) {
        float *pw = partial + (int64_t)blockIdx.x * a.cols, *pb = pw + (int64_t)gridDim.x * a.cols;
#pragma unroll
        for (int p = 0; p < R::N / 2; ++p) {
            const int i = part.at(2 * p), j = part.at(2 * p + 1);
            if (i < a.cols) pw[i] = dw[p].x, pb[i] = db[p].x;
            if (j < a.cols) pw[j] = dw[p].y, pb[j] = db[p].y;
        }
    }
    ring.leave(err);
}

// ------------------------------------------- rows beyond registers or the ring

constexpr int kLong = 1024;  // two blocks an SM (1024 x 20000 floats: 55 us, by one 71)

template <class T>
__global__ void __launch_bounds__(kLong, 2) layer_norm_long_kernel(const __grid_constant__ heddle_layer_norm_args a) {
    allow_dependents();
    await_previous();
    const float cols = (float)a.cols, inv = 1.0f / cols;
    BlockPairs total;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ldx;
        T* y = static_cast<T*>(a.y) + r * a.ldy;
        float sum = 0.0f;
        float2 sums = both(0.0f);
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) sum += to_float(x[i]);
        const Mean mean(total(sum), cols, inv);
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) {
            const float d = to_float(x[i]) - mean.value;
            sums = make_float2(sums.x + d, fmaf(d, d, sums.y));
        }
        const Spread spread(total(sums), inv, a.eps);
        const float rstd = spread.rstd, o = -spread.left * rstd;
        if (a.mean && threadIdx.x == 0) a.mean[r] = mean.value + spread.left, a.rstd[r] = rstd;
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) {
            const float n = fmaf(to_float(x[i]) - mean.value, rstd, o);
            y[i] = from_float<T>(fmaf(n, a.weight ? to_float(static_cast<const T*>(a.weight)[i]) : 1.0f,
                                      a.bias ? to_float(static_cast<const T*>(a.bias)[i]) : 0.0f));
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kLong)
    layer_norm_long_grad_kernel(const __grid_constant__ heddle_layer_norm_grad_args a) {
    allow_dependents();
    await_previous();
    const float cols = (float)a.cols, inv = 1.0f / cols;
    const T* w = static_cast<const T*>(a.weight);
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T*>(a.x) + r * a.ldx, *dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* dres = static_cast<const T*>(a.dres) + r * a.ldr;
        T* dx = static_cast<T*>(a.dx) + r * a.lddx;
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s[2] = {0.0f, 0.0f};
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) {
            const float t = to_float(dy[i]) * (w ? to_float(w[i]) : 1.0f);
            s[0] += t;
            s[1] = fmaf(t, (to_float(x[i]) - mean) * rstd, s[1]);
        }
        block_sums(s[0], s[1], turn);
        s[0] *= inv, s[1] *= inv;
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) {
            const float t = to_float(dy[i]) * (w ? to_float(w[i]) : 1.0f), n = (to_float(x[i]) - mean) * rstd;
            dx[i] = from_float<T>(fmaf(rstd, fmaf(-n, s[1], t - s[0]), a.dres ? to_float(dres[i]) : 0.0f));
        }
    }
}

// A thread a column, a block of columns and a run of rows a block.
template <class T>
__global__ void __launch_bounds__(256)
    layer_norm_long_sums_kernel(const __grid_constant__ heddle_layer_norm_grad_args a, float* partial) {
    allow_dependents();
    await_previous();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.cols) return;
    const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy);
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float g = to_float(dy[r * a.lddy + i]), n = (to_float(x[r * a.ldx + i]) - a.mean[r]) * a.rstd[r];
        dw = fmaf(g, n, dw);
        db += g;
    }
    partial[(int64_t)blockIdx.y * a.cols + i] = dw;
    partial[((int64_t)gridDim.y + blockIdx.y) * a.cols + i] = db;
}

// The blocks' sums, 32 columns of dw or dbias a block, whose warps take them by
// turns: as many as go through them in one round of loads (11306 rows of 640
// float16 values, 1216 blocks, forward and backward: 31 us by 32 warps, 37 by 8;
// 30 rows of 6310 floats: 14.7 and 13.1).
constexpr int kJoin = 32;    // warps at most
constexpr int kAtOnce = 10;  // loads that a thread waits for together
int join_warps(int64_t parts) { return parts <= 8 * kAtOnce ? 8 : parts <= 16 * kAtOnce ? 16 : kJoin; }
__global__ void __launch_bounds__(32 * kJoin)
    layer_norm_join_kernel(const float* partial, int blocks, int64_t cols, float* dw, float* dbias) {
    allow_dependents();
    await_previous();
    __shared__ float s[kJoin][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    const int64_t i = (int64_t)blockIdx.x * 32 + lane;
    float* out = blockIdx.y ? dbias : dw;
    if (!out) return;
    float v = 0.0f;
    if (i < cols) {
        const float* p = partial + (int64_t)blockIdx.y * blocks * cols + i;
        for (int b0 = warp; b0 < blocks; b0 += warps * kAtOnce) {
            float f[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) f[k] = b0 + k * warps < blocks ? p[(b0 + k * warps) * cols] : 0.0f;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) v += f[k];
        }
    }
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < cols) {
#pragma unroll 8
        for (int k = 1; k < warps; ++k) v += s[k][lane];
        out[i] = v;
    }
}

// -------------------------------------------------------------------- launches

int size_of(int32_t dtype) { return dtype == HEDDLE_FP32 ? 4 : 2; }
int64_t at_most(int64_t want, int64_t most) { return want < most ? want : most; }

constexpr int kShared = 208 * 1024;  // of an SM's, shared by the blocks that it runs

// How a call's rows are taken.  What the order of sums depends on goes by sizes
// alone.
enum Way { kLanes, kBlocks, kRing, kLongRows };
struct Plan {
    Way way;
    // rows of no whole units, whose values are dealt out one by one; but not in a
    // block's forward pass over 16-bit ones (65568 x 2047 bfloat16: units put
    // together from two 155 us, value by value 175; backward 236 and 220)
    bool strided;
    bool whole;        // whole units at 16 bytes throughout
    bool staged;       // rows leave by way of shared memory
    int lanes, units;  // of a short row: lanes; units a lane, or a thread of a block, holds
    int threads, stages;
    size_t shared;
    int64_t blocks;
};

// Short rows: up to 64 units, of which a lane has one, or two of 32 lanes.
// (2^20 x 128 bfloat16 by 16 lanes: 101 us, by 32 167; 262144 x 512 by two units
// a lane or by blocks: forward 88 and 92, backward 175 and 182; 522247 x 257: 228
// and 389.)
void plan_short(const OpContext& x, Plan& p, int64_t rows, int64_t units, int by_one, int by_two) {
    p.way = kLanes;
    p.lanes = units <= 4 ? 4 : units <= 8 ? 8 : units <= 16 ? 16 : 32;
    p.units = units <= 32 ? 1 : 2;
    p.threads = kShort;
    p.blocks = at_most(ceil_div(rows, kShort / p.lanes), (int64_t)x.num_sms * (p.units == 1 ? by_one : by_two));
}

// `arrays` of rows through the ring, by up to `an_sm` blocks an SM: as many as
// leave each three slots of `most` arrays.  `fixed`: shared memory beside it.
void plan_ring(Plan& p, int64_t row_bytes, int arrays, int most, bool whole, bool direct, int fixed, int& an_sm) {
    const int64_t place = row_place(row_bytes);
    auto stages = [&](int n, bool out) {
        return (kShared / an_sm - (int64_t)sizeof(RingBars) - fixed - (out ? place : 0)) / (n * place);
    };
    while (an_sm > 1 && stages(most, true) < 3) --an_sm;
    p.way = stages(most, false) >= 2 ? kRing : kLongRows;
    p.staged = !whole && !direct && stages(arrays, true) >= 2;
    p.stages = (int)at_most(stages(arrays, p.staged), kRingStages);
    p.shared = sizeof(RingBars) + fixed + (p.stages * arrays + p.staged) * place;
}

constexpr int kEach = 2;  // units a thread of a block holds
int block_of(int64_t units) { return (int)at_most(ceil_div(ceil_div(units, kEach), 32) * 32, kLong); }
int blocks_an_sm(int threads_an_sm, int threads) {
    const int n = threads_an_sm / threads;
    return n < 1 ? 1 : n > 24 ? 24 : n;
}

template <class T>
Plan plan_forward(const OpContext& x, const heddle_layer_norm_args& a) {
    Plan p{};
    constexpr int size = sizeof(T), V = 16 / size;
    const int64_t units = ceil_div(a.cols, V);
    p.strided = a.cols % V != 0;
    if (units <= 64) {
        plan_short(x, p, a.rows, units, kShortResident<T, 1>, kShortResident<T, 2>);
        return p;
    }
    const bool whole = !p.strided && rows_whole(a.x, a.ldx, a.rows, size) && rows_whole(a.y, a.ldy, a.rows, size);
    p.threads = block_of(units);
    p.units = kEach;
    p.way = units > kEach * kLong ? kLongRows : kBlocks;
    int an_sm = blocks_an_sm(1024, p.threads);
    // rows of 512 to 1024 units of 16-bit values by smaller blocks, three an SM:
    // 16384 x 8192 bfloat16 takes 87 us, two units a thread 98 (26214 x 5120: 87
    // and 96; 32768 x 4096 the other way round, 92 and 100)
    if (!p.strided && size == 2 && units > 512 && units <= 1024) {
        p.units = 4;
        p.threads = (int)ceil_div(ceil_div(units, 4), 32) * 32;
        an_sm = blocks_an_sm(768, p.threads);
    }
    p.shared = affine_bytes<T>(p.threads, p.units, !whole && p.units == 4);
    if (p.way == kBlocks && !whole)
        plan_ring(p, a.cols * size, 1, 1, false, size == 4 && p.strided, (int)p.shared, an_sm);
    if (p.way == kLongRows) p.threads = kLong, an_sm = 2;
    p.blocks = at_most(a.rows, (int64_t)x.num_sms * an_sm);
    return p;
}

// Rows that a block of the sums beyond the ring takes are those of its place
// among so many.
int64_t long_parts(int64_t rows) { return at_most(rows, 32); }

Plan plan_grad(const OpContext& x, const heddle_layer_norm_grad_args& a) {
    Plan p{};
    const int size = size_of(a.dtype), V = 16 / size;
    const int64_t units = ceil_div(a.cols, V);
    p.strided = a.cols % V != 0;
    if (units <= 64) {
        plan_short(x, p, a.rows, units, kShortGradResident<1>, kShortGradResident<2>);
        return p;
    }
    p.threads = block_of(units);
    p.way = kLongRows;
    // threads an SM, by the registers that each takes (131072 x 1024 bfloat16:
    // 174 us by 512, 211 by 1024)
    int an_sm = blocks_an_sm(size == 2 ? 512 : p.strided ? 608 : 1024, p.threads);
    p.whole = !p.strided && rows_whole(a.x, a.ldx, a.rows, size) && rows_whole(a.dy, a.lddy, a.rows, size) &&
              rows_whole(a.dres, a.ldr, a.rows, size) && rows_whole(a.dx, a.lddx, a.rows, size);
    if (units <= kEach * kLong) plan_ring(p, a.cols * size, a.dres ? 3 : 2, 3, p.whole, p.strided, 0, an_sm);
    if (p.way == kLongRows) p.threads = kLong, an_sm = 2;
    p.blocks = at_most(a.rows, (int64_t)x.num_sms * an_sm);
    return p;
}

template <class K, class... A>
cudaError_t launch_planned(const OpContext& x, K* kernel, std::atomic<uint64_t>& asked, const Plan& p, cudaStream_t st,
                           A... args) {
    const cudaError_t e = allow_shared(kernel, kShared, x.device, asked);
    if (e != cudaSuccess) return e;
    return launch(x, kernel, dim3((unsigned)p.blocks), p.threads, p.shared, st, args...);
}

template <class T, bool STRIDED>
cudaError_t forward_short(const OpContext& x, const heddle_layer_norm_args& a, const Plan& p, cudaStream_t st) {
    constexpr int size = sizeof(T);
    const bool whole = rows_whole(a.x, a.ldx, a.rows, size) && rows_whole(a.y, a.ldy, a.rows, size);
    auto* kernel = p.lanes == 4    ? layer_norm_kernel<T, 4, 1, STRIDED, kShort>
                   : p.lanes == 8  ? layer_norm_kernel<T, 8, 1, STRIDED, kShort>
                   : p.lanes == 16 ? layer_norm_kernel<T, 16, 1, STRIDED, kShort>
                   : p.units == 1  ? layer_norm_kernel<T, 32, 1, STRIDED, kShort>
                                   : layer_norm_kernel<T, 32, 2, STRIDED, kShort>;
    return launch(x, kernel, dim3((unsigned)p.blocks), kShort, 0, st, a, whole);
}

template <class T, int MOST>
cudaError_t forward_blocks(const OpContext& x, const heddle_layer_norm_args& a, const Plan& p, cudaStream_t st) {
    static std::atomic<uint64_t> asked[5];
    if (p.way == kRing) {
        auto* kernel = layer_norm_ring_kernel<T, kEach, false, MOST>;
        if constexpr (sizeof(T) == 4)
            if (p.strided) kernel = layer_norm_ring_kernel<T, kEach, true, MOST>;
        if constexpr (sizeof(T) == 2)
            if (p.units == 4)
                return launch_planned(x, layer_norm_ring_kernel<T, 4, false, 256>, asked[4], p, st, a, p.stages,
                                      p.staged, x.err);
        return launch_planned(x, kernel, asked[p.strided], p, st, a, p.stages, p.staged, x.err);
    }
    if constexpr (sizeof(T) == 2)
        if (p.units == 4) return launch_planned(x, layer_norm_kernel<T, 0, 4, false, 256>, asked[2], p, st, a, true);
    return launch_planned(x, layer_norm_kernel<T, 0, kEach, false, MOST>, asked[3], p, st, a, true);
}

template <class T>
cudaError_t forward_typed(const OpContext& x, const heddle_layer_norm_args& a, cudaStream_t st) {
    const Plan p = plan_forward<T>(x, a);
    if (p.way == kLanes) return p.strided ? forward_short<T, true>(x, a, p, st) : forward_short<T, false>(x, a, p, st);
    if (p.way == kLongRows) return launch(x, layer_norm_long_kernel<T>, dim3((unsigned)p.blocks), kLong, 0, st, a);
    return p.threads <= 512 ? forward_blocks<T, 512>(x, a, p, st) : forward_blocks<T, 1024>(x, a, p, st);
}

template <class T, bool STRIDED>
cudaError_t backward_short(const OpContext& x, const heddle_layer_norm_grad_args& a, const Plan& p, float* partial,
                           cudaStream_t st) {
    constexpr int size = sizeof(T);
    const bool whole = rows_whole(a.x, a.ldx, a.rows, size) && rows_whole(a.dy, a.lddy, a.rows, size) &&
                       rows_whole(a.dres, a.ldr, a.rows, size) && rows_whole(a.dx, a.lddx, a.rows, size);
    auto* kernel = p.lanes == 4    ? layer_norm_grad_kernel<T, 4, 1, STRIDED>
                   : p.lanes == 8  ? layer_norm_grad_kernel<T, 8, 1, STRIDED>
                   : p.lanes == 16 ? layer_norm_grad_kernel<T, 16, 1, STRIDED>
                   : p.units == 1  ? layer_norm_grad_kernel<T, 32, 1, STRIDED>
                                   : layer_norm_grad_kernel<T, 32, 2, STRIDED>;
    return launch(x, kernel, dim3((unsigned)p.blocks), kShort, 0, st, a, partial, whole);
}

template <class T, bool WHOLE, bool STRIDED>
cudaError_t backward_ring(const OpContext& x, const heddle_layer_norm_grad_args& a, const Plan& p, float* partial,
                          cudaStream_t st) {
    static std::atomic<uint64_t> asked[3];
    const int arrays = a.dres ? 3 : 2;
    if (p.threads > 512)
        return launch_planned(x, layer_norm_grad_ring_kernel<T, kEach, WHOLE, STRIDED, 1, 1024>, asked[0], p, st, a,
                              partial, p.stages, arrays, p.staged, x.err);
    if (p.stages < 6 || !WHOLE)
        return launch_planned(x, layer_norm_grad_ring_kernel<T, kEach, WHOLE, STRIDED, 1, 512>, asked[1], p, st, a,
                              partial, p.stages, arrays, p.staged, x.err);
    return launch_planned(x, layer_norm_grad_ring_kernel<T, kEach, true, false, 2, 512>, asked[2], p, st, a, partial,
                          p.stages, arrays, p.staged, x.err);
}

template <class T>
cudaError_t backward_rows(const OpContext& x, const heddle_layer_norm_grad_args& a, const Plan& p, float* partial,
                          cudaStream_t st) {
    if (p.way == kLanes)
        return p.strided ? backward_short<T, true>(x, a, p, partial, st)
                         : backward_short<T, false>(x, a, p, partial, st);
    if (p.strided) return backward_ring<T, false, true>(x, a, p, partial, st);
    return p.whole ? backward_ring<T, true, false>(x, a, p, partial, st)
                   : backward_ring<T, false, false>(x, a, p, partial, st);
}

template <class T>
cudaError_t backward_typed(const OpContext& x, const heddle_layer_norm_grad_args& a, float* partial, cudaStream_t st) {
    const Plan p = plan_grad(x, a);
    const bool sums = a.dw || a.dbias;
    int64_t parts = a.rows ? p.blocks : 0;
    cudaError_t e = cudaSuccess;
    if (p.way == kLongRows) {  // the sums first: dx may take dy's place
        parts = long_parts(a.rows);
        const dim3 grid((unsigned)ceil_div(a.cols, 256), (unsigned)parts);
        if (sums && a.rows) e = launch(x, layer_norm_long_sums_kernel<T>, grid, 256, 0, st, a, partial);
        if (e == cudaSuccess && a.dx && a.rows)
            e = launch(x, layer_norm_long_grad_kernel<T>, dim3((unsigned)p.blocks), kLong, 0, st, a);
    } else if (a.rows) {
        e = backward_rows<T>(x, a, p, partial, st);
    }
    if (e == cudaSuccess && sums)
        e = launch(x, layer_norm_join_kernel, dim3((unsigned)ceil_div(a.cols, 32), 2), 32 * join_warps(parts), 0,
                   st, (const float*)partial, (int)parts, a.cols, a.dw, a.dbias);
    return e;
}

}  // namespace

cudaError_t launch_layer_norm(const OpContext& x, const heddle_layer_norm_args& a, cudaStream_t st) {
    switch (a.dtype) {
        case HEDDLE_BF16: return forward_typed<__nv_bfloat16>(x, a, st);
        case HEDDLE_FP16: return forward_typed<__half>(x, a, st);
        default: return forward_typed<float>(x, a, st);
    }
}

size_t layer_norm_grad_scratch(const OpContext& x, const heddle_layer_norm_grad_args& a) {
    const Plan p = plan_grad(x, a);
    // a short row's kernel writes its sums whether they are asked for or not
    if (!a.dw && !a.dbias && p.way != kLanes) return 0;
    return align256(sizeof(float) * 2 * (size_t)(p.way == kLongRows ? long_parts(a.rows) : p.blocks) * a.cols);
}

cudaError_t launch_layer_norm_grad(const OpContext& x, const heddle_layer_norm_grad_args& a, unsigned char* ws,
                                   cudaStream_t st) {
    const Plan p = plan_grad(x, a);
    float* partial = a.dw || a.dbias || p.way == kLanes ? reinterpret_cast<float*>(ws) : nullptr;
    switch (a.dtype) {
        case HEDDLE_BF16: return backward_typed<__nv_bfloat16>(x, a, partial, st);
        case HEDDLE_FP16: return backward_typed<__half>(x, a, partial, st);
        default: return backward_typed<float>(x, a, partial, st);
    }
}

}  // namespace hd
