// heddle_dropout.cu -- dropout into the residual stream, its mask made anew in
// either direction.
//
// The random numbers are Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32 x 32 products and exclusive ors over a counter of 128 bits, four words a
// counter, one a value.  They cost about 60 instructions for four values, and
// memory brings four 16-bit values to an SM in a cycle.

#include "heddle_rows.cuh"

namespace hd {
namespace {

struct Dropout {
    heddle_dropout_args a;
    uint32_t least;  // the smallest number that is kept
    float scale;
};

// Ten rounds: the counter in c, the key in k.
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ (k0 + r * 0x9E3779B9u);
        c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ (k1 + r * 0xBB67AE85u);
        c[3] = (uint32_t)a;
    }
}

__device__ __forceinline__ void numbers(uint32_t (&c)[4], const Dropout& d, uint64_t four, uint64_t offset) {
    c[0] = (uint32_t)four, c[1] = (uint32_t)(four >> 32);
    c[2] = (uint32_t)offset, c[3] = (uint32_t)(offset >> 32);
    philox(c, (uint32_t)d.a.seed, (uint32_t)(d.a.seed >> 32));
}

__device__ __forceinline__ float dropped(const Dropout& d, uint32_t u, float x) {
    return u < d.least ? 0.0f : x * d.scale;
}

constexpr int kThreads = 256;
constexpr int kUnits = 2;  // of 16 bytes a thread takes at a time

// Rows of whole 16-byte units; everything is one row where rows follow each
// other, and its end may then be part of a unit.
template <class T, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads) dropout_units_kernel(const __grid_constant__ Dropout d) {
    allow_dependents();
    await_previous();
    constexpr int V = 16 / sizeof(T);
    const T *x = static_cast<const T*>(d.a.x), *res = static_cast<const T*>(d.a.residual);
    T* y = static_cast<T*>(d.a.y);
    const uint64_t offset = d.a.offset + (d.a.step ? (uint64_t)*d.a.step : 0);
    const int64_t cols = d.a.cols, per = (cols + V - 1) / V, total = d.a.rows * per;
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; i0 < total; i0 += kUnits * step) {
        uint4 v[kUnits], w[kUnits];
        int64_t row[kUnits], col[kUnits];
        bool live[kUnits], full[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int64_t i = i0 + k * step;
            live[k] = i < total;
            row[k] = d.a.rows == 1 ? 0 : i / per;
            col[k] = (i - row[k] * per) * V;
            full[k] = live[k] && col[k] + V <= cols;
            if (full[k]) {
                v[k] = *reinterpret_cast<const uint4*>(x + row[k] * d.a.ldx + col[k]);
                if (RESIDUAL) w[k] = *reinterpret_cast<const uint4*>(res + row[k] * d.a.ldr + col[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            if (!live[k]) continue;
            const uint64_t first = (uint64_t)row[k] * cols + col[k];
            uint32_t u[V / 4][4];
#pragma unroll
            for (int q = 0; q < V / 4; ++q) numbers(u[q], d, first / 4 + q, offset);
            if (full[k]) {
                T* t = reinterpret_cast<T*>(&v[k]);
                const T* r = reinterpret_cast<const T*>(&w[k]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float f = dropped(d, u[e / 4][e % 4], to_float(t[e]));
                    if (RESIDUAL) f += to_float(r[e]);
                    t[e] = from_float<T>(f);
                }
                *reinterpret_cast<uint4*>(y + row[k] * d.a.ldy + col[k]) = v[k];
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (col[k] + e >= cols) break;
                    float f = dropped(d, u[e / 4][e % 4], to_float(x[row[k] * d.a.ldx + col[k] + e]));
                    if (RESIDUAL) f += to_float(res[row[k] * d.a.ldr + col[k] + e]);
                    y[row[k] * d.a.ldy + col[k] + e] = from_float<T>(f);
                }
            }
        }
    }
}

// Any strides and addresses: four columns a thread, whose numbers are those of
// one counter or two.
template <class T>
__global__ void __launch_bounds__(kThreads) dropout_any_kernel(const __grid_constant__ Dropout d) {
    allow_dependents();
    await_previous();
    const T *x = static_cast<const T*>(d.a.x), *res = static_cast<const T*>(d.a.residual);
    T* y = static_cast<T*>(d.a.y);
    const uint64_t offset = d.a.offset + (d.a.step ? (uint64_t)*d.a.step : 0);
    const int64_t cols = d.a.cols, per = (cols + 3) / 4, total = d.a.rows * per;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / per, col = (i - row * per) * 4;
        const uint64_t first = (uint64_t)row * cols + col;
        const int skip = (int)(first & 3);
        uint32_t u[2][4];
        numbers(u[0], d, first / 4, offset);
        if (skip) numbers(u[1], d, first / 4 + 1, offset);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (col + e >= cols) break;
            uint32_t n = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j == skip + e) n = u[j / 4][j % 4];
            float f = dropped(d, n, to_float(x[row * d.a.ldx + col + e]));
            if (res) f += to_float(res[row * d.a.ldr + col + e]);
            y[row * d.a.ldy + col + e] = from_float<T>(f);
        }
    }
}

template <class T>
cudaError_t run(const OpContext& x, Dropout d, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T), size = sizeof(T);
    heddle_dropout_args& a = d.a;
    if (a.rows > 1 && a.ldx == a.cols && a.ldy == a.cols && (!a.residual || a.ldr == a.cols))
        a.cols *= a.rows, a.rows = 1;
    const bool units = (a.rows == 1 || a.cols % V == 0) && rows_whole(a.x, a.ldx, a.rows, size) &&
                       rows_whole(a.y, a.ldy, a.rows, size) && rows_whole(a.residual, a.ldr, a.rows, size);
    const int64_t per = units ? kUnits * kThreads : kThreads, most = (int64_t)x.num_sms * 16;
    const int64_t want = ceil_div(a.rows * ceil_div(a.cols, units ? V : 4), per);
    const dim3 grid((unsigned)(want < most ? want : most));
    if (!units) return launch(x, dropout_any_kernel<T>, grid, kThreads, 0, st, d);
    return a.residual ? launch(x, dropout_units_kernel<T, true>, grid, kThreads, 0, st, d)
                      : launch(x, dropout_units_kernel<T, false>, grid, kThreads, 0, st, d);
}

}  // namespace

cudaError_t launch_dropout(const OpContext& x, const heddle_dropout_args& a, cudaStream_t st) {
    Dropout d{};
    d.a = a;
    const double all = 4294967296.0, least = nearbyint(a.p * all);
    d.least = (uint32_t)(least < all ? least : all - 1.0);
    d.scale = (float)(all / (all - (double)d.least));
    if (a.dtype == HEDDLE_BF16) return run<__nv_bfloat16>(x, d, st);
    if (a.dtype == HEDDLE_FP16) return run<__half>(x, d, st);
    return run<float>(x, d, st);
}

}  // namespace hd
