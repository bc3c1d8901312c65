// heddle_dropout.cu -- dropout into the residual stream, its mask made anew in
// either direction.
//
// The random numbers are Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32 x 32 products and exclusive ors over a counter of 128 bits, four words a
// counter, one a value.  They cost about 60 instructions for four values, and
// memory brings four 16-bit values to an SM in a cycle.  16384 x 8192 bfloat16
// with the residual, forward and backward: 227 us, 5.9 TB/s.

#include "heddle_rows.cuh"

namespace hd {
namespace {

constexpr int kRounds = 10;

struct Dropout {
    heddle_dropout_args a;
    uint32_t least;  // the smallest number that is kept
    float scale;
    // each round's: added up by the host, so that an exclusive or takes them as
    // they come with the launch
    uint32_t key[kRounds][2];
};

// Two of the twenty products are the same for all counters of one offset whose
// upper halves (`high`) agree, 2^32 of them: the first round's second and the
// second round's first.  They are kept.
struct Start {
    uint32_t high, c1, hi, lo, c3;
};
__device__ __forceinline__ Start start_of(const Dropout& d, uint32_t high, uint64_t offset) {
    const uint64_t b = (uint64_t)(uint32_t)offset * 0xCD9E8D57u;
    const uint32_t c0 = (uint32_t)(b >> 32) ^ high ^ d.key[0][0];
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u;
    return {high, (uint32_t)b, (uint32_t)(a >> 32), (uint32_t)a, (uint32_t)(offset >> 32) ^ d.key[0][1]};
}

// The four numbers of the counter (low, s.high, offset).
__device__ __forceinline__ void numbers(uint32_t (&c)[4], const Dropout& d, const Start& s, uint32_t low) {
    const uint64_t first = (uint64_t)low * 0xD2511F53u;
    const uint64_t second = (uint64_t)((uint32_t)(first >> 32) ^ s.c3) * 0xCD9E8D57u;
    c[0] = (uint32_t)(second >> 32) ^ s.c1 ^ d.key[1][0];
    c[1] = (uint32_t)second;
    c[2] = s.hi ^ (uint32_t)first ^ d.key[1][1];
    c[3] = s.lo;
#pragma unroll
    for (int r = 2; r < kRounds; ++r) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ d.key[r][0];
        c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ d.key[r][1];
        c[3] = (uint32_t)a;
    }
}

// to + (u < least ? 0 : x scale), the product under a predicate: a selection
// would take another instruction of the pipe that the exclusive ors fill.
__device__ __forceinline__ float kept(const Dropout& d, uint32_t u, float x, float to) {
    asm("{\n\t.reg .pred p;\n\tsetp.ge.u32 p, %1, %2;\n\t@p fma.rn.f32 %0, %3, %4, %0;\n\t}"
        : "+f"(to)
        : "r"(u), "r"(d.least), "f"(x), "f"(d.scale));
    return to;
}

constexpr int kThreads = 256;
// Blocks an SM: as many as the numbers' registers allow without spilling, in
// four rounds (a unit a thread in more or fewer registers, two units at a
// time, the next unit fetched ahead: 230 to 298 us where this takes 227).
constexpr int kResident = 6, kTurns = 4;

// Whole 16-byte units.  FLAT: rows follow each other and are taken as one,
// whose end may be part of a unit.
template <class T, bool RESIDUAL, bool FLAT>
__global__ void __launch_bounds__(kThreads, kResident) dropout_units_kernel(const __grid_constant__ Dropout d) {
    allow_dependents();
    await_previous();
    constexpr int V = 16 / sizeof(T);
    const T *x = static_cast<const T*>(d.a.x), *res = static_cast<const T*>(d.a.residual);
    T* y = static_cast<T*>(d.a.y);
    const uint64_t offset = d.a.offset + (d.a.step ? (uint64_t)*d.a.step : 0);
    Start start = start_of(d, 0, offset);
    const int64_t per = d.a.cols / V, total = FLAT ? per : d.a.rows * per, step = (int64_t)gridDim.x * kThreads;
    auto take = [&](int64_t i, const float (&f)[V], float (&to)[V]) {
        const uint64_t four = (uint64_t)i * (V / 4);
        if (four >> 32 != start.high) start = start_of(d, (uint32_t)(four >> 32), offset);
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            uint32_t u[4];
            numbers(u, d, start, (uint32_t)four + q);
#pragma unroll
            for (int e = 0; e < 4; ++e) to[4 * q + e] = kept(d, u[e], f[4 * q + e], to[4 * q + e]);
        }
    };
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += step) {
        const int64_t row = FLAT ? 0 : i / per, col = (i - row * per) * V;
        float f[V], to[V] = {};
        unpack<T>(*reinterpret_cast<const uint4*>(x + row * d.a.ldx + col), f);
        if (RESIDUAL) unpack<T>(*reinterpret_cast<const uint4*>(res + row * d.a.ldr + col), to);
        take(i, f, to);
        *reinterpret_cast<uint4*>(y + row * d.a.ldy + col) = pack<T>(to);
    }
    const int64_t left = FLAT ? d.a.cols - per * V : 0;
    if (left && blockIdx.x == 0 && threadIdx.x == 0) {
        float f[V] = {}, to[V] = {};
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < left) f[e] = to_float(x[per * V + e]), to[e] = RESIDUAL ? to_float(res[per * V + e]) : 0.0f;
        take(per, f, to);
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < left) y[per * V + e] = from_float<T>(to[e]);
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
        const uint64_t four = first / 4;
        numbers(u[0], d, start_of(d, (uint32_t)(four >> 32), offset), (uint32_t)four);
        if (skip) numbers(u[1], d, start_of(d, (uint32_t)((four + 1) >> 32), offset), (uint32_t)(four + 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (col + e >= cols) break;
            uint32_t n = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j == skip + e) n = u[j / 4][j % 4];
            const float to = res ? to_float(res[row * d.a.ldr + col + e]) : 0.0f;
            y[row * d.a.ldy + col + e] = from_float<T>(kept(d, n, to_float(x[row * d.a.ldx + col + e]), to));
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
    const int64_t most = (int64_t)x.num_sms * kResident * kTurns;
    const int64_t want = ceil_div(units ? ceil_div(a.rows * a.cols, V) : a.rows * ceil_div(a.cols, 4), kThreads);
    const dim3 grid((unsigned)(want < most ? want : most));
    if (!units) return launch(x, dropout_any_kernel<T>, grid, kThreads, 0, st, d);
    if (a.rows == 1)
        return a.residual ? launch(x, dropout_units_kernel<T, true, true>, grid, kThreads, 0, st, d)
                          : launch(x, dropout_units_kernel<T, false, true>, grid, kThreads, 0, st, d);
    return a.residual ? launch(x, dropout_units_kernel<T, true, false>, grid, kThreads, 0, st, d)
                      : launch(x, dropout_units_kernel<T, false, false>, grid, kThreads, 0, st, d);
}

}  // namespace

cudaError_t launch_dropout(const OpContext& x, const heddle_dropout_args& a, cudaStream_t st) {
    Dropout d{};
    d.a = a;
    const double all = 4294967296.0, least = nearbyint(a.p * all);
    d.least = (uint32_t)(least < all ? least : all - 1.0);
    d.scale = (float)(all / (all - (double)d.least));
    for (int r = 0; r < kRounds; ++r) {
        d.key[r][0] = (uint32_t)a.seed + r * 0x9E3779B9u;
        d.key[r][1] = (uint32_t)(a.seed >> 32) + r * 0xBB67AE85u;
    }
    if (a.dtype == HEDDLE_BF16) return run<__nv_bfloat16>(x, d, st);
    if (a.dtype == HEDDLE_FP16) return run<__half>(x, d, st);
    return run<float>(x, d, st);
}

}  // namespace hd
