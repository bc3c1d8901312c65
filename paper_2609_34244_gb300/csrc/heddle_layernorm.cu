// heddle_layernorm.cu -- layer norm and its gradients.
//
// Bound by memory.  A row is held in the registers of a group of threads: its
// mean first, then the squares of its deviations from it, so that a large mean
// costs no digits and nothing is read twice.  A block walks over rows and
// fetches the next one while it adds up the one at hand.  Gradients: the same,
// with the weights' sums over rows in registers, one set a block, which a
// second kernel adds in order.

#include "heddle_rows.cuh"

namespace hd {
namespace {

// The group's sums of N values, the same in every thread.  `turn` alternates
// between calls: one barrier each.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if constexpr (G > 32) {
        constexpr int W = G / 32;
        __shared__ float part[2][N][W];
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) part[turn][i][warp] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = part[turn][i][lane % W];
#pragma unroll
            for (int o = W / 2; o; o >>= 1) v[i] += __shfl_xor_sync(~0u, v[i], o);
        }
        turn ^= 1;
    }
}

template <int G>
constexpr int kBlock = G == 32 ? 256 : G;

template <class T, int G, int U, bool STRIDED>
__global__ void __launch_bounds__(kBlock<G>)
    layer_norm_kernel(const __grid_constant__ heddle_layer_norm_args a, bool whole) {
    allow_dependents();
    await_previous();
    using R = RowPart<T, G, U, STRIDED>;
    constexpr int kGroups = kBlock<G> / G;
    const R part{(int)(threadIdx.x % G), (int)a.cols};
    const float n_cols = (float)a.cols;
    const T* x = static_cast<const T*>(a.x);
    uint4 w[U], b[U], now[U], next[U];
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G;
    if (r >= a.rows) return;  // whole warps where a group is one
    part.load(next, x + r * a.ldx, whole);
    if (a.weight) part.load(w, static_cast<const T*>(a.weight), whole);
    if (a.bias) part.load(b, static_cast<const T*>(a.bias), whole);
    int turn = 0;
    for (; r < a.rows; r += step) {
#pragma unroll
        for (int u = 0; u < U; ++u) now[u] = next[u];
        if (r + step < a.rows) part.load(next, x + (r + step) * a.ldx, whole);
        float sum[1] = {0.0f};
#pragma unroll
        for (int e = 0; e < R::N; ++e) sum[0] += R::get(now, e);
        group_sum<G>(sum, turn);
        const float mean = sum[0] / n_cols;
        float sq[1] = {0.0f};
#pragma unroll
        for (int e = 0; e < R::N; ++e) {
            const float d = part.in(e) ? R::get(now, e) - mean : 0.0f;
            sq[0] = fmaf(d, d, sq[0]);
        }
        group_sum<G>(sq, turn);
        const float rstd = 1.0f / sqrtf(sq[0] / n_cols + a.eps);
        if (a.mean && part.lane == 0) a.mean[r] = mean, a.rstd[r] = rstd;
#pragma unroll
        for (int e = 0; e < R::N; ++e) {
            const float n = (R::get(now, e) - mean) * rstd;
            R::set(now, e, fmaf(n, a.weight ? R::get(w, e) : 1.0f, a.bias ? R::get(b, e) : 0.0f));
        }
        part.store(static_cast<T*>(a.y) + r * a.ldy, now, whole);
    }
}

// SUMS: with the sums over rows, partial[dw, db][block][cols].
template <class T, int G, int U, bool STRIDED, bool SUMS>
__global__ void __launch_bounds__(kBlock<G>)
    layer_norm_grad_kernel(const __grid_constant__ heddle_layer_norm_grad_args a, float* partial, bool whole) {
    allow_dependents();
    await_previous();
    using R = RowPart<T, G, U, STRIDED>;
    constexpr int kGroups = kBlock<G> / G;
    const R part{(int)(threadIdx.x % G), (int)a.cols};
    const float n_cols = (float)a.cols;
    const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy), *dres = static_cast<const T*>(a.dres);
    uint4 w[U], xv[U], gv[U], rv[U];
    float dw[SUMS ? R::N : 1] = {}, db[SUMS ? R::N : 1] = {};
    if (a.weight) part.load(w, static_cast<const T*>(a.weight), whole);
    int turn = 0;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    for (int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G; r < a.rows; r += step) {
        part.load(xv, x + r * a.ldx, whole);
        part.load(gv, dy + r * a.lddy, whole);
        if (dres && a.dx) part.load(rv, dres + r * a.ldr, whole);
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < R::N; ++e) {
            // past the row's end dy and the weight are zeros
            const float n = (R::get(xv, e) - mean) * rstd, g = R::get(gv, e);
            const float t = a.weight ? __fmul_rn(g, R::get(w, e)) : g;
            s[0] += t;
            s[1] = fmaf(t, part.in(e) ? n : 0.0f, s[1]);
            if constexpr (SUMS) {
                dw[e] = fmaf(g, n, dw[e]);
                db[e] += g;
            }
        }
        if (!a.dx) continue;
        group_sum<G>(s, turn);
        s[0] /= n_cols, s[1] /= n_cols;
#pragma unroll
        for (int e = 0; e < R::N; ++e) {
            const float n = (R::get(xv, e) - mean) * rstd, g = R::get(gv, e);
            const float t = a.weight ? __fmul_rn(g, R::get(w, e)) : g;
            R::set(gv, e, fmaf(rstd, fmaf(-n, s[1], t - s[0]), dres ? R::get(rv, e) : 0.0f));
        }
        part.store(static_cast<T*>(a.dx) + r * a.lddx, gv, whole);
    }
    if constexpr (SUMS) {
        float *pw = partial + (int64_t)blockIdx.x * a.cols, *pb = pw + (int64_t)gridDim.x * a.cols;
        if constexpr (G > 32) {
#pragma unroll
            for (int e = 0; e < R::N; ++e)
                if (part.in(e)) pw[part.at(e)] = dw[e], pb[part.at(e)] = db[e];
        } else {  // the block's groups, in order
            __shared__ float s[kGroups][G * R::N];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < R::N; ++e) s[threadIdx.x / G][part.at(e)] = k ? db[e] : dw[e];
                __syncthreads();
                for (int i = threadIdx.x; i < a.cols; i += kBlock<G>) {
                    float v = 0.0f;
#pragma unroll
                    for (int g = 0; g < kGroups; ++g) v += s[g][i];
                    (k ? pb : pw)[i] = v;
                }
            }
        }
    }
}

// ------------------------------------------------- rows beyond the registers

constexpr int kLong = 1024;

template <class T>
__global__ void __launch_bounds__(kLong) layer_norm_long_kernel(const __grid_constant__ heddle_layer_norm_args a) {
    allow_dependents();
    await_previous();
    const float n_cols = (float)a.cols;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ldx;
        T* y = static_cast<T*>(a.y) + r * a.ldy;
        float sum[1] = {0.0f}, sq[1] = {0.0f};
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) sum[0] += to_float(x[i]);
        group_sum<kLong>(sum, turn);
        const float mean = sum[0] / n_cols;
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) {
            const float d = to_float(x[i]) - mean;
            sq[0] = fmaf(d, d, sq[0]);
        }
        group_sum<kLong>(sq, turn);
        const float rstd = 1.0f / sqrtf(sq[0] / n_cols + a.eps);
        if (a.mean && threadIdx.x == 0) a.mean[r] = mean, a.rstd[r] = rstd;
        for (int64_t i = threadIdx.x; i < a.cols; i += kLong) {
            const float n = (to_float(x[i]) - mean) * rstd;
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
    const float n_cols = (float)a.cols;
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
        group_sum<kLong>(s, turn);
        s[0] /= n_cols, s[1] /= n_cols;
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

// The blocks' sums, 32 columns of dw or dbias a block.
__global__ void __launch_bounds__(1024)
    layer_norm_join_kernel(const float* partial, int blocks, int64_t cols, float* dw, float* dbias) {
    allow_dependents();
    await_previous();
    __shared__ float s[32][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t i = (int64_t)blockIdx.x * 32 + lane;
    float* out = blockIdx.y ? dbias : dw;
    if (!out) return;
    float v = 0.0f;
    if (i < cols)
#pragma unroll 8
        for (int b = warp; b < blocks; b += 32) v += partial[((int64_t)blockIdx.y * blocks + b) * cols + i];
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < cols) {
        for (int k = 1; k < 32; ++k) v += s[k][lane];
        out[i] = v;
    }
}

// -------------------------------------------------------------------- launches

int size_of(int32_t dtype) { return dtype == HEDDLE_FP32 ? 4 : 2; }

// Threads a row, by the 16-byte units that it takes: up to two a thread, in
// warps where they do; 0: beyond the registers.
int group_of(int64_t cols, int32_t dtype) {
    const int64_t units = ceil_div(cols, 16 / size_of(dtype));
    return units <= 64 ? 32 : units <= 256 ? 128 : units <= 512 ? 256 : units <= 1024 ? 512 : units <= 2048 ? 1024 : 0;
}

int64_t at_most(int64_t want, int64_t most) { return want < most ? want : most; }

int64_t blocks_of(const OpContext& x, int64_t rows, int group, int threads_an_sm) {
    if (!group) return at_most(rows, (int64_t)x.num_sms * 2);
    const int block = group == 32 ? 256 : group;
    return at_most(ceil_div(rows, block / group), (int64_t)x.num_sms * (threads_an_sm / block));
}

// Rows that a block of the sums beyond the registers takes are those of its
// place among so many.
int64_t long_parts(int64_t rows) { return at_most(rows, 32); }

constexpr int kFwdThreads = 1024, kGradThreads = 1024;  // an SM

template <class T, bool STRIDED>
cudaError_t forward(const OpContext& x, const heddle_layer_norm_args& a, cudaStream_t st) {
    const int group = group_of(a.cols, a.dtype), size = sizeof(T);
    const dim3 grid((unsigned)blocks_of(x, a.rows, group, kFwdThreads));
    const bool whole = rows_whole(a.x, a.ldx, a.rows, size) && rows_whole(a.y, a.ldy, a.rows, size) &&
                       rows_whole(a.weight, 0, 1, size) && rows_whole(a.bias, 0, 1, size);
    switch (group) {
        case 32: return launch(x, layer_norm_kernel<T, 32, 2, STRIDED>, grid, 256, 0, st, a, whole);
        case 128: return launch(x, layer_norm_kernel<T, 128, 2, STRIDED>, grid, 128, 0, st, a, whole);
        case 256: return launch(x, layer_norm_kernel<T, 256, 2, STRIDED>, grid, 256, 0, st, a, whole);
        case 512: return launch(x, layer_norm_kernel<T, 512, 2, STRIDED>, grid, 512, 0, st, a, whole);
        case 1024: return launch(x, layer_norm_kernel<T, 1024, 2, STRIDED>, grid, 1024, 0, st, a, whole);
        default: return launch(x, layer_norm_long_kernel<T>, grid, kLong, 0, st, a);
    }
}

template <class T, bool STRIDED, bool SUMS>
cudaError_t backward(const OpContext& x, const heddle_layer_norm_grad_args& a, float* partial, unsigned blocks,
                     cudaStream_t st) {
    const int size = sizeof(T);
    const bool whole = rows_whole(a.x, a.ldx, a.rows, size) && rows_whole(a.dy, a.lddy, a.rows, size) &&
                       rows_whole(a.dres, a.ldr, a.rows, size) && rows_whole(a.dx, a.lddx, a.rows, size) &&
                       rows_whole(a.weight, 0, 1, size);
    const dim3 grid(blocks);
    switch (group_of(a.cols, a.dtype)) {
        case 32: return launch(x, layer_norm_grad_kernel<T, 32, 2, STRIDED, SUMS>, grid, 256, 0, st, a, partial, whole);
        case 128:
            return launch(x, layer_norm_grad_kernel<T, 128, 2, STRIDED, SUMS>, grid, 128, 0, st, a, partial, whole);
        case 256:
            return launch(x, layer_norm_grad_kernel<T, 256, 2, STRIDED, SUMS>, grid, 256, 0, st, a, partial, whole);
        case 512:
            return launch(x, layer_norm_grad_kernel<T, 512, 2, STRIDED, SUMS>, grid, 512, 0, st, a, partial, whole);
        default:
            return launch(x, layer_norm_grad_kernel<T, 1024, 2, STRIDED, SUMS>, grid, 1024, 0, st, a, partial, whole);
    }
}

template <class T>
cudaError_t backward_typed(const OpContext& x, const heddle_layer_norm_grad_args& a, float* partial, cudaStream_t st) {
    const int group = group_of(a.cols, a.dtype);
    const bool sums = a.dw || a.dbias, strided = a.cols % (16 / (int)sizeof(T)) != 0;
    unsigned blocks = (unsigned)blocks_of(x, a.rows, group, kGradThreads);
    cudaError_t e = cudaSuccess;
    if (!group) {  // the sums first: dx may take dy's place
        const unsigned rows = blocks;
        blocks = (unsigned)long_parts(a.rows);
        const dim3 grid((unsigned)ceil_div(a.cols, 256), blocks);
        if (sums && a.rows) e = launch(x, layer_norm_long_sums_kernel<T>, grid, 256, 0, st, a, partial);
        if (e == cudaSuccess && a.dx && a.rows)
            e = launch(x, layer_norm_long_grad_kernel<T>, dim3(rows), kLong, 0, st, a);
    } else if (a.rows) {
        if (sums)
            e = strided ? backward<T, true, true>(x, a, partial, blocks, st)
                        : backward<T, false, true>(x, a, partial, blocks, st);
        else
            e = strided ? backward<T, true, false>(x, a, partial, blocks, st)
                        : backward<T, false, false>(x, a, partial, blocks, st);
    }
    if (e == cudaSuccess && sums)
        e = launch(x, layer_norm_join_kernel, dim3((unsigned)ceil_div(a.cols, 32), 2), 1024, 0, st, partial,
                   (int)(a.rows ? blocks : 0), a.cols, a.dw, a.dbias);
    return e;
}

}  // namespace

cudaError_t launch_layer_norm(const OpContext& x, const heddle_layer_norm_args& a, cudaStream_t st) {
    const bool strided = a.cols % (16 / size_of(a.dtype)) != 0;
    switch (a.dtype) {
        case HEDDLE_BF16:
            return strided ? forward<__nv_bfloat16, true>(x, a, st) : forward<__nv_bfloat16, false>(x, a, st);
        case HEDDLE_FP16: return strided ? forward<__half, true>(x, a, st) : forward<__half, false>(x, a, st);
        default: return strided ? forward<float, true>(x, a, st) : forward<float, false>(x, a, st);
    }
}

size_t layer_norm_grad_scratch(const OpContext& x, const heddle_layer_norm_grad_args& a) {
    if (!a.dw && !a.dbias) return 0;
    const int group = group_of(a.cols, a.dtype);
    const int64_t parts = group ? blocks_of(x, a.rows, group, kGradThreads) : long_parts(a.rows);
    return align256(sizeof(float) * 2 * (size_t)parts * a.cols);
}

cudaError_t launch_layer_norm_grad(const OpContext& x, const heddle_layer_norm_grad_args& a, unsigned char* ws,
                                   cudaStream_t st) {
    float* partial = reinterpret_cast<float*>(ws);
    switch (a.dtype) {
        case HEDDLE_BF16: return backward_typed<__nv_bfloat16>(x, a, partial, st);
        case HEDDLE_FP16: return backward_typed<__half>(x, a, partial, st);
        default: return backward_typed<float>(x, a, partial, st);
    }
}

}  // namespace hd
