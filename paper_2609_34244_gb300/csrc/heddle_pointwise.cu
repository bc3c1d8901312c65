// heddle_pointwise.cu -- the activations' gradients ahead of the backward
// products: dz = dy act'(pre) with the bias gradient's column sums, and the
// gated block's dg = dy up act'(gate), du = dy act(gate).
//
// Bound by memory: the gated block's 4096 x 14336 reads 587 MB and writes
// 235 MB in 124 us (6.6e12 bytes a second).  Sums of before the activation are
// read as the forward saved them, in 32 bits, so that dg and du are rounded
// once, to the type that the tensor cores multiply; a relu whose sum is within
// the rounding of zero may fall on its other side.

#include "heddle_ops.cuh"

namespace hd {
namespace {

// V values of a row in one access of V * sizeof(T) bytes, as floats.
template <class T, int V>
__device__ __forceinline__ void load_values(const T* p, float (&v)[V]) {
    struct alignas(V * sizeof(T)) Pack {
        T t[V];
    } u = *reinterpret_cast<const Pack*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_float(u.t[i]);
}
template <class T, int V>
__device__ __forceinline__ void store_values(T* p, const float (&v)[V]) {
    struct alignas(V * sizeof(T)) Pack {
        T t[V];
    } u;
#pragma unroll
    for (int i = 0; i < V; ++i) u.t[i] = from_float<T>(v[i]);
    *reinterpret_cast<Pack*>(p) = u;
}
template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&v)[V]) {
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 f = *reinterpret_cast<const float4*>(p + i);
            v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = p[i];
    }
}

constexpr int kRowsPerBlock = 8;  // rows in flight, one per warp

// A block takes 32 V columns and the rows of its chunk, a warp every eighth
// of them; the chunk's column sums go to partial[chunk][n].
template <class T, int V>
__global__ void __launch_bounds__(256) act_grad_kernel(ActGradArgs a, float* partial, int64_t rows_per_chunk) {
    allow_dependents();
    await_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t n0 = ((int64_t)blockIdx.x * 32 + lane) * V;
    const int64_t first = blockIdx.y * rows_per_chunk;
    const int64_t last = min(a.m, first + rows_per_chunk);
    float sum[V] = {};
    constexpr int kDepth = V > 1 ? 2 : 4;  // rows in flight a warp
    if (n0 < a.n)
        for (int64_t m = first + warp; m < last; m += kDepth * kRowsPerBlock) {
            float dy[kDepth][V], z[kDepth][V];
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const int64_t r = m + k * kRowsPerBlock;
                if (r >= last) break;
                load_values<T, V>(static_cast<const T*>(a.dy) + r * a.lddy + n0, dy[k]);
                if (a.act != HEDDLE_ACT_NONE) load_floats<V>(a.pre + r * a.ldp + n0, z[k]);
            }
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const int64_t r = m + k * kRowsPerBlock;
                if (r >= last) break;
                if (a.act != HEDDLE_ACT_NONE) {
#pragma unroll
                    for (int i = 0; i < V; ++i) dy[k][i] *= act_slope(z[k][i], a.act);
                }
                if (a.dz) store_values<T, V>(static_cast<T*>(a.dz) + r * a.lddz + n0, dy[k]);
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] += dy[k][i];
            }
        }
    if (!partial) return;
    __shared__ float s[kRowsPerBlock][32 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[warp][lane * V + i] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * V; c += 256) {
        const int64_t n = (int64_t)blockIdx.x * 32 * V + c;
        if (n >= a.n) break;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowsPerBlock; ++w) v += s[w][c];
        partial[blockIdx.y * a.n + n] = v;
    }
}

template <class T>
__global__ void __launch_bounds__(256) column_sum_kernel(const float* partial, int chunks, int64_t n, T* out) {
    allow_dependents();
    await_previous();
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    float v = 0.0f;
#pragma unroll 8
    for (int i = 0; i < chunks; ++i) v += partial[i * n + c];
    out[c] = from_float<T>(v);
}

template <class T, int V>
__global__ void __launch_bounds__(256) gate_grad_kernel(GateGradArgs a) {
    allow_dependents();
    await_previous();
    const int64_t per_row = (a.n + V - 1) / V;
    const int64_t total = a.m * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per_row, n = (i - m * per_row) * V;
        float dy[V], g[V], u[V], dg[V], du[V];
        load_values<T, V>(static_cast<const T*>(a.dy) + m * a.lddy + n, dy);
        load_floats<V>(a.gate + m * a.lds + n, g);
        load_floats<V>(a.up + m * a.lds + n, u);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            dg[j] = dy[j] * u[j] * act_slope(g[j], a.act);
            du[j] = dy[j] * act_value(g[j], a.act);
        }
        store_values<T, V>(static_cast<T*>(a.dg) + m * a.ldo + n, dg);
        store_values<T, V>(static_cast<T*>(a.du) + m * a.ldo + n, du);
    }
}

bool vec16(const void* p, int64_t ld, int size) { return !p || (((uintptr_t)p % 16) == 0 && ld * size % 16 == 0); }

// Chunks of rows: blocks for every SM, at least 32 rows in each.
int64_t row_chunk(const OpContext& x, int64_t m, int64_t blocks_x) {
    const int64_t want = ceil_div(8 * (int64_t)x.num_sms, blocks_x < 1 ? 1 : blocks_x);
    int64_t rows = ceil_div(m, want);
    rows = rows < 32 ? 32 : rows;
    return rows;
}

template <class T>
cudaError_t act_grad(const OpContext& x, const ActGradArgs& a, unsigned char* ws, cudaStream_t st) {
    float* partial = a.dbias ? reinterpret_cast<float*>(ws) : nullptr;
    const bool wide = a.n % 8 == 0 && vec16(a.dy, a.lddy, 2) && vec16(a.dz, a.lddz, 2) &&
                      (a.act == HEDDLE_ACT_NONE || vec16(a.pre, a.ldp, 4));
    const int V = wide ? 8 : 1;
    const int64_t bx = ceil_div(a.n, 32 * V);
    const int64_t rows = row_chunk(x, a.m, bx);
    const int64_t chunks = ceil_div(a.m, rows);
    if (chunks > 65535 || bx > INT32_MAX) return cudaErrorInvalidConfiguration;
    if (chunks) {
        const dim3 grid((unsigned)bx, (unsigned)chunks);
        if (wide)
            launch(x, act_grad_kernel<T, 8>, grid, 256, 0, st, a, partial, rows);
        else
            launch(x, act_grad_kernel<T, 1>, grid, 256, 0, st, a, partial, rows);
    }
    if (a.dbias)  // without rows the sums are zero, and nothing is read
        launch(x, column_sum_kernel<T>, dim3((unsigned)ceil_div(a.n, 256)), 256, 0, st, partial, (int)chunks, a.n,
               static_cast<T*>(a.dbias));
    return cudaGetLastError();
}

template <class T>
cudaError_t gate_grad(const OpContext& x, const GateGradArgs& a, cudaStream_t st) {
    const bool wide = a.n % 8 == 0 && vec16(a.dy, a.lddy, 2) && vec16(a.dg, a.ldo, 2) && vec16(a.du, a.ldo, 2) &&
                      vec16(a.gate, a.lds, 4) && vec16(a.up, a.lds, 4);
    const int64_t total = a.m * ceil_div(a.n, wide ? 8 : 1);
    const int64_t most = (int64_t)x.num_sms * 32;
    const unsigned grid = (unsigned)(ceil_div(total, 256) < most ? ceil_div(total, 256) : most);
    if (wide)
        launch(x, gate_grad_kernel<T, 8>, grid, 256, 0, st, a);
    else
        launch(x, gate_grad_kernel<T, 1>, grid, 256, 0, st, a);
    return cudaGetLastError();
}

}  // namespace

size_t act_grad_scratch(const OpContext& x, const ActGradArgs& a) {
    if (!a.dbias) return 0;
    // the smaller of the two column tilings has the more row chunks
    const int64_t rows = row_chunk(x, a.m, ceil_div(a.n, 256));
    const int64_t rows1 = row_chunk(x, a.m, ceil_div(a.n, 32));
    return align256(sizeof(float) * (size_t)a.n * (size_t)ceil_div(a.m, rows < rows1 ? rows : rows1));
}

cudaError_t launch_act_grad(const OpContext& x, const ActGradArgs& a, unsigned char* ws, cudaStream_t st) {
    return a.dtype == HEDDLE_BF16 ? act_grad<__nv_bfloat16>(x, a, ws, st) : act_grad<__half>(x, a, ws, st);
}

cudaError_t launch_gate_grad(const OpContext& x, const GateGradArgs& a, cudaStream_t st) {
    return a.dtype == HEDDLE_BF16 ? gate_grad<__nv_bfloat16>(x, a, st) : gate_grad<__half>(x, a, st);
}

}  // namespace hd
