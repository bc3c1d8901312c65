// heddle_gemv.cu -- the forward products of one or two rows, and of up to eight
// with few weights: the weights' stream, and the latency of its start and end,
// are the time.
//
// A block of eight warps takes four rows of weights (two of each matrix of
// the gated block); every warp an eighth of the contraction, 16 bytes a lane
// and row, so that a block's whole stream is in flight at once.  Products
// are summed in 32 bits per lane, across the lanes, then across the warps in
// order.  One row of 4096 x 4096 bfloat16 weights, a call in a graph of them:
// 7.5 us where the weights come from memory (4.4e12 bytes a second), 4.9 where
// L2 holds them; the tensor cores' kernel takes 11.5 and 10.1.  Every row costs
// as many multiply-adds again (gemv_takes).

#include "heddle_ops.cuh"

namespace hd {
namespace {

constexpr int kRows = 4, kWarps = 8;

template <class T>
__device__ __forceinline__ void to_floats(const uint4& u, float (&v)[8]) {
    const T* t = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(t[i]);
}

template <class T, int M, bool GATED>
__global__ void __launch_bounds__(256) gemv_kernel(const __grid_constant__ GemmArgs g) {
    __shared__ float part[kWarps][kRows * M];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    constexpr int kOut = GATED ? kRows / 2 : kRows;  // columns of C a block takes at a time
    const int64_t units = g.K / 8;
    for (int64_t n0 = (int64_t)blockIdx.x * kOut; n0 < g.N; n0 += (int64_t)gridDim.x * kOut) {
        const T* w[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int64_t n = min(n0 + r % kOut, g.N - 1);  // rows past the last are not stored
            const GemmOperand& b = g.b[GATED ? r / kOut : 0];
            w[r] = static_cast<const T*>(b.p) + n * b.ld;
        }
        float acc[kRows][M] = {};
#pragma unroll(M <= 2 ? 2 : 1)
        for (int64_t u = warp * 32 + lane; u < units; u += kWarps * 32) {
            uint4 wv[kRows], xv[M];
#pragma unroll
            for (int r = 0; r < kRows; ++r) wv[r] = *reinterpret_cast<const uint4*>(w[r] + u * 8);
#pragma unroll
            for (int m = 0; m < M; ++m)
                xv[m] = *reinterpret_cast<const uint4*>(static_cast<const T*>(g.a[0].p) +
                                                        (M <= 2 ? m : min((int64_t)m, g.M - 1)) * g.a[0].ld + u * 8);
            float wf[kRows][8];
#pragma unroll
            for (int r = 0; r < kRows; ++r) to_floats<T>(wv[r], wf[r]);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                float xf[8];
                to_floats<T>(xv[m], xf);
#pragma unroll
                for (int r = 0; r < kRows; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[r][m] = fmaf(wf[r][i], xf[i], acc[r][m]);
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m) {
                const float s = warp_sum(acc[r][m]);
                if (lane == 0) part[warp][r * M + m] = s;
            }
        __syncthreads();
        const int m = threadIdx.x % M, c = threadIdx.x / M;
        if (c < kOut && n0 + c < g.N && m < g.M) {
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                s[0] += part[k][c * M + m];
                if (GATED) s[1] += part[k][(kOut + c) * M + m];
            }
            const int64_t n = n0 + c;
            float y;
            if (GATED) {
                if (g.pre[0]) g.pre[0][m * g.ldp + n] = s[0], g.pre[1][m * g.ldp + n] = s[1];
                y = act_value(s[0], g.act) * s[1];
            } else {
                if (g.bias) s[0] += to_float(static_cast<const T*>(g.bias)[n]);
                if (g.pre[0]) g.pre[0][m * g.ldp + n] = s[0];
                y = act_value(s[0], g.act);
                if (g.residual) y += to_float(static_cast<const T*>(g.residual)[m * g.ldr + n]);
            }
            static_cast<T*>(g.out[0])[m * g.ldo + n] = from_float<T>(y);
        }
        __syncthreads();
    }
}

template <class T, int M>
void launch(const OpContext& x, const GemmArgs& g, cudaStream_t st) {
    const bool gated = g.kind == kGemmGated;
    const int64_t want = ceil_div(g.N, gated ? kRows / 2 : kRows), most = (int64_t)x.num_sms * 16;
    const unsigned grid = (unsigned)(want < most ? want : most);
    if (gated)
        gemv_kernel<T, M, true><<<grid, 256, 0, st>>>(g);
    else
        gemv_kernel<T, M, false><<<grid, 256, 0, st>>>(g);
}

template <class T>
cudaError_t launch_rows(const OpContext& x, const GemmArgs& g, cudaStream_t st) {
    if (g.M == 1)
        launch<T, 1>(x, g, st);
    else if (g.M == 2)
        launch<T, 2>(x, g, st);
    else if (g.M <= 4)
        launch<T, 4>(x, g, st);
    else
        launch<T, 8>(x, g, st);
    return cudaGetLastError();
}

bool units16(const GemmOperand& o, int64_t rows) { return (uintptr_t)o.p % 16 == 0 && (rows == 1 || o.ld % 8 == 0); }

}  // namespace

// All times with the weights from memory.  One or two rows always: at 4096 x
// 4096 7.5 and 11.4 us against 11.5 and 11.9 on the tensor cores.  Up to four or
// eight where the rows of weights are so few that tiles of them leave most SMs
// idle, each with the whole contraction to itself: four rows of 8192 by 64, 2048
// and 4096 columns 6.2, 12.6 and 18.6 us against 17.0, 17.5 and 18.7; eight by
// 64 and 2048 8.1 and 17.0 against 17.0 and 17.5.  More weights than that cost
// this kernel their multiply-adds: 14336 x 4096 with four rows 33 against 26.
bool gemv_takes(const OpContext& x, const GemmArgs& g) {
    if (g.kind != kGemmLinear && g.kind != kGemmGated) return false;
    const int64_t weights = g.kind == kGemmGated ? 2 * g.N : g.N, rows = g.M <= 4 ? 4 : 8;
    return (g.M <= 2 || (g.M <= 8 && weights * rows <= 108ll * x.num_sms)) && g.K > 0 && g.K % 8 == 0 &&
           units16(g.a[0], g.M) && units16(g.b[0], g.N) && (g.kind == kGemmLinear || units16(g.b[1], g.N));
}

cudaError_t launch_gemv(const OpContext& x, const GemmArgs& g, cudaStream_t st) {
    return g.dtype == HEDDLE_BF16 ? launch_rows<__nv_bfloat16>(x, g, st) : launch_rows<__half>(x, g, st);
}

}  // namespace hd
