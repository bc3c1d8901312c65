// heddle_gemm.cu -- the products of the layer operators with their epilogues.

#include "heddle_ops.cuh"

namespace hd {
namespace {

constexpr int kTile = 64, kStep = 16;

// C tile of 64 x 64, 4 x 4 values a thread, operands staged in shared memory
// in steps of 16, sums in 32 bits.  Any stride and size.
template <class T>
__global__ void __launch_bounds__(256) gemm_kernel(GemmArgs g) {
    __shared__ float sa[kStep][kTile + 4], sb[2][kStep][kTile + 4];
    const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
    const int z = blockIdx.z;
    const bool gated = g.kind == kGemmGated;
    const bool amn = g.kind == kGemmPair, bmn = g.kind == kGemmPair || g.kind == kGemmSum;
    const int terms = g.kind == kGemmSum ? g.count : 1;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[2][4][4] = {};
    for (int t = 0; t < terms; ++t) {
        const GemmOperand a = g.a[g.kind == kGemmPair ? z : t];
        for (int64_t k0 = 0; k0 < g.K; k0 += kStep) {
            for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
                const int ra = amn ? i % kTile : i / kStep, ka = amn ? i / kTile : i % kStep;
                float v = 0.0f;
                if (m0 + ra < g.M && k0 + ka < g.K) {
                    const int64_t at = amn ? (k0 + ka) * a.ld + m0 + ra : (m0 + ra) * a.ld + k0 + ka;
                    v = to_float(static_cast<const T*>(a.p)[at]);
                }
                sa[ka][ra] = v;
                const int rb = bmn ? i % kTile : i / kStep, kb = bmn ? i / kTile : i % kStep;
                for (int d = 0; d < (gated ? 2 : 1); ++d) {
                    const GemmOperand b = g.b[gated ? d : g.kind == kGemmPair ? z : t];
                    v = 0.0f;
                    if (n0 + rb < g.N && k0 + kb < g.K) {
                        const int64_t at = bmn ? (k0 + kb) * b.ld + n0 + rb : (n0 + rb) * b.ld + k0 + kb;
                        v = to_float(static_cast<const T*>(b.p)[at]);
                    }
                    sb[d][kb][rb] = v;
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kStep; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[0][i][j] += sa[k][ty * 4 + i] * sb[0][k][tx * 4 + j];
                        if (gated) acc[1][i][j] += sa[k][ty * 4 + i] * sb[1][k][tx * 4 + j];
                    }
            __syncthreads();
        }
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
            if (m >= g.M || n >= g.N) continue;
            float v = acc[0][i][j];
            if (g.kind == kGemmLinear) {
                if (g.bias) v += to_float(static_cast<const T*>(g.bias)[n]);
                if (g.pre[0]) g.pre[0][m * g.ldp + n] = v;
                v = act_value(v, g.act);
                if (g.residual) v += to_float(static_cast<const T*>(g.residual)[m * g.ldr + n]);
            } else if (gated) {
                if (g.pre[0]) {
                    g.pre[0][m * g.ldp + n] = v;
                    g.pre[1][m * g.ldp + n] = acc[1][i][j];
                }
                v = act_value(v, g.act) * acc[1][i][j];
            }
            static_cast<T*>(g.out[z])[m * g.ldo + n] = from_float<T>(v);
        }
}

}  // namespace

size_t gemm_scratch(const OpContext&, const GemmArgs&) { return 0; }

cudaError_t launch_gemm(const OpContext&, const GemmArgs& g, unsigned char*, cudaStream_t st) {
    const int64_t gx = ceil_div(g.N, kTile), gy = ceil_div(g.M, kTile);
    if (gy > 65535) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)gx, (unsigned)gy, g.kind == kGemmPair ? g.count : 1);
    if (g.dtype == HEDDLE_BF16)
        gemm_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(g);
    else
        gemm_kernel<__half><<<grid, 256, 0, st>>>(g);
    return cudaGetLastError();
}

}  // namespace hd
