// heddle_ops.cuh -- definitions shared by the layer operators' translation
// units: element types, activations, the context's part that operators use
// and the launchers behind the C entries (heddle_opapi.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <utility>

#include "heddle.h"
#include "heddle_launch.cuh"
#include "heddle_scratch.cuh"

namespace hd {

// Device error flags of the operators (heddle_device_errors).
constexpr uint32_t kErrOpWait = 16u;      // a wait inside an operator ran out
constexpr uint32_t kErrOpPosition = 32u;  // a position outside its rotation table

constexpr int kSched = 4;

struct DeviceMemory {
    static void* allocate(size_t size) {
        // allowed during a capture, and no part of the graph
        cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
        cudaThreadExchangeStreamCaptureMode(&mode);
        void* p = nullptr;
        const cudaError_t e = cudaMalloc(&p, size);
        cudaThreadExchangeStreamCaptureMode(&mode);
        if (e == cudaSuccess) return p;
        cudaGetLastError();
        return nullptr;
    }
    static void release(void* p) { cudaFree(p); }
};

// What an operator call uses of its context.
struct OpContext {
    int device = 0;
    int num_sms = 0;
    uint32_t* err = nullptr;  // device error flags
    // two counters of kernels that hand out work, zero between launches, and two
    // maxima as floats' bits (attention's gradients)
    int32_t* sched = nullptr;
    Scratch<DeviceMemory> scratch;
    Refusal refusal;  // of scratch that a call can do without
    // the end of the last call that took scratch, on the stream of that id; none in graphs
    cudaEvent_t last = nullptr;
    unsigned long long last_stream = 0;
    bool any_last = false, takes_scratch = false;  // takes_scratch: the call at hand does
    char* msg = nullptr;
    size_t msg_size = 0;
    mutable bool chained = false;  // the call has launched a kernel already
};

// A kernel of a call.  All but the first start under the end of the one before
// (their launch, barriers and tensor memory cost a few microseconds): every
// kernel allows that at its start, and waits in some thread of every block,
// whatever its share of the work, before it reads what the call's kernels
// wrote and before it writes.  The caller's own tensors may be read earlier.
template <class... P, class... A>
cudaError_t launch(const OpContext& x, void (*kernel)(P...), dim3 grid, int block, size_t smem, cudaStream_t st,
                   A&&... args) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = x.chained ? 1 : 0;
    x.chained = true;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

template <class T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float(float v) { return v; }
template <>
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }

__device__ __forceinline__ float act_value(float z, int act) {
    if (act == HEDDLE_ACT_SILU) return z / (1.0f + expf(-z));
    if (act == HEDDLE_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    if (act == HEDDLE_ACT_RELU) return z < 0.0f ? 0.0f : z;  // NaN stays
    return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
    if (act == HEDDLE_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    if (act == HEDDLE_ACT_GELU)
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    if (act == HEDDLE_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    return 1.0f;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// ------------------------------------------------------------------ products

// One operand of a product C[M][N] = sum over K: row r, step k at
// p[r * ld + k], or at p[k * ld + r] where the rows are contiguous (mn).
struct GemmOperand {
    const void* p;
    int64_t ld;
};

// kLinear: out = act(A B^T + bias) + residual, the sum before act to pre.
// kGated: out = act(A B0^T) * (A B1^T), both products to pre[0], pre[1].
// kSum: out = A0 B0 + A1 B1 (terms of them; the B rows contiguous).
// kPair: out[z] = A[z]^T B[z] (batch of them; both rows contiguous).
enum GemmKind { kGemmLinear, kGemmGated, kGemmSum, kGemmPair };

struct GemmArgs {
    int64_t M, N, K;
    int32_t kind, dtype, act, count;  // count: terms (kSum) or batch (kPair)
    GemmOperand a[2], b[2];
    void* out[2];
    int64_t ldo;
    const void* bias;
    const void* residual;
    int64_t ldr;
    float* pre[2];
    int64_t ldp;
};
size_t gemm_scratch(const OpContext& x, const GemmArgs& g);
// Lays out in `ws`, in one launch, what bulk tensor copies do not take as it
// is of several products' operands (at most four), which then name the copies.
cudaError_t lay_out_operands(const OpContext& x, GemmArgs* const* list, int count, unsigned char* ws, cudaStream_t st);
cudaError_t launch_gemm(const OpContext& x, const GemmArgs& g, unsigned char* ws, cudaStream_t st);

// Forward products of few rows in whole 16-byte units, without the tensor
// cores (heddle_gemv.cu).
bool gemv_takes(const OpContext& x, const GemmArgs& g);
cudaError_t launch_gemv(const OpContext& x, const GemmArgs& g, cudaStream_t st);

// dz = dy act'(pre) (dz null: not written), partial column sums of it
struct ActGradArgs {
    int64_t m, n;
    int32_t dtype, act;
    const void* dy;
    int64_t lddy;
    const float* pre;
    int64_t ldp;
    void* dz;
    int64_t lddz;
    void* dbias;
};
size_t act_grad_scratch(const OpContext& x, const ActGradArgs& a);
cudaError_t launch_act_grad(const OpContext& x, const ActGradArgs& a, unsigned char* ws, cudaStream_t st);

struct GateGradArgs {
    int64_t m, n;
    int32_t dtype, act;
    const void* dy;
    int64_t lddy;
    const float* gate;
    const float* up;
    int64_t lds;
    void* dg;
    void* du;
    int64_t ldo;
};
cudaError_t launch_gate_grad(const OpContext& x, const GateGradArgs& a, cudaStream_t st);

// --------------------------------------------------------------- other passes

cudaError_t launch_qk_norm_rope(const OpContext& x, const heddle_qk_norm_rope_args& a, cudaStream_t st);
size_t qk_norm_rope_grad_scratch(const OpContext& x, const heddle_qk_norm_rope_grad_args& a);
cudaError_t launch_qk_norm_rope_grad(const OpContext& x, const heddle_qk_norm_rope_grad_args& a, unsigned char* ws,
                                     cudaStream_t st);

size_t attention_scratch(const OpContext& x, const heddle_attention_args& a);
cudaError_t launch_attention(const OpContext& x, const heddle_attention_args& a, unsigned char* ws, cudaStream_t st);
// keep: with room for the scores' gradients between the backward's passes
size_t attention_grad_scratch(const OpContext& x, const heddle_attention_grad_args& a, bool keep);
cudaError_t launch_attention_grad(const OpContext& x, const heddle_attention_grad_args& a, unsigned char* ws, bool keep,
                                  cudaStream_t st);

}  // namespace hd

// The operators' part of a context (heddle_capi.cu).
hd::OpContext* heddle_op_context(heddle_ctx* ctx);
