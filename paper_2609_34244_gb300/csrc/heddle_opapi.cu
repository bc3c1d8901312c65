// heddle_opapi.cu -- the C entries of the layer operators (include/heddle.h):
// checks of the arguments, scratch, launches on the caller's stream.

#include <stdarg.h>
#include <stdio.h>

#include "heddle_ops.cuh"

using hd::OpContext;

namespace {

constexpr int64_t kMaxSize = INT32_MAX;

heddle_status fail(OpContext* x, heddle_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(x->msg, x->msg_size, fmt, ap);
    va_end(ap);
    return st;
}

// Makes the context's device current for the duration of a call.
struct OpDeviceGuard {
    int prev = -1;
    explicit OpDeviceGuard(OpContext* x) {
        x->chained = false;
        x->takes_scratch = false;
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        if (prev != x->device) cudaSetDevice(x->device);
        else prev = -1;
    }
    ~OpDeviceGuard() {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

// Whether a graph is being captured of the stream, or of one that it may not
// run beside.
bool capturing(cudaStream_t st) {
    cudaStreamCaptureStatus status;
    if (cudaStreamIsCapturing(st, &status) == cudaSuccess) return status != cudaStreamCaptureStatusNone;
    cudaGetLastError();
    return true;
}

// At least `need` bytes of scratch, which the last call that took some may
// still be using on another stream: the call waits for its end there.
heddle_status reserve(OpContext* x, size_t need, cudaStream_t st) {
    if (need == 0) return HEDDLE_OK;
    const bool captured = capturing(st);
    if (!x->scratch.reserve(need, captured)) return fail(x, HEDDLE_E_NOMEM, "%zu bytes of operator scratch", need);
    if (captured) return HEDDLE_OK;
    unsigned long long id = 0;
    cudaError_t e = cudaStreamGetId(st, &id);
    if (e == cudaSuccess && x->any_last && id != x->last_stream) e = cudaStreamWaitEvent(st, x->last, 0);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(x, HEDDLE_E_CUDA, "the call's stream: %s", cudaGetErrorString(e));
    }
    x->last_stream = id;
    x->takes_scratch = true;
    return HEDDLE_OK;
}

// The end of a call that may have launched kernels on the stream.
heddle_status done(OpContext* x, cudaError_t e, const char* what, cudaStream_t st) {
    if (x->takes_scratch) {
        const cudaError_t r = cudaEventRecord(x->last, st);
        if (e == cudaSuccess) e = r;
        x->any_last = true;
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(x, HEDDLE_E_CUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    x->msg[0] = 0;
    return HEDDLE_OK;
}

// A call without outputs.
heddle_status nothing(OpContext* x) {
    x->msg[0] = 0;
    return HEDDLE_OK;
}

int elem_size(int32_t dtype) { return dtype == HEDDLE_FP32 ? 4 : 2; }

bool aligned_to(const void* p, int size) { return ((uintptr_t)p & (size - 1)) == 0; }

#define REQUIRE(cond, st, ...)                      \
    do {                                            \
        if (!(cond)) return fail(x, st, __VA_ARGS__); \
    } while (0)

heddle_status check_sizes(OpContext* x, int64_t m, int64_t n, int64_t k, int32_t dtype, int32_t act) {
    REQUIRE(m >= 0 && n >= 0 && k >= 0, HEDDLE_E_ARG, "negative size");
    REQUIRE(m <= kMaxSize && n <= kMaxSize && k <= kMaxSize, HEDDLE_E_LIMIT, "a size exceeds 2^31 - 1");
    REQUIRE(dtype == HEDDLE_BF16 || dtype == HEDDLE_FP16, HEDDLE_E_ARG, "dtype %d: BF16 or FP16", dtype);
    REQUIRE(act >= HEDDLE_ACT_NONE && act <= HEDDLE_ACT_GELU, HEDDLE_E_ARG, "unknown activation %d", act);
    return HEDDLE_OK;
}

// A matrix of rows x cols; empty ones may be null.
heddle_status check_matrix(OpContext* x, const char* name, const void* p, int64_t ld, int64_t rows, int64_t cols,
                           int size) {
    if (rows == 0 || cols == 0) return HEDDLE_OK;
    REQUIRE(p, HEDDLE_E_ARG, "%s is null", name);
    REQUIRE(aligned_to(p, size), HEDDLE_E_ARG, "%s is not aligned to its element", name);
    REQUIRE(ld >= cols, HEDDLE_E_ARG, "row stride %lld of %s is below its %lld columns", (long long)ld, name,
            (long long)cols);
    REQUIRE(ld <= ((int64_t)1 << 36), HEDDLE_E_LIMIT, "row stride of %s exceeds 2^36", name);
    return HEDDLE_OK;
}

#define CHECK(call)                              \
    do {                                         \
        const heddle_status st_ = (call);        \
        if (st_ != HEDDLE_OK) return st_;        \
    } while (0)

heddle_status check_heads(OpContext* x, const char* name, const heddle_heads& t, int64_t b, int64_t n, int64_t h,
                          int64_t d, int size, bool writes) {
    if (b == 0 || n == 0 || h == 0) return HEDDLE_OK;
    REQUIRE(t.data, HEDDLE_E_ARG, "%s is null", name);
    REQUIRE(aligned_to(t.data, size), HEDDLE_E_ARG, "%s is not aligned to its element", name);
    const int64_t lim = (int64_t)1 << 40;
    REQUIRE(t.batch_stride >= 0 && t.token_stride >= 0 && t.head_stride >= 0, HEDDLE_E_ARG, "negative stride of %s",
            name);
    REQUIRE(t.batch_stride <= lim && t.token_stride <= lim && t.head_stride <= lim, HEDDLE_E_LIMIT,
            "a stride of %s exceeds 2^40", name);
    if (writes)  // distinct elements have distinct addresses along every axis
        REQUIRE((b == 1 || t.batch_stride >= d) && (n == 1 || t.token_stride >= d) && (h == 1 || t.head_stride >= d),
                HEDDLE_E_ARG, "a stride of the output %s is below head_dim", name);
    return HEDDLE_OK;
}

heddle_status check_norm_rope(OpContext* x, const heddle_qk_norm_rope_args& a, bool outputs) {
    REQUIRE(a.dtype >= HEDDLE_BF16 && a.dtype <= HEDDLE_FP32, HEDDLE_E_ARG, "unknown dtype %d", a.dtype);
    REQUIRE(a.tokens >= 0 && a.q_heads >= 0 && a.k_heads >= 0, HEDDLE_E_ARG, "negative size");
    REQUIRE(a.head_dim >= 1, HEDDLE_E_ARG, "head_dim %d", a.head_dim);
    REQUIRE(a.head_dim <= 256, HEDDLE_E_LIMIT, "head_dim %d exceeds 256", a.head_dim);
    REQUIRE(a.tokens <= kMaxSize && a.tokens * ((int64_t)a.q_heads + a.k_heads) <= kMaxSize, HEDDLE_E_LIMIT,
            "tokens times heads exceed 2^31 - 1");
    REQUIRE(a.rot_dim >= 0 && a.rot_dim <= a.head_dim && a.rot_dim % 2 == 0, HEDDLE_E_ARG,
            "rot_dim %d: even, at most head_dim", a.rot_dim);
    REQUIRE(a.eps >= 0.0f && isfinite(a.eps), HEDDLE_E_ARG, "eps is negative or not finite");
    if (a.tokens == 0) return HEDDLE_OK;
    const int size = elem_size(a.dtype);
    CHECK(check_heads(x, "q", a.q, 1, a.tokens, a.q_heads, a.head_dim, size, false));
    CHECK(check_heads(x, "k", a.k, 1, a.tokens, a.k_heads, a.head_dim, size, false));
    CHECK(check_heads(x, "q_out", a.q_out, 1, a.tokens, a.q_heads, a.head_dim, size, outputs));
    CHECK(check_heads(x, "k_out", a.k_out, 1, a.tokens, a.k_heads, a.head_dim, size, outputs));
    REQUIRE(!a.q_heads || (a.wq && aligned_to(a.wq, size)), HEDDLE_E_ARG, "wq is null or not aligned");
    REQUIRE(!a.k_heads || (a.wk && aligned_to(a.wk, size)), HEDDLE_E_ARG, "wk is null or not aligned");
    if (a.rot_dim) {
        REQUIRE(a.positions && a.cos && a.sin, HEDDLE_E_ARG, "positions, cos or sin is null");
        REQUIRE(aligned_to(a.positions, 4) && aligned_to(a.cos, 4) && aligned_to(a.sin, 4), HEDDLE_E_ARG,
                "positions, cos or sin is not aligned");
        REQUIRE(a.table_len >= 0, HEDDLE_E_ARG, "negative table_len");
    }
    return HEDDLE_OK;
}

heddle_status check_attention(OpContext* x, const heddle_attention_args& a, bool outputs) {
    REQUIRE(a.dtype == HEDDLE_BF16 || a.dtype == HEDDLE_FP16, HEDDLE_E_ARG, "dtype %d: BF16 or FP16", a.dtype);
    REQUIRE(a.batch >= 0 && a.q_len >= 0 && a.kv_len >= 0, HEDDLE_E_ARG, "negative size");
    REQUIRE(a.q_heads >= 1 && a.kv_heads >= 1 && a.q_heads % a.kv_heads == 0, HEDDLE_E_ARG,
            "%d query heads over %d key heads", a.q_heads, a.kv_heads);
    REQUIRE(a.head_dim >= 1, HEDDLE_E_ARG, "head_dim %d", a.head_dim);
    REQUIRE(a.head_dim <= 256, HEDDLE_E_LIMIT, "head_dim %d exceeds 256", a.head_dim);
    REQUIRE(a.batch <= kMaxSize && a.q_len <= kMaxSize && a.kv_len <= kMaxSize, HEDDLE_E_LIMIT,
            "a size exceeds 2^31 - 1");
    REQUIRE((double)a.batch * a.q_heads * (double)a.q_len < 2147483648.0 &&
                (double)a.batch * a.kv_heads * (double)a.kv_len < 2147483648.0,
            HEDDLE_E_LIMIT, "batch times heads times length exceeds 2^31 - 1");
    REQUIRE(a.window >= 0 && a.sinks >= 0, HEDDLE_E_ARG, "negative window or sinks");
    REQUIRE(a.window <= kMaxSize && a.sinks <= kMaxSize, HEDDLE_E_LIMIT, "window or sinks exceeds 2^31 - 1");
    REQUIRE(isfinite(a.scale), HEDDLE_E_ARG, "scale is not finite");
    CHECK(check_heads(x, "q", a.q, a.batch, a.q_len, a.q_heads, a.head_dim, 2, false));
    CHECK(check_heads(x, "k", a.k, a.batch, a.kv_len, a.kv_heads, a.head_dim, 2, false));
    CHECK(check_heads(x, "v", a.v, a.batch, a.kv_len, a.kv_heads, a.head_dim, 2, false));
    CHECK(check_heads(x, "o", a.o, a.batch, a.q_len, a.q_heads, a.head_dim, 2, outputs));
    REQUIRE(aligned_to(a.lse, 4) && aligned_to(a.q_lens, 4) && aligned_to(a.kv_lens, 4), HEDDLE_E_ARG,
            "lse, q_lens or kv_lens is not aligned");
    return HEDDLE_OK;
}

}  // namespace

extern "C" {

heddle_status heddle_linear(heddle_ctx* ctx, const heddle_linear_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    const heddle_linear_args& a = *args;
    CHECK(check_sizes(x, a.m, a.n, a.k, a.dtype, a.act));
    CHECK(check_matrix(x, "x", a.x, a.ldx, a.m, a.k, 2));
    CHECK(check_matrix(x, "w", a.w, a.ldw, a.n, a.k, 2));
    CHECK(check_matrix(x, "y", a.y, a.ldy, a.m, a.n, 2));
    if (a.residual) CHECK(check_matrix(x, "residual", a.residual, a.ldr, a.m, a.n, 2));
    REQUIRE(aligned_to(a.bias, 2), HEDDLE_E_ARG, "bias is not aligned to its element");
    if (a.pre) CHECK(check_matrix(x, "pre", a.pre, a.ldp, a.m, a.n, 4));
    if (a.m == 0 || a.n == 0) return nothing(x);
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;
    hd::GemmArgs g{};
    g.M = a.m, g.N = a.n, g.K = a.k;
    g.kind = hd::kGemmLinear, g.dtype = a.dtype, g.act = a.act, g.count = 1;
    g.a[0] = {a.x, a.ldx};
    g.b[0] = {a.w, a.ldw};
    g.out[0] = a.y, g.ldo = a.ldy;
    g.bias = a.bias;
    g.residual = a.residual, g.ldr = a.ldr;
    g.pre[0] = a.pre, g.ldp = a.ldp;
    CHECK(reserve(x, hd::gemm_scratch(*x, g), st));
    return done(x, hd::launch_gemm(*x, g, x->scratch.get(), st), "heddle_linear", st);
}

heddle_status heddle_linear_backward(heddle_ctx* ctx, const heddle_linear_grad_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    const heddle_linear_grad_args& a = *args;
    CHECK(check_sizes(x, a.m, a.n, a.k, a.dtype, a.act));
    CHECK(check_matrix(x, "dy", a.dy, a.lddy, a.m, a.n, 2));
    if (a.dw) {
        CHECK(check_matrix(x, "x", a.x, a.ldx, a.m, a.k, 2));
        CHECK(check_matrix(x, "dw", a.dw, a.lddw, a.n, a.k, 2));
    }
    if (a.dx) {
        CHECK(check_matrix(x, "w", a.w, a.ldw, a.n, a.k, 2));
        CHECK(check_matrix(x, "dx", a.dx, a.lddx, a.m, a.k, 2));
    }
    REQUIRE(aligned_to(a.dbias, 2), HEDDLE_E_ARG, "dbias is not aligned to its element");
    if (a.act != HEDDLE_ACT_NONE) CHECK(check_matrix(x, "pre", a.pre, a.ldp, a.m, a.n, 4));
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;

    hd::ActGradArgs ag{};
    ag.m = a.m, ag.n = a.n, ag.dtype = a.dtype, ag.act = a.act;
    ag.dy = a.dy, ag.lddy = a.lddy, ag.pre = a.pre, ag.ldp = a.ldp;
    ag.dbias = a.n ? a.dbias : nullptr;
    const bool own_dz = a.act != HEDDLE_ACT_NONE && (a.dx || a.dw) && a.m && a.n;
    ag.lddz = hd::ceil_div(a.n, 64) * 64;  // rows of whole 128-byte lines for the products
    const size_t dz_bytes = own_dz ? hd::align256((size_t)a.m * ag.lddz * 2) : 0;

    hd::GemmArgs gx{}, gw{};
    gx.M = a.m, gx.N = a.k, gx.K = a.n;
    gx.kind = hd::kGemmSum, gx.dtype = a.dtype, gx.count = 1;
    gx.b[0] = {a.w, a.ldw};
    gx.out[0] = a.dx, gx.ldo = a.lddx;
    gw.M = a.n, gw.N = a.k, gw.K = a.m;
    gw.kind = hd::kGemmPair, gw.dtype = a.dtype, gw.count = 1;
    gw.b[0] = {a.x, a.ldx};
    gw.out[0] = a.dw, gw.ldo = a.lddw;
    const bool want_x = a.dx && a.m && a.k, want_w = a.dw && a.n && a.k;
    // with dz in the scratch its stride counts, whatever its base will be
    gx.a[0] = gw.a[0] = own_dz ? hd::GemmOperand{nullptr, ag.lddz} : hd::GemmOperand{a.dy, a.lddy};
    // places of their own: operands are laid out while the activation's gradient is at work
    const size_t need = (want_x ? hd::gemm_scratch(*x, gx) : 0) + (want_w ? hd::gemm_scratch(*x, gw) : 0);
    const size_t sums_bytes = hd::act_grad_scratch(*x, ag);
    CHECK(reserve(x, dz_bytes + sums_bytes + need, st));
    unsigned char *ws = x->scratch.get(), *sums = ws + dz_bytes, *rest = sums + sums_bytes;
    if (own_dz) {
        ag.dz = ws;
        gx.a[0] = gw.a[0] = {ag.dz, ag.lddz};
    }
    cudaError_t e = cudaSuccess;
    if (ag.dz || ag.dbias) e = hd::launch_act_grad(*x, ag, sums, st);
    hd::GemmArgs* both[2];
    int count = 0;
    if (want_x) both[count++] = &gx;
    if (want_w) both[count++] = &gw;
    if (e == cudaSuccess && a.m && a.n && a.k) e = hd::lay_out_operands(*x, both, count, rest, st);
    if (e == cudaSuccess && want_x) e = hd::launch_gemm(*x, gx, rest, st);
    if (e == cudaSuccess && want_w) e = hd::launch_gemm(*x, gw, rest, st);
    return done(x, e, "heddle_linear_backward", st);
}

heddle_status heddle_gated_ffn(heddle_ctx* ctx, const heddle_gated_ffn_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    const heddle_gated_ffn_args& a = *args;
    CHECK(check_sizes(x, a.m, a.n, a.k, a.dtype, a.act));
    CHECK(check_matrix(x, "x", a.x, a.ldx, a.m, a.k, 2));
    CHECK(check_matrix(x, "w_gate", a.w_gate, a.ldg, a.n, a.k, 2));
    CHECK(check_matrix(x, "w_up", a.w_up, a.ldu, a.n, a.k, 2));
    CHECK(check_matrix(x, "y", a.y, a.ldy, a.m, a.n, 2));
    REQUIRE(!a.gate == !a.up, HEDDLE_E_ARG, "gate and up are given together");
    if (a.gate) {
        CHECK(check_matrix(x, "gate", a.gate, a.lds, a.m, a.n, 4));
        CHECK(check_matrix(x, "up", a.up, a.lds, a.m, a.n, 4));
    }
    if (a.m == 0 || a.n == 0) return nothing(x);
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;
    hd::GemmArgs g{};
    g.M = a.m, g.N = a.n, g.K = a.k;
    g.kind = hd::kGemmGated, g.dtype = a.dtype, g.act = a.act, g.count = 1;
    g.a[0] = {a.x, a.ldx};
    g.b[0] = {a.w_gate, a.ldg};
    g.b[1] = {a.w_up, a.ldu};
    g.out[0] = a.y, g.ldo = a.ldy;
    g.pre[0] = a.gate, g.pre[1] = a.up, g.ldp = a.lds;
    CHECK(reserve(x, hd::gemm_scratch(*x, g), st));
    return done(x, hd::launch_gemm(*x, g, x->scratch.get(), st), "heddle_gated_ffn", st);
}

heddle_status heddle_gated_ffn_backward(heddle_ctx* ctx, const heddle_gated_ffn_grad_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    const heddle_gated_ffn_grad_args& a = *args;
    CHECK(check_sizes(x, a.m, a.n, a.k, a.dtype, a.act));
    REQUIRE(!a.dw_gate == !a.dw_up, HEDDLE_E_ARG, "dw_gate and dw_up are given together");
    CHECK(check_matrix(x, "dy", a.dy, a.lddy, a.m, a.n, 2));
    CHECK(check_matrix(x, "gate", a.gate, a.lds, a.m, a.n, 4));
    CHECK(check_matrix(x, "up", a.up, a.lds, a.m, a.n, 4));
    if (a.dw_gate) {
        CHECK(check_matrix(x, "x", a.x, a.ldx, a.m, a.k, 2));
        CHECK(check_matrix(x, "dw_gate", a.dw_gate, a.lddw, a.n, a.k, 2));
        CHECK(check_matrix(x, "dw_up", a.dw_up, a.lddw, a.n, a.k, 2));
    }
    if (a.dx) {
        CHECK(check_matrix(x, "w_gate", a.w_gate, a.ldg, a.n, a.k, 2));
        CHECK(check_matrix(x, "w_up", a.w_up, a.ldu, a.n, a.k, 2));
        CHECK(check_matrix(x, "dx", a.dx, a.lddx, a.m, a.k, 2));
    }
    const bool want_x = a.dx && a.m && a.k, want_w = a.dw_gate && a.n && a.k;
    if (!want_x && !want_w) return nothing(x);
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;

    const int64_t ld = hd::ceil_div(a.n, 64) * 64;  // rows of whole 128-byte lines for the products
    const size_t half = hd::align256((size_t)a.m * ld * 2);
    hd::GemmArgs gx{}, gw{};
    gx.M = a.m, gx.N = a.k, gx.K = a.n;
    gx.kind = hd::kGemmSum, gx.dtype = a.dtype, gx.count = 2;
    gx.b[0] = {a.w_gate, a.ldg};
    gx.b[1] = {a.w_up, a.ldu};
    gx.out[0] = a.dx, gx.ldo = a.lddx;
    gw.M = a.n, gw.N = a.k, gw.K = a.m;
    gw.kind = hd::kGemmPair, gw.dtype = a.dtype, gw.count = 2;
    gw.b[0] = gw.b[1] = {a.x, a.ldx};
    gw.out[0] = a.dw_gate, gw.out[1] = a.dw_up, gw.ldo = a.lddw;
    // dg and du in the scratch: their stride counts, whatever the base will be
    gx.a[0] = gx.a[1] = gw.a[0] = gw.a[1] = {nullptr, ld};
    const size_t need = (want_x ? hd::gemm_scratch(*x, gx) : 0) + (want_w ? hd::gemm_scratch(*x, gw) : 0);
    CHECK(reserve(x, 2 * half + need, st));
    unsigned char *ws = x->scratch.get(), *rest = ws + 2 * half;
    gx.a[0] = gw.a[0] = {ws, ld};
    gx.a[1] = gw.a[1] = {ws + half, ld};

    hd::GateGradArgs gg{};
    gg.m = a.m, gg.n = a.n, gg.dtype = a.dtype, gg.act = a.act;
    gg.dy = a.dy, gg.lddy = a.lddy, gg.gate = a.gate, gg.up = a.up, gg.lds = a.lds;
    gg.dg = ws, gg.du = ws + half, gg.ldo = ld;
    cudaError_t e = a.m && a.n ? hd::launch_gate_grad(*x, gg, st) : cudaSuccess;
    hd::GemmArgs* both[2];
    int count = 0;
    if (want_x) both[count++] = &gx;
    if (want_w) both[count++] = &gw;
    if (e == cudaSuccess && a.m && a.n && a.k) e = hd::lay_out_operands(*x, both, count, rest, st);
    if (e == cudaSuccess && want_x) e = hd::launch_gemm(*x, gx, rest, st);
    if (e == cudaSuccess && want_w) e = hd::launch_gemm(*x, gw, rest, st);
    return done(x, e, "heddle_gated_ffn_backward", st);
}

heddle_status heddle_qk_norm_rope(heddle_ctx* ctx, const heddle_qk_norm_rope_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    CHECK(check_norm_rope(x, *args, true));
    if (args->tokens == 0 || args->q_heads + args->k_heads == 0) return nothing(x);
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;
    return done(x, hd::launch_qk_norm_rope(*x, *args, st), "heddle_qk_norm_rope", st);
}

heddle_status heddle_qk_norm_rope_backward(heddle_ctx* ctx, const heddle_qk_norm_rope_grad_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    const heddle_qk_norm_rope_args& a = args->fwd;
    CHECK(check_norm_rope(x, a, false));
    const int size = elem_size(a.dtype);
    CHECK(check_heads(x, "dq", args->dq, 1, a.tokens, a.q_heads, a.head_dim, size, true));
    CHECK(check_heads(x, "dk", args->dk, 1, a.tokens, a.k_heads, a.head_dim, size, true));
    REQUIRE(args->dwq && args->dwk, HEDDLE_E_ARG, "dwq or dwk is null");
    REQUIRE(aligned_to(args->dwq, 4) && aligned_to(args->dwk, 4), HEDDLE_E_ARG, "dwq or dwk is not aligned");
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;
    CHECK(reserve(x, hd::qk_norm_rope_grad_scratch(*x, *args), st));
    return done(x, hd::launch_qk_norm_rope_grad(*x, *args, x->scratch.get(), st),
                "heddle_qk_norm_rope_backward", st);
}

heddle_status heddle_attention(heddle_ctx* ctx, const heddle_attention_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    CHECK(check_attention(x, *args, true));
    if (args->batch == 0 || args->q_len == 0) return nothing(x);
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;
    CHECK(reserve(x, hd::attention_scratch(*x, *args), st));
    return done(x, hd::launch_attention(*x, *args, x->scratch.get(), st), "heddle_attention", st);
}

heddle_status heddle_attention_backward(heddle_ctx* ctx, const heddle_attention_grad_args* args, void* stream) {
    if (!ctx) return HEDDLE_E_ARG;
    OpContext* x = heddle_op_context(ctx);
    REQUIRE(args, HEDDLE_E_ARG, "args is null");
    const heddle_attention_args& a = args->fwd;
    CHECK(check_attention(x, a, false));
    CHECK(check_heads(x, "d_o", args->d_o, a.batch, a.q_len, a.q_heads, a.head_dim, 2, false));
    CHECK(check_heads(x, "dq", args->dq, a.batch, a.q_len, a.q_heads, a.head_dim, 2, true));
    CHECK(check_heads(x, "dk", args->dk, a.batch, a.kv_len, a.kv_heads, a.head_dim, 2, true));
    CHECK(check_heads(x, "dv", args->dv, a.batch, a.kv_len, a.kv_heads, a.head_dim, 2, true));
    REQUIRE(a.lse || a.batch * a.q_len == 0, HEDDLE_E_ARG, "lse is null");
    if (a.batch == 0 || (a.q_len == 0 && a.kv_len == 0)) return nothing(x);
    OpDeviceGuard guard(x);
    cudaStream_t st = (cudaStream_t)stream;
    // room to keep the scores' gradients, or without them where that is refused
    const size_t most = hd::attention_grad_scratch(*x, *args, true);
    const size_t least = hd::attention_grad_scratch(*x, *args, false);
    bool keep = most <= x->scratch.size();
    if (!keep && most > least && x->refusal.worth_asking(most)) {
        keep = x->scratch.reserve(most, capturing(st), true);
        keep ? x->refusal.granted(most) : x->refusal.refused(most);
    }
    CHECK(reserve(x, keep ? most : least, st));
    return done(x, hd::launch_attention_grad(*x, *args, x->scratch.get(), keep, st),
                "heddle_attention_backward", st);
}

}  // extern "C"
