// heddle_gemm.cu -- the products of the layer operators with their epilogues
// on the tensor cores.
//
// A persistent CTA per SM computes 128 x BN tiles of C.  One thread streams
// operand tiles of 64 steps into a ring of shared-memory stages by bulk
// tensor copies, one issues the products (128 x BN x 16, sums in tensor
// memory), four warps read finished sums back and run the epilogue while the
// next tile's products fill the other half of tensor memory.

#include <mutex>

#include "heddle_tc.cuh"

namespace hd {

cudaError_t make_map(CUtensorMap* map, const void* base, int dtype, int rank, const uint64_t* dims,
                     const uint64_t* strides, const uint32_t* box) {
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                               const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                               CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Encode encode = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) ==
                cudaSuccess &&
            found == cudaDriverEntryPointSuccess)
            encode = reinterpret_cast<Encode>(fn);
    });
    if (!encode) return cudaErrorNotSupported;
    const cuuint32_t one[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(
        map, dtype == HEDDLE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank,
        const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

namespace {

using namespace tc;

constexpr int BM = 128, BK = 64;
constexpr int kThreads = 256;  // producer, issuer, tensor-memory and spare warp, four epilogue warps
constexpr int kPitch = 36;     // floats per row of an epilogue warp's 32 x 32 transposing tile

struct KernelArgs {
    GemmArgs g;
    int32_t steps;       // 64-wide contraction steps per term
    int32_t terms;
    int32_t a_rows;      // rows of A a copy takes (all 128, or fewer where M is)
    int32_t m_tiles, n_tiles;
    int64_t tiles;
    int32_t vec;         // outputs, residual, bias and saved sums by 16- and 8-byte accesses
    uint32_t* err;
};

template <int BN, int KIND>
struct Shape {
    static constexpr int kStageA = BM * BK * 2, kStageB = BN * BK * 2;
    static constexpr int kStage = kStageA + kStageB;
    static constexpr int kEpi = 4 * 32 * kPitch * 4;
    static constexpr int kStages = (227 * 1024 - 1024 - 512 - kEpi) / kStage < 8 ? (227 * 1024 - 1024 - 512 - kEpi) / kStage : 8;
    static constexpr int kBytes = 1024 + kStages * kStage + kEpi + 512;
    static constexpr int kCols = BN == 256 ? 512 : 2 * BN;  // both halves of tensor memory in use
};

// Tiles in order of groups of 16 tile rows, column by column within one: the
// CTAs at work share few rows of A and columns of B.
__device__ __forceinline__ void tile_at(const KernelArgs& p, int64_t t, int& z, int& tm, int& tn) {
    const int64_t per = (int64_t)p.m_tiles * p.n_tiles;
    z = (int)(t / per);
    t -= z * per;
    const int64_t wide = 16ll * p.n_tiles;
    const int g = (int)(t / wide);
    const int rows = min(16, p.m_tiles - g * 16);
    const int in = (int)(t - g * wide);
    tm = g * 16 + in % rows;
    tn = in / rows;
}

template <class T>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
    return to_float(static_cast<const T*>(p)[i]);
}
template <class T>
__device__ __forceinline__ void load_four(const void* p, int64_t i, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const T*>(p) + i);
    const T* t = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = to_float(t[j]);
}

template <class T>
__device__ __forceinline__ void store_four(T* p, const float (&v)[4]) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        uint2 u;
        T* t = reinterpret_cast<T*>(&u);
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = from_float<T>(v[j]);
        *reinterpret_cast<uint2*>(p) = u;
    }
}

// V sums of one row of C from column n on to what heddle_linear stores.
template <class T, int V>
__device__ __forceinline__ void finish_linear(const GemmArgs& g, int64_t m, int64_t n, float (&c)[V]) {
    if (g.bias) {
        float b[V];
        if constexpr (V == 4)
            load_four<T>(g.bias, n, b);
        else
            b[0] = load_one<T>(g.bias, n);
#pragma unroll
        for (int j = 0; j < V; ++j) c[j] += b[j];
    }
    if (g.pre[0]) {
        if constexpr (V == 4)
            store_four(g.pre[0] + m * g.ldp + n, c);
        else
            g.pre[0][m * g.ldp + n] = c[0];
    }
    if (g.act != HEDDLE_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < V; ++j) c[j] = act_value(c[j], g.act);
    }
    if (g.residual) {
        float r[V];
        if constexpr (V == 4)
            load_four<T>(g.residual, m * g.ldr + n, r);
        else
            r[0] = load_one<T>(g.residual, m * g.ldr + n);
#pragma unroll
        for (int j = 0; j < V; ++j) c[j] += r[j];
    }
}

// A warp's 32 rows x 32 columns from its transposing tile to out: rows of
// memory are written by neighbouring lanes, four values each where the
// alignment allows, else one.
template <class T, bool LINEAR, class TO>
__device__ __forceinline__ void store_block(const KernelArgs& p, TO* out, int64_t ld, int64_t m0, int64_t n0,
                                            const float* t) {
    const GemmArgs& g = p.g;
    const int lane = threadIdx.x % 32;
    __syncwarp();
    if (p.vec && n0 + 32 <= g.N) {
        const int col = (lane % 8) * 4;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = i * 4 + lane / 8;
            if (m0 + row >= g.M) continue;
            const float4 f = *reinterpret_cast<const float4*>(t + row * kPitch + col);
            float c[4] = {f.x, f.y, f.z, f.w};
            if (LINEAR) finish_linear<T, 4>(g, m0 + row, n0 + col, c);
            store_four(out + (m0 + row) * ld + n0 + col, c);
        }
    } else if (n0 + lane < g.N) {
        const int rows = (int)min((int64_t)32, g.M - m0);
        for (int row = 0; row < rows; ++row) {
            float c[1] = {t[row * kPitch + lane]};
            if (LINEAR) finish_linear<T, 1>(g, m0 + row, n0 + lane, c);
            out[(m0 + row) * ld + n0 + lane] = from_float<TO>(c[0]);
        }
    }
    __syncwarp();
}

__device__ __forceinline__ void put_row(float* t, const uint32_t (&v)[32], int lane) {
#pragma unroll
    for (int j = 0; j < 32; j += 4)
        *reinterpret_cast<uint4*>(t + lane * kPitch + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
}

template <int BN, int KIND>
__global__ void __launch_bounds__(kThreads, 1)
    gemm_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap a1,
                const __grid_constant__ CUtensorMap b0, const __grid_constant__ CUtensorMap b1,
                const __grid_constant__ KernelArgs p) {
    using S = Shape<BN, KIND>;
    constexpr bool kAcrossA = KIND == kGemmPair, kAcrossB = KIND == kGemmPair || KIND == kGemmSum;
    constexpr int kOut = KIND == kGemmGated ? BN / 2 : BN;  // columns of C a tile covers
    extern __shared__ unsigned char raw[];
    unsigned char* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    unsigned char* stages = base;
    float* epi = reinterpret_cast<float*>(base + S::kStages * S::kStage);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + S::kStages * S::kStage + S::kEpi);
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages,
                   freed = done + 16;
    volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(bars + 2 * S::kStages + 4);
    uint32_t* tmem_at = const_cast<uint32_t*>(gave_up) + 1;

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(done + 8 * b, 1);
            mbar_init(freed + 8 * b, 4);
        }
        *gave_up = 0;
        mbar_fence_init();
    }
    if (warp == 2) tmem_alloc(smem_u32(tmem_at), S::kCols);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_at;
    const int per_tile = p.steps * p.terms;

    if (warp == 0 && per_tile && elect_one()) {  // producer
        prefetch_map(&a0);
        prefetch_map(&b0);
        int s = 0;
        uint32_t phase = 0;
        bool go = true;
        const uint32_t bytes = (kAcrossA ? S::kStageA : p.a_rows * BK * 2) + S::kStageB;
        for (int64_t t = blockIdx.x; go && t < p.tiles; t += gridDim.x) {
            int z, tm, tn;
            tile_at(p, t, z, tm, tn);
            for (int it = 0; it < per_tile; ++it) {
                if (!(go = mbar_wait(empty + 8 * s, phase ^ 1, gave_up))) break;
                const uint32_t bar = full + 8 * s, sa = smem_u32(stages + s * S::kStage), sb = sa + S::kStageA;
                const bool second = KIND == kGemmSum ? it >= p.steps : KIND == kGemmPair ? z : false;
                const CUtensorMap* ma = second ? &a1 : &a0;
                const CUtensorMap* mb = second ? &b1 : &b0;
                const int k = (KIND == kGemmSum && second ? it - p.steps : it) * BK;
                mbar_expect(bar, bytes);
                if (kAcrossA) {
#pragma unroll
                    for (int j = 0; j < BM / 64; ++j) load_2d(sa + j * 8192, ma, bar, tm * BM + j * 64, k);
                } else {
                    load_2d(sa, ma, bar, k, tm * BM);
                }
                if (KIND == kGemmGated) {
                    load_2d(sb, &b0, bar, k, tn * kOut);
                    load_2d(sb + kOut * BK * 2, &b1, bar, k, tn * kOut);
                } else if (kAcrossB) {
#pragma unroll
                    for (int j = 0; j < BN / 64; ++j) load_2d(sb + j * 8192, mb, bar, tn * BN + j * 64, k);
                } else {
                    load_2d(sb, mb, bar, k, tn * BN);
                }
                if (++s == S::kStages) s = 0, phase ^= 1;
            }
        }
    } else if (warp == 1 && per_tile && elect_one()) {  // issuer
        const uint32_t idesc = instr_desc(p.g.dtype == HEDDLE_BF16, kAcrossA, kAcrossB, BN);
        int s = 0, half = 0;
        uint32_t phase = 0, round[2] = {0, 0};
        bool go = true;
        for (int64_t t = blockIdx.x; go && t < p.tiles; t += gridDim.x) {
            if (!(go = mbar_wait(freed + 8 * half, round[half] ^ 1, gave_up))) break;
            round[half] ^= 1;
            fence_after();
            for (int it = 0; it < per_tile; ++it) {
                if (!(go = mbar_wait(full + 8 * s, phase, gave_up))) break;
                fence_after();
                const uint32_t sa = smem_u32(stages + s * S::kStage), sb = sa + S::kStageA;
                const uint64_t da = smem_desc(sa, 8192), db = smem_desc(sb, 8192);
#pragma unroll
                for (int k = 0; k < BK / 16; ++k)
                    mma_ss(tmem + half * BN, da + (kAcrossA ? 128 * k : 2 * k), db + (kAcrossB ? 128 * k : 2 * k),
                           idesc, it | k);
                commit(empty + 8 * s);
                if (++s == S::kStages) s = 0, phase ^= 1;
            }
            if (go) commit(done + 8 * half);
            half ^= 1;
        }
    } else if (warp >= 4) {  // epilogue
        const int w = warp - 4;
        float* t0 = epi + w * 32 * kPitch;
        int half = 0;
        uint32_t round[2] = {0, 0};
        for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
            int z, tm, tn;
            tile_at(p, t, z, tm, tn);
            if (per_tile) {
                if (!__all_sync(~0u, mbar_wait(done + 8 * half, round[half], gave_up))) break;
                round[half] ^= 1;
                fence_after();
            }
            const uint32_t acc = tmem + half * BN + ((uint32_t)(w * 32) << 16);
            const int64_t m0 = (int64_t)tm * BM + w * 32;
            const bool rows = m0 < p.g.M;
#pragma unroll 1
            for (int c = 0; c < kOut; c += 32) {
                const int64_t n0 = (int64_t)tn * kOut + c;
                if (!rows || n0 >= p.g.N) break;
                uint32_t v[32];
                if (per_tile) {
                    tmem_ld32(acc + c, v);
                    wait_ld();
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0;  // a sum over nothing
                }
                if (KIND == kGemmGated) {
                    uint32_t u[32];
                    if (per_tile) {
                        tmem_ld32(acc + kOut + c, u);
                        wait_ld();
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) u[j] = 0;
                    }
                    if (p.g.pre[0]) {
                        put_row(t0, v, lane);
                        store_block<float, false>(p, p.g.pre[0], p.g.ldp, m0, n0, t0);
                        put_row(t0, u, lane);
                        store_block<float, false>(p, p.g.pre[1], p.g.ldp, m0, n0, t0);
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        v[j] = __float_as_uint(act_value(__uint_as_float(v[j]), p.g.act) * __uint_as_float(u[j]));
                }
                put_row(t0, v, lane);
                constexpr bool kLinear = KIND == kGemmLinear;
                if (p.g.dtype == HEDDLE_BF16)
                    store_block<__nv_bfloat16, kLinear>(p, static_cast<__nv_bfloat16*>(p.g.out[z]), p.g.ldo, m0, n0,
                                                        t0);
                else
                    store_block<__half, kLinear>(p, static_cast<__half*>(p.g.out[z]), p.g.ldo, m0, n0, t0);
            }
            fence_before();
            if (lane == 0) mbar_arrive(freed + 8 * half);
            half ^= 1;
        }
    }
    __syncthreads();
    if (*gave_up) {
        if (threadIdx.x == 0) atomicOr(p.err, kErrOpWait);
        drain();
        __syncthreads();
    }
    if (warp == 2) tmem_free(tmem, S::kCols);
}

// ---------------------------------------------------------------- operands

// Rows of `cols` 16-bit values to rows at a stride of whole 16-byte units.
__global__ void __launch_bounds__(256) lay_out_kernel(const uint16_t* src, int64_t ld, int64_t rows, int64_t cols,
                                                      uint16_t* dst, int64_t dld) {
    const int64_t per = (cols + 7) / 8, total = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per, c = (i - r * per) * 8;
        uint16_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? src[r * ld + c + j] : 0;
        uint4 u;
        u.x = v[0] | (uint32_t)v[1] << 16, u.y = v[2] | (uint32_t)v[3] << 16;
        u.z = v[4] | (uint32_t)v[5] << 16, u.w = v[6] | (uint32_t)v[7] << 16;
        *reinterpret_cast<uint4*>(dst + r * dld + c) = u;
    }
}

// Whether bulk tensor copies read the operand as it is; a single row's
// stride does not matter.
bool copies_as_is(const GemmOperand& o, int64_t rows) {
    return (uintptr_t)o.p % 16 == 0 && (rows == 1 || o.ld % 8 == 0);
}

struct Plan {
    int64_t rows[2], cols[2];  // of A and B as stored
    int a_count, b_count;
};
Plan plan_of(const GemmArgs& g) {
    Plan p{};
    const bool across_a = g.kind == kGemmPair, across_b = across_a || g.kind == kGemmSum;
    p.rows[0] = across_a ? g.K : g.M, p.cols[0] = across_a ? g.M : g.K;
    p.rows[1] = across_b ? g.K : g.N, p.cols[1] = across_b ? g.N : g.K;
    p.a_count = g.kind == kGemmSum || g.kind == kGemmPair ? g.count : 1;
    p.b_count = g.kind == kGemmGated ? 2 : p.a_count;
    return p;
}
bool same(const GemmOperand& a, const GemmOperand& b) { return a.p == b.p && a.ld == b.ld; }

cudaError_t lay_out(GemmOperand& o, int64_t rows, int64_t cols, unsigned char*& ws, const OpContext& x,
                    cudaStream_t st) {
    if (copies_as_is(o, rows)) {
        if (rows == 1) o.ld = ceil_div(cols, 8) * 8;
        return cudaSuccess;
    }
    const int64_t ld = ceil_div(cols, 8) * 8;
    const int64_t units = rows * (ld / 8), most = (int64_t)x.num_sms * 32;
    lay_out_kernel<<<(unsigned)(ceil_div(units, 256) < most ? ceil_div(units, 256) : most), 256, 0, st>>>(
        static_cast<const uint16_t*>(o.p), o.ld, rows, cols, reinterpret_cast<uint16_t*>(ws), ld);
    o = {ws, ld};
    ws += align256((size_t)rows * ld * 2);
    return cudaGetLastError();
}

cudaError_t map_of(CUtensorMap* m, const GemmOperand& o, int dtype, int64_t rows, int64_t cols, int box_rows) {
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)o.ld * 2};
    const uint32_t box[2] = {64, (uint32_t)box_rows};
    return make_map(m, o.p, dtype, 2, dims, strides, box);
}

bool unit16(const void* p, int64_t ld, int size, int unit) {
    return !p || ((uintptr_t)p % unit == 0 && ld * size % unit == 0);
}

template <int BN, int KIND>
cudaError_t run(const OpContext& x, const CUtensorMap (&a)[2], const CUtensorMap (&b)[2], KernelArgs& p,
                cudaStream_t st) {
    using S = Shape<BN, KIND>;
    static_assert(S::kStages >= 3, "the ring needs room");
    constexpr int kOut = KIND == kGemmGated ? BN / 2 : BN;
    p.n_tiles = (int)ceil_div(p.g.N, kOut);
    p.tiles = (int64_t)p.m_tiles * p.n_tiles * (KIND == kGemmPair ? p.g.count : 1);
    auto* k = gemm_kernel<BN, KIND>;
    static std::atomic<uint64_t> asked{0};
    const cudaError_t e = allow_shared(k, S::kBytes, x.device, asked);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)(p.tiles < x.num_sms ? p.tiles : x.num_sms);
    k<<<grid, kThreads, S::kBytes, st>>>(a[0], a[1], b[0], b[1], p);
    return cudaGetLastError();
}

template <int KIND>
cudaError_t run_kind(const OpContext& x, int bn, const CUtensorMap (&a)[2], const CUtensorMap (&b)[2], KernelArgs& p,
                     cudaStream_t st) {
    if (bn == 256) return run<256, KIND>(x, a, b, p, st);
    if (bn == 128) return run<128, KIND>(x, a, b, p, st);
    return run<64, KIND>(x, a, b, p, st);
}

}  // namespace

size_t gemm_scratch(const OpContext&, const GemmArgs& g) {
    const Plan pl = plan_of(g);
    size_t n = 0;
    for (int i = 0; i < pl.a_count; ++i)
        if (!copies_as_is(g.a[i], pl.rows[0])) n += align256((size_t)pl.rows[0] * (ceil_div(pl.cols[0], 8) * 8) * 2);
    for (int i = 0; i < pl.b_count; ++i)
        if (!copies_as_is(g.b[i], pl.rows[1])) n += align256((size_t)pl.rows[1] * (ceil_div(pl.cols[1], 8) * 8) * 2);
    return n;
}

cudaError_t launch_gemm(const OpContext& x, const GemmArgs& args, unsigned char* ws, cudaStream_t st) {
    KernelArgs p{};
    p.g = args;
    GemmArgs& g = p.g;
    const Plan pl = plan_of(g);
    p.steps = (int32_t)ceil_div(g.K, BK);
    p.terms = g.kind == kGemmSum ? g.count : 1;
    p.m_tiles = (int32_t)ceil_div(g.M, BM);
    p.err = x.err;
    const int size = 2;
    p.vec = unit16(g.out[0], g.ldo, size, 8) && unit16(g.out[1], g.ldo, size, 8) &&
            unit16(g.residual, g.ldr, size, 8) && unit16(g.bias, 0, size, 8) && unit16(g.pre[0], g.ldp, 4, 16) &&
            unit16(g.pre[1], g.ldp, 4, 16);

    // columns a tile: the widest whose tiles are enough for every SM
    const int64_t batch = g.kind == kGemmPair ? g.count : 1;
    int bn = 256;
    while (bn > 64 && p.m_tiles * batch * ceil_div(g.N, g.kind == kGemmGated ? bn / 2 : bn) < x.num_sms) bn /= 2;
    const bool across_a = g.kind == kGemmPair, across_b = across_a || g.kind == kGemmSum;
    p.a_rows = across_a ? 64 : (int)(g.M < BM ? ceil_div(g.M, 8) * 8 : BM);
    CUtensorMap a[2] = {}, b[2] = {};
    if (g.K > 0) {
        cudaError_t e = cudaSuccess;
        for (int i = 0; e == cudaSuccess && i < pl.a_count; ++i) {
            e = lay_out(g.a[i], pl.rows[0], pl.cols[0], ws, x, st);
            if (e == cudaSuccess) e = map_of(&a[i], g.a[i], g.dtype, pl.rows[0], pl.cols[0], p.a_rows);
        }
        const int b_box = across_b ? 64 : g.kind == kGemmGated ? bn / 2 : bn;
        for (int i = 0; e == cudaSuccess && i < pl.b_count; ++i) {
            if (i == 1 && same(args.b[0], args.b[1])) {
                b[1] = b[0];
                break;
            }
            e = lay_out(g.b[i], pl.rows[1], pl.cols[1], ws, x, st);
            if (e == cudaSuccess) e = map_of(&b[i], g.b[i], g.dtype, pl.rows[1], pl.cols[1], b_box);
        }
        if (e != cudaSuccess) return e;
    }
    switch (g.kind) {
        case kGemmLinear: return run_kind<kGemmLinear>(x, bn, a, b, p, st);
        case kGemmGated: return run_kind<kGemmGated>(x, bn, a, b, p, st);
        case kGemmSum: return run_kind<kGemmSum>(x, bn, a, b, p, st);
        default: return run_kind<kGemmPair>(x, bn, a, b, p, st);
    }
}

}  // namespace hd
