// heddle_gemm.cu -- the products of the layer operators with their epilogues
// on the tensor cores.
//
// A persistent CTA per SM computes 128 x BN tiles of C, or a pair of CTAs
// 256 x 256 tiles, each with half of the rows of A and of B in its shared
// memory: a third less to fetch from L2 than two CTAs alone.  One thread
// streams operand tiles of 64 steps into a ring of shared-memory stages by
// bulk tensor copies, one issues the products (sums in tensor memory), eight
// warps read finished sums back and run the epilogue while the next tile's
// products fill the other half of tensor memory.  With few rows the stages
// hold as many rows of A as there are, so that the ring holds more of B,
// whose stream from memory is then the time.
//
// Bound by the tensor cores where rows are many: 2048 x 4096 x 14336 in
// bfloat16 with the residual 130 us (1.85e15 operations a second), its
// gradients 124 us each (1.94e15); the gated block's 4096 x 14336 x 4096
// 515 us forward with both sums saved in 32 bits (1.87e15), 550 us for dx,
// 490 us for the weights' gradients (1.96e15: single CTAs of 128 x 256 reached
// 1.4e15, the copies from L2 being their time).  With 16 rows of the gated
// block the weights' stream takes 40 us (5.9e12 bytes a second).  Bound by
// their epilogue where the contraction is short (choose_tile).

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
constexpr int kEpiWarps = 8;   // two for every 32 rows of a tile, half of its columns each
constexpr int kThreads = 128 + 32 * kEpiWarps;  // producer, issuer, tensor-memory and spare warp, epilogue
constexpr int kCols = 16;      // columns that an epilogue warp takes at a time
constexpr int kPitch = 20;     // floats per row of its 32 x 16 transposing tile

struct KernelArgs {
    GemmArgs g;
    int32_t steps;       // 64-wide contraction steps per term
    int32_t terms;
    int32_t a_rows;      // rows of A a copy takes (all 128, or fewer where M is)
    int32_t stages, stage;  // of the ring, and its bytes each
    int32_t deep;           // 64-wide steps a stage holds: 1, or kDeep where rows are few
    int32_t m_tiles, n_tiles;
    int64_t tiles;
    int32_t vec;         // outputs, residual, bias and saved sums by 16- and 8-byte accesses
    int32_t direct;      // outputs, residual and saved sums by 32-byte accesses, a row a lane
    uint32_t* err;
};

constexpr int kMaxStages = 32;
// With few rows a step's products are short and its barriers are the time, so
// a stage holds four, of one copy an operand where that gives the layout.
constexpr int kDeep = 4;
constexpr int kEpi = kEpiWarps * 32 * kPitch * 4;
constexpr int kBarBytes = 16 * kMaxStages + 64;
constexpr int kShared = 227 * 1024;  // all that a CTA may take
constexpr int kRing = kShared - 1024 - kEpi - kBarBytes;

template <int BN, bool PAIR>
struct Shape {
    static constexpr int kTileM = PAIR ? 2 * BM : BM;
    static constexpr int kRowsB = PAIR ? BN / 2 : BN;  // rows of B in this CTA
    static constexpr int kStageA = BM * BK * 2, kStageB = kRowsB * BK * 2;
    static constexpr int kTmem = BN > 128 ? 512 : 2 * BN;  // both halves of tensor memory in use
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

// Sixteen columns of a row as they come from tensor memory, a row a lane: the
// 32 bytes that memory is written by.  Through shared memory a warp's rows come
// out side by side, but each block waits for the one before: weights' gradients
// of 17 rows, 243 MB and all of it output, 140 us, this way 106, and 116 with
// rows of 128 bytes gathered in shared memory.
__device__ __forceinline__ void store_32(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(__cvta_generic_to_global(p)),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void load_32(const void* p, uint32_t* v) {
    const uint4 a = *static_cast<const uint4*>(p), b = *(static_cast<const uint4*>(p) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
template <class T>
__device__ __forceinline__ void finish_row(const KernelArgs& p, void* out, int64_t m, int64_t n0, bool live,
                                           uint32_t (&v)[kCols], const uint32_t (&r)[kCols], bool linear) {
    const GemmArgs& g = p.g;
    if (linear && g.bias) {
        uint32_t b[8];
        load_32(static_cast<const T*>(g.bias) + n0, b);
#pragma unroll
        for (int j = 0; j < kCols; ++j)
            v[j] = __float_as_uint(__uint_as_float(v[j]) + to_float(reinterpret_cast<const T*>(b)[j]));
    }
    if (linear && g.residual) {
#pragma unroll
        for (int j = 0; j < kCols; ++j)
            v[j] = __float_as_uint(__uint_as_float(v[j]) + to_float(reinterpret_cast<const T*>(r)[j]));
    }
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < kCols; ++j) reinterpret_cast<T*>(w)[j] = from_float<T>(__uint_as_float(v[j]));
    if (live) store_32(static_cast<T*>(out) + m * g.ldo + n0, w);
}

// How a warp goes over a block of 32 rows x 16 columns: neighbouring lanes on
// a row of memory, four values each where the alignment allows, else one.
struct Walk {
    int row, col;  // a lane's first; the others lie `step` rows apart
    bool four;
    __device__ Walk(const KernelArgs& p, int64_t n0) {
        const int lane = threadIdx.x % 32;
        four = p.vec && n0 + kCols <= p.g.N;
        row = four ? lane / 4 : lane / kCols;
        col = four ? lane % 4 * 4 : lane % kCols;
    }
    // of a lane's 4 or 16 rows, those that lie in C
    __device__ int rows(const KernelArgs& p, int64_t m0, int64_t n0) const {
        const int64_t left = p.g.M - m0 - row;
        if (left <= 0 || n0 + col >= p.g.N) return 0;
        return four ? (int)min((left + 7) / 8, (int64_t)4) : (int)min((left + 1) / 2, (int64_t)16);
    }
};

// The block's residual, fetched before the sums are waited for: it is added
// last, and a load behind the stores of another row would wait for memory.
__device__ __forceinline__ void fetch_residual(const KernelArgs& p, int64_t m0, int64_t n0, uint32_t (&r)[kCols]) {
    const Walk w(p, n0);
    const int n = w.rows(p, m0, n0);
    const uint16_t* at = static_cast<const uint16_t*>(p.g.residual) + (m0 + w.row) * p.g.ldr + n0 + w.col;
    if (w.four) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 u = i < n ? *reinterpret_cast<const uint2*>(at + i * 8 * p.g.ldr) : make_uint2(0, 0);
            r[2 * i] = u.x, r[2 * i + 1] = u.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i] = i < n ? at[i * 2 * p.g.ldr] : 0;
    }
}

// heddle_linear's bias, saved sums and activation on a block in its
// transposing tile.  A loop, not unrolled: sixteen copies of an activation
// waited for their instructions (1023 x 2047 x 4099 with gelu: 42 us).
template <class T>
__device__ __forceinline__ void activate_block(const KernelArgs& p, int64_t m0, int64_t n0, float* t) {
    const GemmArgs& g = p.g;
    const Walk w(p, n0);
    const int n = w.rows(p, m0, n0);
    t += w.row * kPitch + w.col;
    float* pre = g.pre[0] ? g.pre[0] + (m0 + w.row) * g.ldp + n0 + w.col : nullptr;
    if (w.four) {
        float b[4] = {};
        if (g.bias) {
            const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const T*>(g.bias) + n0 + w.col);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = to_float(reinterpret_cast<const T*>(&u)[j]);
        }
#pragma unroll 1
        for (int i = 0; i < n; ++i, t += 8 * kPitch) {
            float4 f = *reinterpret_cast<const float4*>(t);
            float c[4] = {f.x + b[0], f.y + b[1], f.z + b[2], f.w + b[3]};
            if (pre) store_four(pre + i * 8 * g.ldp, c);
            if (g.act != HEDDLE_ACT_NONE) {
#pragma unroll
                for (int j = 0; j < 4; ++j) c[j] = act_value(c[j], g.act);
            }
            *reinterpret_cast<float4*>(t) = make_float4(c[0], c[1], c[2], c[3]);
        }
    } else if (n) {
        const float b = g.bias ? load_one<T>(g.bias, n0 + w.col) : 0.0f;
#pragma unroll 1
        for (int i = 0; i < n; i += 4) {
            float c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = t[(i + j) * 2 * kPitch] + b;
                if (pre && i + j < n) pre[(i + j) * 2 * g.ldp] = c[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) t[(i + j) * 2 * kPitch] = act_value(c[j], g.act);
        }
    }
}

// A block from its transposing tile to out, the residual added.
template <class T, bool RESIDUAL, class TO>
__device__ __forceinline__ void store_block(const KernelArgs& p, TO* out, int64_t ld, int64_t m0, int64_t n0,
                                            const float* t, const uint32_t (&r)[kCols]) {
    const Walk w(p, n0);
    const int n = w.rows(p, m0, n0);
    t += w.row * kPitch + w.col;
    out += (m0 + w.row) * ld + n0 + w.col;
    if (w.four) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 f = *reinterpret_cast<const float4*>(t + i * 8 * kPitch);
            float c[4] = {f.x, f.y, f.z, f.w};
            if (RESIDUAL) {
                const uint32_t two[2] = {r[2 * i], r[2 * i + 1]};
#pragma unroll
                for (int j = 0; j < 4; ++j) c[j] += to_float(reinterpret_cast<const T*>(two)[j]);
            }
            if (i < n) store_four(out + i * 8 * ld, c);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float c = t[i * 2 * kPitch];
            if (RESIDUAL) {
                const uint16_t bits = (uint16_t)r[i];
                c += to_float(*reinterpret_cast<const T*>(&bits));
            }
            if (i < n) out[i * 2 * ld] = from_float<TO>(c);
        }
    }
    __syncwarp();
}

// What a finished block of 16-bit results goes through.
template <class T, bool LINEAR>
__device__ __forceinline__ void finish_block(const KernelArgs& p, void* to, int64_t m0, int64_t n0, float* t,
                                             const uint32_t (&r)[kCols]) {
    const GemmArgs& g = p.g;
    T* out = static_cast<T*>(to);
    if (LINEAR && (g.bias || g.pre[0] || g.act != HEDDLE_ACT_NONE)) activate_block<T>(p, m0, n0, t);
    if (LINEAR && g.residual)
        store_block<T, true>(p, out, g.ldo, m0, n0, t, r);
    else
        store_block<T, false>(p, out, g.ldo, m0, n0, t, r);
}

__device__ __forceinline__ void put_row(float* t, const uint32_t (&v)[kCols], int lane) {
#pragma unroll
    for (int j = 0; j < kCols; j += 4)
        *reinterpret_cast<uint4*>(t + lane * kPitch + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
}

// Tiles are taken in an order that keeps those in flight together close in
// both operands.  kGemmGated: a tile holds the same columns of both sums, so
// that act(g) u is formed where they are read back.  kGemmSum: two terms, one
// after the other, into the same sums.  kGemmPair: two products with one right
// operand, as one list of tiles.
template <int BN, int KIND, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1)
    gemm_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap a1,
                const __grid_constant__ CUtensorMap b0, const __grid_constant__ CUtensorMap b1,
                const __grid_constant__ KernelArgs p) {
    using S = Shape<BN, PAIR>;
    constexpr bool kAcrossA = KIND == kGemmPair, kAcrossB = KIND == kGemmPair || KIND == kGemmSum;
    constexpr int kOut = KIND == kGemmGated ? BN / 2 : BN;  // columns of C a tile covers
    // blocks of sums an epilogue warp reads back at a time
    constexpr int kAhead = KIND == kGemmGated || kOut / 2 < 2 * kCols ? 1 : 2;
    extern __shared__ unsigned char raw[];
    unsigned char* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    unsigned char* stages = base;
    float* epi = reinterpret_cast<float*>(base + kRing);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + kRing + kEpi);
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, done = empty + 8 * kMaxStages,
                   freed = done + 16;
    volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(bars + 2 * kMaxStages + 4);
    uint32_t* tmem_at = const_cast<uint32_t*>(gave_up) + 1;

    allow_dependents();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = PAIR ? cluster_rank() : 0;
    const int64_t first = PAIR ? blockIdx.x / 2 : blockIdx.x, step = PAIR ? gridDim.x / 2 : gridDim.x;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(done + 8 * b, 1);
            mbar_init(freed + 8 * b, (PAIR ? 2 : 1) * kEpiWarps);
        }
        *gave_up = 0;
        mbar_fence_init();
    }
    if (warp == 2) {
        if (PAIR)
            tmem_alloc_pair(smem_u32(tmem_at), S::kTmem);
        else
            tmem_alloc(smem_u32(tmem_at), S::kTmem);
    }
    fence_before();
    if (PAIR)
        cluster_sync();
    else
        __syncthreads();
    fence_after();
    await_previous();
    const uint32_t tmem = *tmem_at;
    constexpr bool kMayBeDeep = !PAIR && BN <= 64 && (KIND == kGemmLinear || KIND == kGemmGated);
    const int deep = kMayBeDeep ? p.deep : 1;
    const int per_tile = (p.steps * p.terms + deep - 1) / deep;

    if (warp == 0 && per_tile && elect_one()) {  // producer
        prefetch_map(&a0);
        prefetch_map(&b0);
        int s = 0;
        uint32_t phase = 0;
        bool go = true;
        const int a_bytes = kAcrossA ? S::kStageA : p.a_rows * BK * 2;
        auto load = [](uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y) {
            if (PAIR)
                load_2d_pair(dst, m, bar, x, y);
            else
                load_2d(dst, m, bar, x, y);
        };
        for (int64_t t = first; go && t < p.tiles; t += step) {
            int z, tm, tn;
            tile_at(p, t, z, tm, tn);
            const int m0 = tm * S::kTileM + (int)rank * BM;
            for (int it = 0; it < per_tile; ++it) {
                if (!(go = mbar_wait(empty + 8 * s, phase ^ 1, gave_up))) break;
                const uint32_t own = full + 8 * s, bar = PAIR ? cluster_at(own, 0) : own;
                const uint32_t sa = smem_u32(stages + s * p.stage), sb = sa + deep * a_bytes;
                if (kMayBeDeep && deep > 1) {
                    mbar_expect(own, p.stage);
                    load_3d(sa, &a0, bar, 0, m0, it * deep);
                    if (KIND == kGemmGated) {  // the two operands by turns
#pragma unroll
                        for (int d = 0; d < kDeep; ++d) {
                            load_2d(sb + d * S::kStageB, &b0, bar, (it * kDeep + d) * BK, tn * kOut);
                            load_2d(sb + d * S::kStageB + S::kStageB / 2, &b1, bar, (it * kDeep + d) * BK, tn * kOut);
                        }
                    } else {
                        load_3d(sb, &b0, bar, 0, tn * kOut, it * deep);
                    }
                    if (++s == p.stages) s = 0, phase ^= 1;
                    continue;
                }
                const bool second = KIND == kGemmSum ? it >= p.steps : KIND == kGemmPair ? z : false;
                const CUtensorMap* ma = second ? &a1 : &a0;
                const CUtensorMap* mb = second ? &b1 : &b0;
                const int k = (KIND == kGemmSum && second ? it - p.steps : it) * BK;
                if (rank == 0) mbar_expect(own, (PAIR ? 2 : 1) * (a_bytes + S::kStageB));
                if (kAcrossA) {
#pragma unroll
                    for (int j = 0; j < BM / 64; ++j) load(sa + j * 8192, ma, bar, m0 + j * 64, k);
                } else {
                    load(sa, ma, bar, k, m0);
                }
                if (KIND == kGemmGated) {
                    if (PAIR) {  // the gate's columns come first, the first CTA's half
                        load(sb, rank ? &b1 : &b0, bar, k, tn * kOut);
                    } else {
                        load(sb, &b0, bar, k, tn * kOut);
                        load(sb + kOut * BK * 2, &b1, bar, k, tn * kOut);
                    }
                } else if (kAcrossB) {
                    const int n0 = tn * BN + (int)rank * S::kRowsB;
#pragma unroll
                    for (int j = 0; j < S::kRowsB / 64; ++j) load(sb + j * 8192, mb, bar, n0 + j * 64, k);
                } else {
                    load(sb, mb, bar, k, tn * BN + (int)rank * S::kRowsB);
                }
                if (++s == p.stages) s = 0, phase ^= 1;
            }
        }
    } else if (warp == 1 && rank == 0 && per_tile && elect_one()) {  // issuer
        const uint32_t idesc = instr_desc(p.g.dtype == HEDDLE_BF16, kAcrossA, kAcrossB, BN, S::kTileM);
        const int a_bytes = kAcrossA ? S::kStageA : p.a_rows * BK * 2;
        int s = 0, half = 0;
        uint32_t phase = 0, round = 0;
        bool go = true;
        for (int64_t t = first; go && t < p.tiles; t += step) {
            if (!(go = mbar_wait(freed + 8 * half, round ^ 1, gave_up))) break;
            fence_after();
            for (int it = 0; it < per_tile; ++it) {
                if (!(go = mbar_wait(full + 8 * s, phase, gave_up))) break;
                fence_after();
                const uint32_t sa = smem_u32(stages + s * p.stage), sb = sa + deep * a_bytes;
                const uint64_t da = smem_desc(sa, 8192), db = smem_desc(sb, 8192);
                if (kMayBeDeep && deep > 1) {
#pragma unroll
                    for (int d = 0; d < kDeep; ++d)
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k)
                            mma_ss(tmem + half * BN, da + (d * a_bytes + 32 * k) / 16,
                                   db + (d * S::kStageB + 32 * k) / 16, idesc, it | d | k);
                    commit(empty + 8 * s);
                    if (++s == p.stages) s = 0, phase ^= 1;
                    continue;
                }
#pragma unroll
                for (int k = 0; k < BK / 16; ++k) {
                    const uint64_t ka = da + (kAcrossA ? 128 * k : 2 * k), kb = db + (kAcrossB ? 128 * k : 2 * k);
                    if (PAIR)
                        mma_ss_pair(tmem + half * BN, ka, kb, idesc, it | k);
                    else
                        mma_ss(tmem + half * BN, ka, kb, idesc, it | k);
                }
                if (PAIR)
                    commit_pair(empty + 8 * s);
                else
                    commit(empty + 8 * s);
                if (++s == p.stages) s = 0, phase ^= 1;
            }
            if (go) {
                if (PAIR)
                    commit_pair(done + 8 * half);
                else
                    commit(done + 8 * half);
            }
            half ^= 1;
            if (!half) round ^= 1;
        }
    } else if (warp >= 4) {  // epilogue
        const int w = warp % 4;
        const int from = (warp - 4) / 4 * (kOut / 2), to = from + kOut / 2;
        float* t0 = epi + (warp - 4) * 32 * kPitch;
        // a tile's sums are waited for as a whole: at most 4096 cycles a step more
        const long long limit = kWaitCycles + 4096ll * per_tile;
        int half = 0;
        uint32_t round = 0;
        for (int64_t t = first; t < p.tiles; t += step) {
            int z, tm, tn;
            tile_at(p, t, z, tm, tn);
            if (per_tile) {
                if (!__all_sync(~0u, mbar_wait(done + 8 * half, round, gave_up, limit))) break;
                fence_after();
            }
            const uint32_t acc = tmem + half * BN + ((uint32_t)(w * 32) << 16);
            const int64_t m0 = (int64_t)tm * S::kTileM + rank * BM + w * 32;
            const bool rows = m0 < p.g.M;
#pragma unroll 1
            for (int c = from; c < to; c += kAhead * kCols) {
                const int64_t n0 = (int64_t)tn * kOut + c;
                if (!rows || n0 >= p.g.N) break;
                uint32_t v[kAhead][kCols], u[kCols], r[kAhead][kCols];
                const int64_t row = m0 + lane;
                const bool direct = p.direct && n0 + kAhead * kCols <= p.g.N;
                if (KIND == kGemmLinear && p.g.residual) {
#pragma unroll
                    for (int h = 0; h < kAhead; ++h) {
                        if (!direct)
                            fetch_residual(p, m0, n0 + h * kCols, r[h]);
                        else if (row < p.g.M)
                            load_32(static_cast<const uint16_t*>(p.g.residual) + row * p.g.ldr + n0 + h * kCols, r[h]);
                    }
                }
                if (per_tile) {
#pragma unroll
                    for (int h = 0; h < kAhead; ++h) tmem_ld16(acc + c + h * kCols, v[h]);
                    if (KIND == kGemmGated) tmem_ld16(acc + kOut + c, u);
                    wait_ld();
                } else {
#pragma unroll
                    for (int j = 0; j < kAhead * kCols; ++j)
                        v[j / kCols][j % kCols] = u[j % kCols] = 0;  // a sum over nothing
                }
                if (KIND == kGemmGated) {
                    if (p.g.pre[0] && direct) {
                        if (row < p.g.M) {
                            float *pg = p.g.pre[0] + row * p.g.ldp + n0, *pu = p.g.pre[1] + row * p.g.ldp + n0;
                            store_32(pg, v[0]), store_32(pg + 8, v[0] + 8);
                            store_32(pu, u), store_32(pu + 8, u + 8);
                        }
                    } else if (p.g.pre[0]) {
                        put_row(t0, v[0], lane);
                        __syncwarp();
                        store_block<float, false>(p, p.g.pre[0], p.g.ldp, m0, n0, t0, u);
                        put_row(t0, u, lane);
                        __syncwarp();
                        store_block<float, false>(p, p.g.pre[1], p.g.ldp, m0, n0, t0, u);
                    }
#pragma unroll
                    for (int j = 0; j < kCols; ++j)
                        v[0][j] =
                            __float_as_uint(act_value(__uint_as_float(v[0][j]), p.g.act) * __uint_as_float(u[j]));
                }
                constexpr bool kLinear = KIND == kGemmLinear;
#pragma unroll
                for (int h = 0; h < kAhead; ++h) {
                    if (h && (c + h * kCols >= to || n0 + h * kCols >= p.g.N)) break;
                    if (direct) {
                        if (p.g.dtype == HEDDLE_BF16)
                            finish_row<__nv_bfloat16>(p, p.g.out[z], row, n0 + h * kCols, row < p.g.M, v[h], r[h],
                                                      kLinear);
                        else
                            finish_row<__half>(p, p.g.out[z], row, n0 + h * kCols, row < p.g.M, v[h], r[h], kLinear);
                        continue;
                    }
                    put_row(t0, v[h], lane);
                    __syncwarp();
                    if (p.g.dtype == HEDDLE_BF16)
                        finish_block<__nv_bfloat16, kLinear>(p, p.g.out[z], m0, n0 + h * kCols, t0, r[h]);
                    else
                        finish_block<__half, kLinear>(p, p.g.out[z], m0, n0 + h * kCols, t0, r[h]);
                }
            }
            fence_before();
            if (lane == 0) {
                if (PAIR)
                    mbar_arrive_cluster(cluster_at(freed + 8 * half, 0));
                else
                    mbar_arrive(freed + 8 * half);
            }
            half ^= 1;
            if (!half) round ^= 1;
        }
    }
    __syncthreads();
    if (*gave_up) {
        if (threadIdx.x == 0) atomicOr(p.err, kErrOpWait);
        drain();
    }
    if (PAIR)
        cluster_sync();  // the other CTA's products read this one's memory, and its warps' arrivals land here
    else
        __syncthreads();
    if (warp == 2) {
        if (PAIR)
            tmem_free_pair(tmem, S::kTmem);
        else
            tmem_free(tmem, S::kTmem);
    }
}

// ---------------------------------------------------------------- operands

// Rows of `cols` 16-bit values to rows at a stride of whole 128-byte lines, of
// up to four operands in one launch: bulk tensor copies need strides of 16
// bytes, and copies of 128 bytes that lie across two lines take twice as long
// (1023 x 2047 x 4099 forward: 52 us at strides of 16 bytes, 42 at whole
// lines).  Bound by memory: 25 MB read and written in 10 us.
struct LayOut {
    const uint16_t* src[4];
    uint16_t* dst[4];
    int64_t ld[4], dld[4], rows[4], cols[4];
};
constexpr int kLayUnits = 4;  // units of eight values a thread moves at a time, loaded before any is stored
__global__ void __launch_bounds__(256) lay_out_kernel(const __grid_constant__ LayOut l) {
    allow_dependents();
    const int o = blockIdx.y;
    const int64_t cols = l.cols[o], per = (cols + 7) / 8, total = l.rows[o] * per;
    const int64_t threads = (int64_t)gridDim.x * 256;
    for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < total; i0 += kLayUnits * threads) {
        uint32_t v[kLayUnits][5];
        int odd[kLayUnits], left[kLayUnits];
        uint16_t* dst[kLayUnits];
#pragma unroll
        for (int k = 0; k < kLayUnits; ++k) {
            const int64_t i = i0 + k * threads;
            left[k] = 0;
            if (i >= total) continue;
            const int64_t r = total <= UINT32_MAX ? (uint32_t)i / (uint32_t)per : i / per, c = (i - r * per) * 8;
            // eight values out of the four or five 32-bit words that hold them
            const uintptr_t at = reinterpret_cast<uintptr_t>(l.src[o] + r * l.ld[o] + c);
            const uint32_t* word = reinterpret_cast<const uint32_t*>(at & ~(uintptr_t)3);
            odd[k] = at >> 1 & 1, left[k] = (int)min((int64_t)8, cols - c);
            dst[k] = l.dst[o] + r * l.dld[o] + c;
#pragma unroll
            for (int j = 0; j < 5; ++j) v[k][j] = 2 * j < left[k] + odd[k] ? word[j] : 0;
        }
#pragma unroll
        for (int k = 0; k < kLayUnits; ++k) {
            if (!left[k]) continue;
            uint32_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u[j] = odd[k] ? __funnelshift_r(v[k][j], v[k][j + 1], 16) : v[k][j];
                if (left[k] == 2 * j + 1) u[j] &= 0xffff;  // the word's other half is the next row's
            }
            *reinterpret_cast<uint4*>(dst[k]) = make_uint4(u[0], u[1], u[2], u[3]);
        }
    }
    await_previous();  // operands are the caller's, and no kernel before has to do with their places
}

// The row stride of what is laid out here: whole 128-byte lines, since copies
// of 128 bytes a row that straddle lines took the products twice as long.
int64_t laid_ld(int64_t cols) { return ceil_div(cols, 64) * 64; }

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
// Adds the operand to `l` where copies do not take it as it is, once if it is
// there already.
void lay_out(GemmOperand& o, int64_t rows, int64_t cols, unsigned char*& ws, LayOut& l, int& n) {
    const int64_t ld = laid_ld(cols);
    if (copies_as_is(o, rows)) {
        if (rows == 1) o.ld = ld;
        return;
    }
    for (int i = 0; i < n; ++i)
        if (l.src[i] == o.p && l.ld[i] == o.ld && l.rows[i] == rows && l.cols[i] == cols) {
            o = {l.dst[i], ld};
            return;
        }
    l.src[n] = static_cast<const uint16_t*>(o.p), l.dst[n] = reinterpret_cast<uint16_t*>(ws);
    l.ld[n] = o.ld, l.dld[n] = ld, l.rows[n] = rows, l.cols[n] = cols;
    o = {ws, ld};
    ws += align256((size_t)rows * ld * 2);
    ++n;
}

cudaError_t map_of(CUtensorMap* m, const GemmOperand& o, int dtype, int64_t rows, int64_t cols, int box_rows) {
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)o.ld * 2};
    const uint32_t box[2] = {64, (uint32_t)box_rows};
    return make_map(m, o.p, dtype, 2, dims, strides, box);
}

// The same operand as steps of 64 columns, several a copy.
cudaError_t deep_map_of(CUtensorMap* m, const GemmOperand& o, int dtype, int64_t rows, int64_t cols, int box_rows) {
    const uint64_t dims[3] = {64, (uint64_t)rows, (uint64_t)(cols / 64)}, strides[2] = {(uint64_t)o.ld * 2, 128};
    const uint32_t box[3] = {64, (uint32_t)box_rows, kDeep};
    return make_map(m, o.p, dtype, 3, dims, strides, box);
}

bool unit16(const void* p, int64_t ld, int size, int unit) {
    return !p || ((uintptr_t)p % unit == 0 && ld * size % unit == 0);
}

// Pairs of CTAs that run at a time; asked for once a kernel and device.
template <class K>
int resident_pairs(K* kernel, const cudaLaunchConfig_t& cfg, int device, std::atomic<int> (&known)[64]) {
    if (device >= 0 && device < 64 && known[device].load(std::memory_order_relaxed) > 0)
        return known[device].load(std::memory_order_relaxed);
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = 1;
    }
    if (device >= 0 && device < 64) known[device].store(n, std::memory_order_relaxed);
    return n;
}

template <int BN, int KIND, bool PAIR>
cudaError_t run(const OpContext& x, const CUtensorMap (&a)[2], const CUtensorMap (&b)[2], KernelArgs& p,
                cudaStream_t st) {
    using S = Shape<BN, PAIR>;
    constexpr int kOut = KIND == kGemmGated ? BN / 2 : BN;
    p.m_tiles = (int)ceil_div(p.g.M, S::kTileM);
    p.n_tiles = (int)ceil_div(p.g.N, kOut);
    p.tiles = (int64_t)p.m_tiles * p.n_tiles * (KIND == kGemmPair ? p.g.count : 1);
    const int a_bytes = KIND == kGemmPair ? S::kStageA : p.a_rows * BK * 2;
    p.stage = p.deep * (a_bytes + S::kStageB);
    // a product reads 128 rows of A wherever they start: they must end in the ring
    const int past = (p.deep - 1) * a_bytes + S::kStageA - p.stage;
    const int room = kRing - (past > 0 ? past : 0);
    p.stages = room / p.stage < kMaxStages ? room / p.stage : kMaxStages;
    auto* k = gemm_kernel<BN, KIND, PAIR>;
    static std::atomic<uint64_t> asked{0};
    const cudaError_t e = allow_shared(k, kShared, x.device, asked);
    if (e != cudaSuccess) return e;
    if constexpr (PAIR) {
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute attr[2] = {};
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {2, 1, 1};
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3(2 * (x.num_sms / 2));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kShared;
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        static std::atomic<int> known[64];
        const int pairs = resident_pairs(k, cfg, x.device, known);
        cfg.gridDim = dim3(2 * (unsigned)(p.tiles < pairs ? p.tiles : pairs));
        cfg.numAttrs = x.chained ? 2 : 1;
        x.chained = true;
        return cudaLaunchKernelEx(&cfg, k, a[0], a[1], b[0], b[1], p);
    } else {
        const unsigned grid = (unsigned)(p.tiles < x.num_sms ? p.tiles : x.num_sms);
        return launch(x, k, grid, kThreads, kShared, st, a[0], a[1], b[0], b[1], p);
    }
}

// Tile of a call: columns, and whether pairs of CTAs take 256 rows.
struct Tile {
    int bn;
    bool pair;
};

// The tile that finishes first by the cycles a 64-wide step of its products
// takes (measured on steps from L2: what is fetched bounds all but the pair),
// those of its epilogue, which the next tile's products hide or not, the rounds
// of tiles that the SMs run, and the start of a pair.  Weights' gradients of 17
// rows, 4544 x 13376: 31 us on single 256-wide tiles, 43 on pairs, 58 on pairs
// of 128; 1024 x 4096 x 4096: 25.5 and 27.3, 2048 x 4096 x 14336 the pair's.
Tile choose_tile(const OpContext& x, const GemmArgs& g, bool direct) {
    const int64_t batch = g.kind == kGemmPair ? g.count : 1;
    const int64_t steps = ceil_div(g.K, BK) * (g.kind == kGemmSum ? g.count : 1);
    const struct {
        Tile t;
        double cycles;
    } all[] = {{{256, true}, 545}, {{224, true}, 485}, {{192, true}, 425}, {{128, true}, 340},
               {{256, false}, 660}, {{128, false}, 440}, {{64, false}, 340}, {{32, false}, 300}};
    Tile best{256, false};
    double least = 1e300;
    for (const auto& c : all) {
        if (c.t.bn < 64 && (g.kind != kGemmLinear || g.M > 64)) continue;  // 32 columns of C at least
        if (c.t.pair && g.M <= BM) continue;
        if (c.t.pair && c.t.bn % 128 && g.kind != kGemmLinear) continue;  // B's halves in whole copies
        const int out = g.kind == kGemmGated ? c.t.bn / 2 : c.t.bn;
        const int64_t tiles = ceil_div(g.M, c.t.pair ? 2 * BM : BM) * ceil_div(g.N, out) * batch;
        const int64_t rounds = ceil_div(tiles, c.t.pair ? x.num_sms / 2 : x.num_sms);
        // few rows: B streams from memory, a step as long as its bytes' share,
        // or as its barriers where a stage holds one
        double cycles = c.cycles;
        if (g.M <= 64) cycles = c.t.bn * 2.2 < 250 && g.kind == kGemmSum ? 250 : c.t.bn * 2.2;
        const double sums = steps * cycles, end = (c.t.pair ? 2450 : 900) + (direct ? 15.0 : 45.0) * out;
        const double time = (c.t.pair ? 6000 : 0) + (rounds - 1) * (sums < end ? end : sums) + sums + end;
        if (time < least) least = time, best = c.t;
    }
    return best;
}

template <int KIND>
cudaError_t run_kind(const OpContext& x, Tile t, const CUtensorMap (&a)[2], const CUtensorMap (&b)[2], KernelArgs& p,
                     cudaStream_t st) {
    if constexpr (KIND == kGemmLinear) {
        if (t.pair && t.bn == 224) return run<224, KIND, true>(x, a, b, p, st);
        if (t.pair && t.bn == 192) return run<192, KIND, true>(x, a, b, p, st);
    }
    if (t.pair && t.bn == 128) return run<128, KIND, true>(x, a, b, p, st);
    if (t.pair) return run<256, KIND, true>(x, a, b, p, st);
    if (t.bn == 256) return run<256, KIND, false>(x, a, b, p, st);
    if (t.bn == 128) return run<128, KIND, false>(x, a, b, p, st);
    if constexpr (KIND == kGemmLinear)
        if (t.bn == 32) return run<32, KIND, false>(x, a, b, p, st);
    return run<64, KIND, false>(x, a, b, p, st);
}

}  // namespace

size_t gemm_scratch(const OpContext&, const GemmArgs& g) {
    const Plan pl = plan_of(g);
    size_t n = 0;
    for (int i = 0; i < pl.a_count; ++i)
        if (!copies_as_is(g.a[i], pl.rows[0])) n += align256((size_t)pl.rows[0] * laid_ld(pl.cols[0]) * 2);
    for (int i = 0; i < pl.b_count; ++i)
        if (!copies_as_is(g.b[i], pl.rows[1])) n += align256((size_t)pl.rows[1] * laid_ld(pl.cols[1]) * 2);
    return n;
}

cudaError_t lay_out_operands(const OpContext& x, GemmArgs* const* list, int count, unsigned char* ws,
                             cudaStream_t st) {
    LayOut l{};
    int n = 0;
    for (int c = 0; c < count; ++c) {
        GemmArgs& g = *list[c];
        const Plan pl = plan_of(g);
        for (int i = 0; i < pl.a_count; ++i) lay_out(g.a[i], pl.rows[0], pl.cols[0], ws, l, n);
        for (int i = 0; i < pl.b_count; ++i) lay_out(g.b[i], pl.rows[1], pl.cols[1], ws, l, n);
    }
    if (!n) return cudaSuccess;
    int64_t units = 0;
    for (int i = 0; i < n; ++i) units = l.rows[i] * l.dld[i] / 8 > units ? l.rows[i] * l.dld[i] / 8 : units;
    const int64_t most = (int64_t)x.num_sms * 8, want = ceil_div(units, 256 * kLayUnits);
    const dim3 grid((unsigned)(want < most ? want : most), n);
    return launch(x, lay_out_kernel, grid, 256, 0, st, l);
}

cudaError_t launch_gemm(const OpContext& x, const GemmArgs& args, unsigned char* ws, cudaStream_t st) {
    if (gemv_takes(x, args)) return launch_gemv(x, args, st);
    KernelArgs p{};
    p.g = args;
    p.deep = 1;
    GemmArgs& g = p.g;
    const Plan pl = plan_of(g);
    p.steps = (int32_t)ceil_div(g.K, BK);
    p.terms = g.kind == kGemmSum ? g.count : 1;
    p.err = x.err;
    const int size = 2;
    p.vec = unit16(g.out[0], g.ldo, size, 8) && unit16(g.out[1], g.ldo, size, 8) &&
            unit16(g.residual, g.ldr, size, 8) && unit16(g.bias, 0, size, 8) && unit16(g.pre[0], g.ldp, 4, 16) &&
            unit16(g.pre[1], g.ldp, 4, 16);

    // an activation goes over a block in shared memory
    p.direct = (g.kind != kGemmLinear || g.act == HEDDLE_ACT_NONE) && unit16(g.out[0], g.ldo, size, 32) &&
               unit16(g.out[1], g.ldo, size, 32) && unit16(g.residual, g.ldr, size, 32) &&
               unit16(g.bias, 0, size, 16) &&
               (g.kind == kGemmLinear ? !g.pre[0]
                                      : unit16(g.pre[0], g.ldp, 4, 32) && unit16(g.pre[1], g.ldp, 4, 32));

    const Tile tile = choose_tile(x, g, p.direct);
    const bool across_a = g.kind == kGemmPair, across_b = across_a || g.kind == kGemmSum;
    p.a_rows = across_a ? 64 : (int)(g.M < BM ? ceil_div(g.M, 8) * 8 : BM);
    CUtensorMap a[2] = {}, b[2] = {};
    if (g.K > 0) {
        GemmArgs* one = &g;
        cudaError_t e = lay_out_operands(x, &one, 1, ws, st);
        if (e != cudaSuccess) return e;
        // whole steps only: columns past the last would be the next row's
        const bool few = g.M <= 64 && !tile.pair && tile.bn <= 64 && !across_b && g.K % BK == 0;
        p.deep = few ? kDeep : 1;
        auto map_a = few ? deep_map_of : map_of, map_b = few && g.kind == kGemmLinear ? deep_map_of : map_of;
        const int rows_b = tile.pair ? tile.bn / 2 : g.kind == kGemmGated ? tile.bn / 2 : tile.bn;
        for (int i = 0; e == cudaSuccess && i < pl.a_count; ++i)
            e = map_a(&a[i], g.a[i], g.dtype, pl.rows[0], pl.cols[0], p.a_rows);
        for (int i = 0; e == cudaSuccess && i < pl.b_count; ++i)
            e = map_b(&b[i], g.b[i], g.dtype, pl.rows[1], pl.cols[1], across_b ? 64 : rows_b);
        if (e != cudaSuccess) return e;
    }
    switch (g.kind) {
        case kGemmLinear: return run_kind<kGemmLinear>(x, tile, a, b, p, st);
        case kGemmGated: return run_kind<kGemmGated>(x, tile, a, b, p, st);
        case kGemmSum: return run_kind<kGemmSum>(x, tile, a, b, p, st);
        default: return run_kind<kGemmPair>(x, tile, a, b, p, st);
    }
}

}  // namespace hd
