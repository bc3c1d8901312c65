// heddle_attn_tc.cu -- attention with a sliding window and first tokens that
// stay visible on the tensor cores, forward and backward.
//
// A tile's 128 rows are the queries of consecutive tokens under one key head:
// row r is query head r % G of the group's G on token r / G, so that a key
// tile read once serves the whole group.  Rows past G * (128 / G) are empty.
// Scores and their gradients stay in tensor memory: the weights P (and dS)
// are written back over the scores as the 16-bit left operand of the next
// product.

#include <type_traits>

#include "heddle_attn.cuh"
#include "heddle_tc.cuh"

namespace hd {
namespace {

using namespace tc;

constexpr int kTile = 128;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
// A row's maximum is kept until a score passes it by this many powers of two:
// weights stay below 2^8, far inside the range of 16-bit types, and the sums
// are rarely scaled again.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two floats to 16-bit values, the first in the low half.
template <class T>
__device__ __forceinline__ uint32_t pack_two(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack_two<__nv_bfloat16>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <>
__device__ __forceinline__ uint32_t pack_two<__half>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Two floats at a time.
__device__ __forceinline__ uint64_t two(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ uint64_t two(uint32_t x, uint32_t y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(x), "r"(y));
    return r;
}
__device__ __forceinline__ float2 apart(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

struct Params {
    heddle_attention_args a;
    heddle_heads d_o, dq, dk, dv;
    const float* delta;
    int32_t group, tokens;  // G, tokens of a tile
    int32_t q_tiles, kv_tiles;
    int32_t splits, twins;  // pieces along the keys; whether they are twins
    float scale_log2;
    float* part_o;    // [splits][batch * q_heads * q_len][head_dim]
    float* part_lse;  // [splits][batch * q_heads * q_len]
    // backward over keys: the first `lead` key tiles in lead_parts parts along
    // the queries, the others in rest_parts; sums of parts as floats
    int32_t lead, lead_parts, rest_parts;
    float *part_dk, *part_dv;  // [slots][128][head_dim]
    // dS of pairs of tiles, where it is kept between the backward's passes:
    // query tile t's key tiles at places from t * ds_stride on, or (0) from
    // where those that causality leaves to the tiles before it end
    unsigned char* ds;
    int64_t ds_head;  // places of a key head
    int32_t ds_stride, ds_lead, ds_wrap, ds_reach;
    int32_t hb0, hbs;  // key heads of the batch that a launch takes: the first, how many
    // the next piece of work and the CTAs that are done, zero between launches;
    // the largest squares of dO's and V's rows
    int32_t* sched;
    uint32_t* err;
};

// Queries and keys of a sequence and how far positions are from query
// indices, in 32 bits: lengths here are at most 2^30.
struct Seq {
    int ql, kl, off;
};
constexpr int64_t kMaxLength = 1 << 30;
__device__ __forceinline__ Seq seq_of(const heddle_attention_args& a, int64_t b) {
    const Span s = span_of(a, b);
    return {(int)s.ql, (int)s.kl, (int)s.off};
}

// The key tiles that a range of queries sees: those of the first tokens ahead
// of the window's, then the window's.
struct KeyTiles {
    int lead, first, count;  // lead tiles from 0, then from `first` on; count of both
    __device__ int at(int j) const { return j < lead ? j : first + j - lead; }
};
__device__ __forceinline__ KeyTiles key_tiles(const Params& p, const Seq& s, int i0, int i1) {
    KeyTiles k{0, 0, 0};
    i1 = min(i1, s.ql);
    if (i0 >= i1) return k;
    const int hi = min(s.off + i1 - 1, s.kl - 1);
    if (hi < 0) return k;
    const int lo = p.a.window ? max(0, max(0, s.off + i0) - (int)p.a.window + 1) : 0;
    k.first = lo / kTile;
    const int sinks = min((int)p.a.sinks, hi + 1);
    k.lead = min((sinks + kTile - 1) / kTile, k.first);
    k.count = k.lead + hi / kTile - k.first + 1;
    return k;
}

// Bits lo .. hi of 32, as far as they are among them.
__device__ __forceinline__ uint32_t bits_between(int lo, int hi) {
    const uint32_t up = hi < 0 ? 0u : hi >= 31 ? ~0u : (2u << hi) - 1;
    const uint32_t below = lo <= 0 ? 0u : lo >= 32 ? ~0u : (1u << lo) - 1;
    return up & ~below;
}

// What the query at a position sees; positions below -1 see nothing either.
struct RowMask {
    int pos, low, sinks;
    __device__ RowMask(int at, const heddle_attention_args& a)
        : pos(max(at, -1)), low(a.window ? max(pos - (int)a.window + 1, 0) : 0), sinks((int)a.sinks) {}
    // bit y: whether it sees key + y
    __device__ uint32_t sees32(int key) const {
        return bits_between(low - key, pos - key) | bits_between(0, min(sinks - 1, pos) - key);
    }
};

// Where dS of a pair of tiles lies, among the launch's.  A query tile's near
// key tiles are consecutive and at most ds_wrap; with no window its last one is
// at most (t tokens + ds_reach) / 128, and a sum of floors is at most the floor
// of the sum.
constexpr int kPlaceBytes = kTile * kTile * 2;
__host__ __device__ __forceinline__ int64_t ds_row(const Params& p, int64_t t) {
    return p.ds_stride ? t * p.ds_stride : (p.tokens * (t * (t - 1) / 2) + p.ds_reach * t) / kTile + t;
}
__device__ __forceinline__ int ds_col(const Params& p, int tile) {
    return tile < p.ds_lead ? tile : p.ds_lead + tile % p.ds_wrap;
}

// Every query of tokens i0 .. i1 - 1 sees every key of the tile at k0.
__device__ __forceinline__ bool all_visible(const Params& p, const Seq& s, int i0, int i1, int k0) {
    return s.off + i0 >= k0 + kTile - 1 && (p.a.window == 0 || s.off + i1 - 1 - k0 < (int)p.a.window ||
                                            k0 + kTile <= (int)p.a.sinks);
}

// Rows [from, 128) of a tile in shared memory to zero, a row a thread; the
// products read them after the next barrier.
template <int DP>
__device__ __forceinline__ void clear_rows(unsigned char* tile, int row, int from) {
    if (row >= from)
#pragma unroll
        for (int h = 0; h < DP / 64; ++h)
#pragma unroll
            for (int c = 0; c < 8; ++c)
                *reinterpret_cast<uint4*>(tile + h * 16384 + row * 128 + c * 16) = make_uint4(0, 0, 0, 0);
}

// A D[128][N] = A B^T step over head_dim (operands' rows run along it).
template <int DP>
__device__ __forceinline__ void mma_dims(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const uint32_t at = (k / 4) * 16384 + (k % 4) * 32;
        mma_ss(d, smem_desc(a + at, 16384), smem_desc(b + at, 16384), idesc, k != 0);
    }
}
// D[128][DP] (+)= W B over 128 rows of B: W in tensor memory, 64 columns in
// runs of RUN, the next one `GAP` columns further.
template <int RUN, int GAP>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t w, uint32_t b, uint32_t idesc, bool add) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
        mma_ts(d, w + k * 8 % RUN + k * 8 / RUN * GAP, smem_desc(b + k * 2048, 16384), idesc, add || k);
}

template <int DP>
__device__ __forceinline__ void load_q_tile(uint32_t dst, const CUtensorMap* m, uint32_t bar, const Params& p,
                                            int t0, int hk, int b) {
#pragma unroll
    for (int h = 0; h < DP / 64; ++h) load_4d(dst + h * 16384, m, bar, h * 64, hk * p.group, t0, b);
}
template <int DP>
__device__ __forceinline__ void load_kv_tile(uint32_t dst, const CUtensorMap* m, uint32_t bar, int k0, int hk,
                                             int b) {
#pragma unroll
    for (int h = 0; h < DP / 64; ++h) load_4d(dst + h * 16384, m, bar, h * 64, hk, k0, b);
}

// Sums times f, and those of a second place times f1 added.
__device__ __forceinline__ void scale_sums(uint32_t (&v)[32], float f, uint32_t second, float f1) {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * f);
    if (!second) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t u[16];
        tmem_ld16(second + 16 * h, u);
        wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j)
            v[16 * h + j] = __float_as_uint(__uint_as_float(v[16 * h + j]) + __uint_as_float(u[j]) * f1);
    }
}

// One row of DP sums times f (and a second place's times f1) from tensor
// memory to memory: 16 bytes at a time where the row allows.
template <class T, int DP>
__device__ __forceinline__ void store_row(uint32_t tmem, T* out, bool live, int D, float f, uint32_t second = 0,
                                          float f1 = 0.0f) {
    const bool wide = ((uintptr_t)out & 15) == 0;
#pragma unroll 1
    for (int c = 0; c < DP; c += 32) {
        __syncwarp();
        uint32_t v[32];
        tmem_ld32(tmem + c, v);
        wait_ld();
        scale_sums(v, f, second ? second + c : 0u, f1);
        if (!live) continue;
        if (wide && c + 32 <= D) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                uint4 u;
                u.x = pack_two<T>(__uint_as_float(v[j]), __uint_as_float(v[j + 1]));
                u.y = pack_two<T>(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3]));
                u.z = pack_two<T>(__uint_as_float(v[j + 4]), __uint_as_float(v[j + 5]));
                u.w = pack_two<T>(__uint_as_float(v[j + 6]), __uint_as_float(v[j + 7]));
                *reinterpret_cast<uint4*>(out + c + j) = u;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (c + j < D) out[c + j] = from_float<T>(__uint_as_float(v[j]));
        }
    }
}
template <int COLS>
__device__ __forceinline__ void store_floats(uint32_t tmem, float* out, bool live, int D, float f,
                                             uint32_t second = 0, float f1 = 0.0f) {
#pragma unroll 1
    for (int c = 0; c < COLS; c += 32) {
        __syncwarp();
        uint32_t v[32];
        tmem_ld32(tmem + c, v);
        wait_ld();
        scale_sums(v, f, second ? second + c : 0u, f1);
        if (!live) continue;
#pragma unroll
        for (int j = 0; j < 32; j += 4)
            if (c + j < D)  // whole units of four: head_dim is a multiple of eight
                *reinterpret_cast<uint4*>(out + c + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
    }
}
// A row of zeros: whole units of eight values, as a head has, where they lie
// so (value by value a tile past its sequence's end took longer than three
// tiles of keys).
template <class T>
__device__ __forceinline__ void zero_row(T* out, int D) {
    constexpr int kUnit = 16 / sizeof(T);
    if (((uintptr_t)out & 15) == 0) {
        for (int c = 0; c < D; c += kUnit) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
    } else {
        for (int c = 0; c < D; ++c) out[c] = from_float<T>(0.0f);
    }
}

// ------------------------------------------------------------------- forward

// NT query tiles of a key head against the key tiles that they see, eight
// warps each: two threads a row, half of the columns each (one warp a row
// left its scheduler idle most of the time).  While one tile's warps turn
// scores into weights the tensor cores run the other's products.
//
// A step of 128 x 128 scores is 2 x 512 cycles of the tensor cores and as long
// a chain of trips to tensor memory (some 600 cycles each), barriers and 128
// exponentials a thread; the two tiles hide each other's.  Bound by that chain
// where sequences are short, with the prologue and epilogue of a CTA: two
// causal sequences of 2048, 32 heads over 8 of 128, 82 us (8.3e14 operations a
// second); one of 8192 takes 422 us (1.3e15).  Not by the exponentials: an
// eighth of them as polynomials took 428, a quarter 487.
template <int DP, int NT>
struct Forward {
    static constexpr int kTileBytes = kTile * DP * 2;
    static constexpr int kHigh = (2 * NT + 1) * 2 * kTile * 4;  // the halves' maxima, by turns; a twin's statistics
    static constexpr int kRoom = 227 * 1024 - 1024 - 512 - kHigh - NT * kTileBytes;
    static constexpr int kSlots = kRoom / kTileBytes < 8 ? kRoom / kTileBytes : 8;  // K and V tiles by turns
    static constexpr int kBytes = 1024 + (NT + kSlots) * kTileBytes + 512 + kHigh;
    static constexpr int kThreads = 64 + NT * 256;
    static constexpr int kCols = NT * (kTile + DP) <= 256 ? 256 : 512;
};

// A piece of the forward pass: NT query tiles of a key head and the key tiles
// they see; tile q takes count[q] of them from from[q] on.  Twins are one
// query tile twice, each with half of its key tiles.
template <int NT, bool TWINS>
struct ForwardPiece {
    int hk, b, split, t0;
    Seq s;
    KeyTiles keys;
    int n, from[NT], count[NT];
    __device__ ForwardPiece(const Params& p, int id) {
        split = id % p.splits;
        id /= p.splits;
        hk = id % p.a.kv_heads;
        id /= p.a.kv_heads;
        b = id % (int)p.a.batch;
        s = seq_of(p.a, b);
        constexpr int kTiles = TWINS ? 1 : NT;
        // the last queries see the most keys: their tiles come first
        t0 = ((p.q_tiles + kTiles - 1) / kTiles - 1 - id / (int)p.a.batch) * kTiles * p.tokens;
        keys = key_tiles(p, s, t0, t0 + kTiles * p.tokens);
        const int j0 = (int)((int64_t)keys.count * split / p.splits),
                  j1 = (int)((int64_t)keys.count * (split + 1) / p.splits);
        n = 0;
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            from[q] = j0;
            if (TWINS) {
                const int half = (j1 - j0 + 1) / 2;
                from[q] = j0 + q * half;
                count[q] = q ? j1 - j0 - half : half;
            } else {
                const KeyTiles own = key_tiles(p, s, t0 + q * p.tokens, t0 + (q + 1) * p.tokens);
                count[q] = 0;
                // up to the last of its tiles in the common order; the first ones are common to all
                if (own.count)
                    count[q] = max(0, min(j1, keys.lead + own.first + own.count - own.lead - keys.first) - j0);
            }
            n = max(n, count[q]);
        }
    }
    // Places in the order of loading.  Tiles share keys and values: K and V by
    // turns.  Twins: both K of a step, then both V, one of each in a last
    // step of the first twin alone.
    __device__ int k_at(int q, int j) const { return TWINS ? 4 * j + q : 2 * j; }
    __device__ int v_at(int q, int j) const { return TWINS ? 4 * j + q + (j < count[NT - 1] ? 2 : 1) : 2 * j + 1; }
};

template <class T, int DP, int NT, bool TWINS>
__global__ void __launch_bounds__(Forward<DP, NT>::kThreads, 1)
    attn_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ Params p) {
    using F = Forward<DP, NT>;
    extern __shared__ unsigned char raw[];
    unsigned char* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    unsigned char* ring = base + NT * F::kTileBytes;
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + F::kSlots * F::kTileBytes);
    const uint32_t full = smem_u32(bars), empty = full + 8 * F::kSlots, q_full = empty + 8 * F::kSlots,
                   s_full = q_full + 16, p_ready = s_full + 16, o_done = p_ready + 16, met = o_done + 16,
                   told = met + 64;
    volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(bars + 2 * F::kSlots + 18);
    uint32_t* tmem_at = const_cast<uint32_t*>(gave_up) + 1;
    float* highs = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(bars) + 512);  // [2][NT][2][128]
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    allow_dependents();
    await_previous();
    const ForwardPiece<NT, TWINS> w(p, blockIdx.x);
    const Seq& s = w.s;
    const KeyTiles& keys = w.keys;
    const int n = w.n, t0 = w.t0, hk = w.hk, b = w.b, split = w.split;

    if (threadIdx.x == 0) {
        for (int i = 0; i < F::kSlots; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int q = 0; q < 2; ++q) {
            mbar_init(q_full + 8 * q, 1);
            mbar_init(s_full + 8 * q, 1);
            mbar_init(p_ready + 8 * q, 8);
            mbar_init(o_done + 8 * q, 1);
        }
        for (int q = 0; q < 8; ++q) mbar_init(met + 8 * q, 2);
        mbar_init(told, 4);
        *gave_up = 0;
        mbar_fence_init();
        if (n > 0) {  // the first loads run while the CTA gathers
            const uint32_t q_bytes = p.group * p.tokens * DP * 2;
#pragma unroll
            for (int q = 0; q < (TWINS ? 1 : NT); ++q)
                if (w.count[q] > 0) {
                    mbar_expect(q_full + 8 * q, q_bytes);
                    load_q_tile<DP>(smem_u32(base + q * F::kTileBytes), &mq, q_full + 8 * q, p, t0 + q * p.tokens, hk,
                                    b);
                }
            mbar_expect(full, F::kTileBytes);
            load_kv_tile<DP>(smem_u32(ring), &mk, full, keys.at(w.from[0]) * kTile, hk, b);
        }
    }
    if (warp == 2) tmem_alloc(smem_u32(tmem_at), F::kCols);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_at;
    if (warp == 0 && n > 0 && elect_one()) {
        int i = 1;
        bool go = true;
        auto load = [&](const CUtensorMap* m, int tile) {
            const int slot = i % F::kSlots;
            if (!(go = go && mbar_wait(empty + 8 * slot, (i / F::kSlots & 1) ^ 1, gave_up))) return;
            mbar_expect(full + 8 * slot, F::kTileBytes);
            load_kv_tile<DP>(smem_u32(ring + slot * F::kTileBytes), m, full + 8 * slot, keys.at(tile) * kTile, hk, b);
            ++i;
        };
        for (int j = 0; go && j < n; ++j) {
            if (j > 0) load(&mk, w.from[0] + j);
            if (TWINS && j < w.count[NT - 1]) load(&mk, w.from[NT - 1] + j);
            load(&mv, w.from[0] + j);
            if (TWINS && j < w.count[NT - 1]) load(&mv, w.from[NT - 1] + j);
        }
    } else if (warp == 1 && n > 0 && elect_one()) {
        const uint32_t bf = p.a.dtype == HEDDLE_BF16;
        const uint32_t id_s = instr_desc(bf, false, false, kTile), id_o = instr_desc(bf, false, true, DP);
        bool go = true;
        for (int j = -1; go && j < n; ++j) {
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                const uint32_t ts = tmem + q * kTile, to_acc = tmem + NT * kTile + q * DP;
                const int iv = w.v_at(q, j), ik = w.k_at(q, j + 1), sv = iv % F::kSlots, sk = ik % F::kSlots;
                const bool last = TWINS || q == NT - 1;  // of those that read the step's keys and values
                if (j >= 0 && j < w.count[q]) {
                    if (!(go = mbar_wait(full + 8 * sv, iv / F::kSlots & 1, gave_up))) break;
                    if (!(go = mbar_wait(p_ready + 8 * q, j & 1, gave_up))) break;
                    fence_after();
                    mma_rows<32, 64>(to_acc, ts, smem_u32(ring + sv * F::kTileBytes), id_o, j > 0);
                    if (j + 1 == w.count[q]) commit(o_done + 8 * q);
                }
                if (last && j >= 0 && (TWINS ? j < w.count[q] : true)) commit(empty + 8 * sv);
                if (j + 1 < w.count[q]) {
                    if (!(go = mbar_wait(full + 8 * sk, ik / F::kSlots & 1, gave_up))) break;
                    if (j < 0 && !(go = mbar_wait(q_full + (TWINS ? 0 : 8 * q), 0, gave_up))) break;
                    fence_after();
                    mma_dims<DP>(ts, smem_u32(base + (TWINS ? 0 : q) * F::kTileBytes),
                                 smem_u32(ring + sk * F::kTileBytes), id_s);
                    commit(s_full + 8 * q);
                }
                if (last && (TWINS ? j + 1 < w.count[q] : j + 1 < n)) commit(empty + 8 * sk);
            }
        }
    } else if (warp >= 2) {
        const int q = (warp - 2) / 8, side = (warp - 2) / 4 % 2, row = (warp % 4) * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t ts = tmem + lanes + q * kTile, to_acc = tmem + lanes + NT * kTile + q * DP;
        const uint32_t pair = met + 8 * (q * 4 + warp % 4);  // this warp and the one of the rows' other half
        const int i0 = t0 + (TWINS ? 0 : q * p.tokens), i1 = i0 + p.tokens;
        const int i = i0 + row / p.group, h = hk * p.group + row % p.group;
        const RowMask mask(s.off + i, p.a);
        const float c = p.scale_log2;
        float top = -INFINITY, sum = 0.0f;
        const int mine = w.count[q];
        // a warp whose rows no query fills only keeps step
        const bool idle = (min(i1, s.ql) - i0) * p.group <= warp % 4 * 32;
        bool go = true;
        // the other half's value for the row, and this one's for it
        auto swap = [&](int turn, float v) {
            float* at = highs + ((turn & 1) * NT + q) * 2 * kTile + row;
            at[side * kTile] = v;
            __syncwarp();
            if (lane == 0) mbar_arrive(pair);
            go = __all_sync(~0u, mbar_wait(pair, turn & 1, gave_up));
            return at[(side ^ 1) * kTile];
        };
        for (int j = 0; j < mine; ++j) {
            const int k0 = keys.at(w.from[q] + j) * kTile;
            const bool whole = all_visible(p, s, i0, min(i1, s.ql), k0);
            if (!(go = __all_sync(~0u, mbar_wait(s_full + 8 * q, j & 1, gave_up)))) break;
            fence_after();
            if (!idle) {
                uint32_t v[2][32];
#pragma unroll
                for (int x = 0; x < 2; ++x) tmem_ld32(ts + 64 * side + 32 * x, v[x]);
                wait_ld();
                if (!whole) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint32_t seen = mask.sees32(k0 + 64 * side + 32 * x);
#pragma unroll
                        for (int y = 0; y < 32; ++y)
                            if (!(seen >> y & 1)) v[x][y] = 0xff800000u;  // -infinity
                    }
                }
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 32; ++y) m4[y % 4] = fmaxf(m4[y % 4], __uint_as_float(v[x][y]));
                float high = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                high = fmaxf(high, swap(j, high));
                if (!go) break;
                float keep = 1.0f;
                if (high > top && (top == -INFINITY || (high - top) * c > kSlack)) {
                    keep = top == -INFINITY ? 0.0f : exp2_fast((top - high) * c);
                    top = high;
                    sum *= keep;
                }
                if (j > 0 && __any_sync(~0u, keep != 1.0f)) {
                    // the product of the step before has completed: the scores'
                    // barrier was committed after it
#pragma unroll 1
                    for (int x = 0; x < DP / 2; x += 16) {
                        uint32_t o[16];
                        tmem_ld16(to_acc + side * (DP / 2) + x, o);
                        wait_ld();
#pragma unroll
                        for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * keep);
                        tmem_st16(to_acc + side * (DP / 2) + x, o);
                    }
                }
                const float sub = top == -INFINITY ? 0.0f : top * c;
                const uint64_t c2 = two(c, c), sub2 = two(-sub, -sub);
                uint64_t part[2] = {0, 0};
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    uint32_t w[16];
#pragma unroll
                    for (int y = 0; y < 32; y += 2) {
                        const float2 z = apart(fma_two(two(v[x][y], v[x][y + 1]), c2, sub2));
                        const float lo = exp2_fast(z.x), hi = exp2_fast(z.y);
                        part[y / 2 % 2] = add_two(part[y / 2 % 2], two(lo, hi));
                        w[y / 2] = pack_two<T>(lo, hi);
                    }
                    tmem_st16(ts + 64 * side + 16 * x, w);  // over scores that this warp itself has read
                }
                const float2 both = apart(add_two(part[0], part[1]));
                sum += both.x + both.y;
            }
            if (side == 0 && s.kl < p.a.kv_len && k0 + kTile > s.kl) {  // values past the sequence
                const int iv = w.v_at(q, j), sv = iv % F::kSlots;
                if (!(go = __all_sync(~0u, mbar_wait(full + 8 * sv, iv / F::kSlots & 1, gave_up)))) break;
                clear_rows<DP>(ring + sv * F::kTileBytes, row, s.kl - k0);
                fence_async_shared();
            }
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + 8 * q);
        }
        if (go && mine > 0) {
            if (!idle) sum += swap(mine, sum);
            if (go) go = __all_sync(~0u, mbar_wait(o_done + 8 * q, 0, gave_up));
        }
        fence_after();
        if (go) {
            // twins: the second tells the first what it has, and the first adds
            // up both tiles' sums, which lie in the same lanes
            float f_mine = 1.0f, f_other = 0.0f;
            bool other = false;
            float* told_at = highs + 2 * NT * 2 * kTile + row;
            if (TWINS && q == 1 && side == 0) {
                told_at[0] = mine > 0 ? top : -INFINITY;
                told_at[kTile] = mine > 0 ? sum : 0.0f;
                __syncwarp();
                if (lane == 0) mbar_arrive(told);
            }
            if (TWINS && q == 0) {
                go = __all_sync(~0u, mbar_wait(told, 0, gave_up));
                other = w.count[NT - 1] > 0;
                if (go && other) go = __all_sync(~0u, mbar_wait(o_done + 8, 0, gave_up));
                fence_after();
                const float top1 = told_at[0], sum1 = told_at[kTile], both = fmaxf(top, top1);
                if (both > -INFINITY) {
                    const float e0 = exp2_fast((top - both) * c), e1 = exp2_fast((top1 - both) * c);
                    sum = sum * e0 + sum1 * e1;
                    f_other = e1, top = both;
                    f_mine = e0;
                } else {  // zeros, or NaN from scores that are
                    sum += sum1;
                }
            }
            const bool inside = row < p.group * p.tokens && i < p.a.q_len;
            const bool some = mine > 0 && i < s.ql && !(sum == 0.0f);
            const float f = some ? 1.0f / sum : 0.0f;
            const float lse = some ? (top * c + log2f(sum)) * kLn2 : -INFINITY;
            const int64_t r = ((int64_t)b * p.a.q_heads + h) * p.a.q_len + i;
            const int D = p.a.head_dim, d0 = side * (DP / 2);
            if (go && !(TWINS && q == 1)) {
                const uint32_t second = to_acc + DP + d0;  // the twin's
                const float f0 = f * f_mine, f1 = f * f_other;
                if (p.splits > 1) {
                    const int64_t at = (int64_t)split * p.a.batch * p.a.q_heads * p.a.q_len + r;
                    if (inside && side == 0) p.part_lse[at] = lse;
                    // a part of no weight is not read
                    if (mine > 0)
                        store_floats<DP / 2>(to_acc + d0, p.part_o + at * D + d0, inside && some, D - d0, f0,
                                             other ? second : 0u, f1);
                } else {
                    T* out = static_cast<T*>(p.a.o.data) + b * p.a.o.batch_stride + i * p.a.o.token_stride +
                             h * p.a.o.head_stride + d0;
                    if (mine > 0)
                        store_row<T, DP / 2>(to_acc + d0, out, inside && some, D - d0, f0, other ? second : 0u, f1);
                    if (inside && !some) zero_row(out, min(D - d0, DP / 2));
                    if (inside && side == 0 && p.a.lse) p.a.lse[r] = lse;
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    if (*gave_up) {
        if (threadIdx.x == 0) atomicOr(p.err, kErrOpWait);
        drain();
        __syncthreads();
    }
    if (warp == 2) tmem_free(tmem, F::kCols);
}

// Joins the parts of rows split along the keys, one warp a row: a call of few
// query tiles takes the keys in parts, enough for every SM.  Single tokens read
// the cache once: 16 histories of up to 8192 with a window of 4096, 8 key heads
// of 128, 269 MB in 52 us both kernels (5.2e12 bytes a second).
template <class T>
__global__ void __launch_bounds__(256) attn_join_kernel(const __grid_constant__ Params p) {
    allow_dependents();
    await_previous();
    const int lane = threadIdx.x % 32, D = p.a.head_dim;
    const int64_t rows = p.a.batch * p.a.q_heads * p.a.q_len;
    const int64_t r = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (r >= rows) return;
    const float mine = lane < p.splits ? p.part_lse[lane * rows + r] : -INFINITY;
    float top = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    // a part without weights has no logarithm; one of NaN makes the row NaN
    const float e = mine == -INFINITY ? 0.0f : expf(mine - top);
    const float total = warp_sum(e);
    const float w = e == 0.0f ? 0.0f : e / total;
    float acc[4] = {};
    for (int x = 0; x < p.splits; ++x) {
        const float f = __shfl_sync(~0u, w, x);
        if (f == 0.0f) continue;
        const float* o = p.part_o + ((int64_t)x * rows + r) * D;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lane + 32 * j < D) acc[j] += f * o[lane + 32 * j];
    }
    const int64_t b = r / (p.a.q_heads * p.a.q_len), h = r / p.a.q_len % p.a.q_heads, i = r % p.a.q_len;
    T* out = static_cast<T*>(p.a.o.data) + b * p.a.o.batch_stride + i * p.a.o.token_stride + h * p.a.o.head_stride;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (lane + 32 * j < D) out[lane + 32 * j] = from_float<T>(acc[j]);
    if (p.a.lse && lane == 0) p.a.lse[r] = total == 0.0f ? -INFINITY : top + logf(total);
}

// ------------------------------------------------------------------ backward

// A kernel's CTAs stay and take one piece of work after another, so that a
// piece's first loads and products run under the end of the one before it.
// The producer takes the next number from memory a piece ahead and hands it
// to the other warps through two places in shared memory.
struct Pieces {
    uint32_t full, empty;  // two barriers each
    volatile int* place;
    __device__ void init(int readers) const {
        for (int i = 0; i < 2; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, readers);
        }
    }
    // the producer's: hands out piece `it`, the id-th, or -1 for the end
    __device__ bool put(int it, int id, volatile uint32_t* gave_up) const {
        if (!mbar_wait(empty + 8 * (it & 1), (it >> 1 & 1) ^ 1, gave_up)) return false;
        place[it & 1] = id;
        mbar_arrive(full + 8 * (it & 1));
        return true;
    }
    // a single thread's
    __device__ int get(int it, volatile uint32_t* gave_up) const {
        if (!mbar_wait(full + 8 * (it & 1), it >> 1 & 1, gave_up)) return -1;
        const int id = place[it & 1];
        mbar_arrive(empty + 8 * (it & 1));
        return id;
    }
    // a warp's
    __device__ int get_warp(int it, volatile uint32_t* gave_up) const {
        if (!__all_sync(~0u, mbar_wait(full + 8 * (it & 1), it >> 1 & 1, gave_up))) return -1;
        const int id = place[it & 1];
        __syncwarp();
        if (threadIdx.x % 32 == 0) mbar_arrive(empty + 8 * (it & 1));
        return id;
    }
};
// The last CTA to end leaves the numbers as the next launch needs them.
__device__ __forceinline__ void leave_pieces(int32_t* sched) {
    __threadfence();
    if (atomicAdd(sched + 1, 1) == (int)gridDim.x - 1) {
        sched[0] = 0;
        sched[1] = 0;
        __threadfence();
    }
}

// What dS is multiplied by before it is rounded, and its products divided by: a
// power of two that takes the largest dS that the call can have, 2 scale times
// the largest gradient's row and value's row by their norms, to 2^15, so that in
// float16 no gradient that is itself in range is lost at either end.  bfloat16
// has the range of the sums.  Finding the maxima takes 4 us of the 241 of the
// windowed step of two sequences of 4095 (16 heads over 4 of 64).
template <class T>
__device__ __forceinline__ float ds_factor(const Params& p) {
    if (std::is_same<T, __nv_bfloat16>::value) return 1.0f;
    const float squares[2] = {__int_as_float(p.sched[2]), __int_as_float(p.sched[3])};
    const float most = 2.0f * p.a.scale * sqrtf(squares[0]) * sqrtf(squares[1]);
    if (!(most > 0.0f && most < INFINITY)) return 1.0f;
    int e;
    frexpf(most, &e);
    return ldexpf(1.0f, min(15 - e, 100));
}

// Sixteen warps turn scores into dS, four for every quarter of a tile's
// columns: with eight, each scheduler's two warps left it idle two thirds of
// the time.
constexpr int kGradWarps = 16, kGradThreads = 64 + 32 * kGradWarps;

// Bars of a backward kernel, in the order that follows its tiles.
struct GradBars {
    uint32_t held, full, full2, empty, a_full, b_full, a_ready, b_ready, stats, done, held_free, work;
    __device__ explicit GradBars(uint32_t at)
        : held(at), full(at + 8), full2(at + 24), empty(at + 40), a_full(at + 56), b_full(at + 64), a_ready(at + 72),
          b_ready(at + 80), stats(at + 96), done(at + 104), held_free(at + 112), work(at + 120) {}
    __device__ void init() const {
        mbar_init(held, 1);
        mbar_init(held_free, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(full2 + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        mbar_init(a_full, 1);
        mbar_init(b_full, 1);
        mbar_init(a_ready, kGradWarps);
        mbar_init(b_ready, kGradWarps);
        mbar_init(b_ready + 8, kGradWarps);
        mbar_init(stats, kGradWarps);
        mbar_init(done, 1);
    }
};
constexpr int kGradBarBytes = 160;
// Chained kernels that hold tensor memory take more than half of an SM's shared
// memory, so that no two of their CTAs share an SM: one that holds it while it
// waits for the end of the kernel before could hold what that kernel's CTA
// waits for, and that wait has no limit.
constexpr int kAlone = 114 * 1024;

// dq of a query tile where dS is not kept: dq = sum over key tiles of dS K with
// S = Q K^T, dP = dO V^T, dS = scale P (dP - delta), rounded to the element type
// in a range of its own (ds_factor).  Q and dO stay in shared memory, K and V
// tiles come in two stages.  Scores of the next tile are computed while this
// one's are turned into dS (two buffers).  CTAs take one query tile after another, the longest first (a grid
// of one tile each: 137 us against 119).  Bound by the chain from scores to dS
// as the forward is: 114 us for two causal sequences of 2048 (32 heads over 8 of
// 128).
template <int DP>
struct GradShape {
    static constexpr int kTileBytes = kTile * DP * 2;
    static constexpr int kStats = 3 * kTile * 8 + 16;
    static constexpr int kUsed = 1024 + 6 * kTileBytes + kGradBarBytes + 64 + kStats;
    static constexpr int kBytes = kUsed > kAlone ? kUsed : kAlone;
};

template <class T, int DP>
__global__ void __launch_bounds__(kGradThreads, 1)
    attn_dq_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                   const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo,
                   const __grid_constant__ Params p, const int pieces) {
    using G = GradShape<DP>;
    extern __shared__ unsigned char raw[];
    unsigned char* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    unsigned char *sq = base, *sdo = base + G::kTileBytes, *stage = base + 2 * G::kTileBytes;  // K, V, K, V
    unsigned char* tail = base + 6 * G::kTileBytes;
    const GradBars bar(smem_u32(tail));
    const Pieces work{bar.work, bar.work + 16, reinterpret_cast<int*>(tail + kGradBarBytes)};
    volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(tail + kGradBarBytes + 8);
    uint32_t* tmem_at = const_cast<uint32_t*>(gave_up) + 1;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    allow_dependents();
    struct Piece {
        int hk, b, t0, t1;
        Seq s;
        KeyTiles keys;
        __device__ Piece(const Params& p, int id) {
            hk = id % p.a.kv_heads;
            id /= p.a.kv_heads;
            b = id % (int)p.a.batch;
            t0 = (p.q_tiles - 1 - id / (int)p.a.batch) * p.tokens;
            s = seq_of(p.a, b);
            t1 = min(t0 + p.tokens, s.ql);
            keys = key_tiles(p, s, t0, t0 + p.tokens);
        }
    };
    if (threadIdx.x == 0) {
        bar.init();
        work.init(1 + kGradWarps);
        *gave_up = 0;
        mbar_fence_init();
    }
    if (warp == 2) tmem_alloc(smem_u32(tmem_at), 512);
    fence_before();
    __syncthreads();
    fence_after();
    await_previous();
    const uint32_t tmem = *tmem_at;
    const uint32_t at_s = tmem, at_dp = tmem + 128, at_dq = tmem + 256, at_ds = tmem + 256 + DP;  // two of 64 columns

    if (warp == 0 && elect_one()) {
        int id = blockIdx.x;
        uint32_t step = 0, held = 0;  // key tiles so far; query tiles so far
        bool go = true;
        for (int it = 0; go; ++it) {
            if (!work.put(it, id < pieces ? id : -1, gave_up) || id >= pieces) break;
            const Piece w(p, id);
            id = (int)gridDim.x + atomicAdd(p.sched, 1);
            if (!w.keys.count) continue;
            if (!(go = mbar_wait(bar.held_free, (held & 1) ^ 1, gave_up))) break;
            ++held;
            mbar_expect(bar.held, 2 * p.group * p.tokens * DP * 2);
            load_q_tile<DP>(smem_u32(sq), &mq, bar.held, p, w.t0, w.hk, w.b);
            load_q_tile<DP>(smem_u32(sdo), &mdo, bar.held, p, w.t0, w.hk, w.b);
            for (int j = 0; j < w.keys.count; ++j, ++step) {
                const uint32_t st = step & 1;
                if (!(go = mbar_wait(bar.empty + 8 * st, (step / 2 & 1) ^ 1, gave_up))) break;
                mbar_expect(bar.full + 8 * st, 2 * G::kTileBytes);
                const int k0 = w.keys.at(j) * kTile;
                load_kv_tile<DP>(smem_u32(stage + 2 * st * G::kTileBytes), &mk, bar.full + 8 * st, k0, w.hk, w.b);
                load_kv_tile<DP>(smem_u32(stage + (2 * st + 1) * G::kTileBytes), &mv, bar.full + 8 * st, k0, w.hk,
                                 w.b);
            }
        }
    } else if (warp == 1 && elect_one()) {
        const uint32_t bf = p.a.dtype == HEDDLE_BF16;
        const uint32_t id_s = instr_desc(bf, false, false, kTile), id_d = instr_desc(bf, false, true, DP);
        uint32_t step = 0, held = 0;
        bool go = true;
        for (int it = 0; go; ++it) {
            const int id = work.get(it, gave_up);
            if (id < 0) break;
            const int n = Piece(p, id).keys.count;
            if (!n) continue;
            if (!(go = mbar_wait(bar.held, held & 1, gave_up))) break;
            ++held;
            for (int j = -1; go && j < n; ++j) {
                const uint32_t g = step + j;  // this step among all; scores run one ahead
                if (j + 1 < n) {
                    const uint32_t st = (g + 1) & 1;
                    if (!(go = mbar_wait(bar.full + 8 * st, (g + 1) / 2 & 1, gave_up))) break;
                    if (g + 1 > 0 && !(go = mbar_wait(bar.a_ready, g & 1, gave_up))) break;  // the last scores are read
                    fence_after();
                    mma_dims<DP>(at_s, smem_u32(sq), smem_u32(stage + 2 * st * G::kTileBytes), id_s);
                    mma_dims<DP>(at_dp, smem_u32(sdo), smem_u32(stage + (2 * st + 1) * G::kTileBytes), id_s);
                    commit(bar.a_full);
                    if (j + 2 == n) commit(bar.held_free);
                }
                if (j >= 0) {
                    const uint32_t st = g & 1;
                    if (!(go = mbar_wait(bar.b_ready + 8 * st, g / 2 & 1, gave_up))) break;
                    fence_after();
                    mma_rows<64, 64>(at_dq, at_ds + 64 * st, smem_u32(stage + 2 * st * G::kTileBytes), id_d, j > 0);
                    commit(bar.empty + 8 * st);
                }
            }
            if (go) commit(bar.done);
            step += n;
        }
    } else if (warp >= 2) {
        const int side = (warp - 2) / 4, row = (warp % 4) * 32 + lane;  // which 32 of a tile's 128 keys
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const int i_row = row / p.group, h_row = row % p.group;
        const float c = p.scale_log2;
        const float factor = ds_factor<T>(p), scale = p.a.scale * factor;
        const uint64_t c2 = two(c, c), scale2 = two(scale, scale);
        uint32_t step = 0, held = 0;
        bool go = true;
        for (int it = 0; go; ++it) {
            const int id = work.get_warp(it, gave_up);
            if (id < 0) break;
            const Piece w(p, id);
            const Seq& s = w.s;
            const int n = w.keys.count;
            const int i = w.t0 + i_row, h = w.hk * p.group + h_row;
            const bool inside = row < p.group * p.tokens && i < p.a.q_len;
            const int64_t r = ((int64_t)w.b * p.a.q_heads + h) * p.a.q_len + i;
            const RowMask mask(i < s.ql ? s.off + i : -1, p.a);
            float lse = inside ? p.a.lse[r] : INFINITY;
            lse = lse == -INFINITY ? INFINITY : lse * kLog2e;  // weights of a row that sees nothing are zero
            const float delta = inside ? p.delta[r] * scale : 0.0f;
            const uint64_t lse2 = two(-lse, -lse), delta2 = two(-delta, -delta);
            for (int j = 0; j < n; ++j, ++step) {
                const uint32_t st = step & 1;
                const int k0 = w.keys.at(j) * kTile;
                const bool whole = w.t0 + p.tokens <= s.ql && all_visible(p, s, w.t0, w.t1, k0);
                if (!(go = __all_sync(~0u, mbar_wait(bar.a_full, st, gave_up)))) break;
                fence_after();
                uint32_t v[32], d[32], u[16];
                tmem_ld32(at_s + lanes + side * 32, v);
                tmem_ld32(at_dp + lanes + side * 32, d);
                wait_ld();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.a_ready);
#pragma unroll
                for (int y = 0; y < 32; y += 2) {
                    const float2 z = apart(fma_two(two(v[y], v[y + 1]), c2, lse2));
                    v[y] = __float_as_uint(exp2_fast(z.x)), v[y + 1] = __float_as_uint(exp2_fast(z.y));
                }
                if (whole) {
#pragma unroll
                    for (int y = 0; y < 32; y += 2) {
                        const float2 z = apart(mul_two(two(v[y], v[y + 1]), fma_two(two(d[y], d[y + 1]), scale2, delta2)));
                        d[y] = __float_as_uint(z.x), d[y + 1] = __float_as_uint(z.y);
                    }
                } else {
                    // a product with what lies in hidden places must not count
                    const uint32_t seen = mask.sees32(k0 + side * 32);
#pragma unroll
                    for (int y = 0; y < 32; ++y) {
                        const float e = seen >> y & 1 ? __uint_as_float(v[y]) : 0.0f;
                        d[y] = __float_as_uint(e == 0.0f ? 0.0f : e * fmaf(__uint_as_float(d[y]), scale, -delta));
                    }
                }
#pragma unroll
                for (int y = 0; y < 16; ++y)
                    u[y] = pack_two<T>(__uint_as_float(d[2 * y]), __uint_as_float(d[2 * y + 1]));
                tmem_st16(at_ds + 64 * st + lanes + side * 16, u);
                if (side == 0 && s.kl < p.a.kv_len && k0 + kTile > s.kl) {  // keys past the sequence
                    clear_rows<DP>(stage + 2 * st * G::kTileBytes, row, s.kl - k0);
                    fence_async_shared();
                }
                wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.b_ready + 8 * st);  // a warp may be a step ahead of another
            }
            if (go && n > 0) {
                go = __all_sync(~0u, mbar_wait(bar.done, held & 1, gave_up));
                ++held;
            }
            fence_after();
            if (go && side == 0) {  // the other sides start on the next piece
                T* out = static_cast<T*>(p.dq.data) + w.b * p.dq.batch_stride + i * p.dq.token_stride +
                         h * p.dq.head_stride;
                if (n > 0)
                    store_row<T, DP>(at_dq + lanes, out, inside, p.a.head_dim, 1.0f / factor);
                else if (inside)
                    zero_row(out, p.a.head_dim);
            }
        }
    }
    fence_before();
    __syncthreads();
    if (*gave_up) {
        if (threadIdx.x == 0) atomicOr(p.err, kErrOpWait);
        drain();
        __syncthreads();
    }
    if (threadIdx.x == 0) leave_pieces(p.sched);
    if (warp == 2) tmem_free(tmem, 512);
}

// dq from dS as the pass over keys left it: dq = sum over key tiles of dS K,
// one product of 128 x 128 by 128 x head_dim a step.  Bound by the stream of dS
// from memory, 32 KB a pair of tiles: 54 us for two causal sequences of 2048
// (32 heads over 8 of 128; 114 with the scores computed again).  CTAs take one
// query tile after another, the longest first; sums alternate between two
// places of tensor memory, so that one tile's result is written under the next
// one's products.
template <int DP>
struct StoredShape {
    static constexpr int kTileBytes = kTile * DP * 2;
    static constexpr int kStage = kPlaceBytes + kTileBytes;
    static constexpr int kStages = DP > 64 ? 3 : 4;
    static constexpr int kBars = 16 * kStages + 32 + 32;
    static constexpr int kBytes = 1024 + kStages * kStage + kBars + 32;
    static_assert(kBytes >= kAlone, "see kAlone");
    static constexpr int kThreads = 256;
};

template <class T, int DP>
__global__ void __launch_bounds__(StoredShape<DP>::kThreads, 1)
    attn_dq_stored_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ Params p, const int pieces) {
    using G = StoredShape<DP>;
    extern __shared__ unsigned char raw[];
    unsigned char* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    unsigned char* tail = base + G::kStages * G::kStage;
    const uint32_t full = smem_u32(tail), empty = full + 8 * G::kStages, done = empty + 8 * G::kStages,
                   freed = done + 16;
    const Pieces work{freed + 16, freed + 32, reinterpret_cast<int*>(tail + G::kBars)};
    volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(tail + G::kBars + 8);
    uint32_t* tmem_at = const_cast<uint32_t*>(gave_up) + 1;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    allow_dependents();
    struct Piece {
        int hb, hk, b, tile, t0;
        Seq s;
        KeyTiles keys;
        __device__ Piece(const Params& p, int id) {
            hb = id % p.hbs;
            hk = (p.hb0 + hb) % p.a.kv_heads;
            b = (p.hb0 + hb) / p.a.kv_heads;
            tile = p.q_tiles - 1 - id / p.hbs;
            t0 = tile * p.tokens;
            s = seq_of(p.a, b);
            keys = key_tiles(p, s, t0, t0 + p.tokens);
        }
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < G::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(done + 8 * i, 1);
            mbar_init(freed + 8 * i, 4);
        }
        work.init(1 + 4);
        *gave_up = 0;
        mbar_fence_init();
    }
    if (warp == 2) tmem_alloc(smem_u32(tmem_at), 2 * DP);
    fence_before();
    __syncthreads();
    fence_after();
    await_previous();
    const uint32_t tmem = *tmem_at;

    if (warp == 0 && elect_one()) {
        int id = blockIdx.x, st = 0;
        uint32_t phase = 0;
        bool go = true;
        for (int it = 0; go; ++it) {
            if (!work.put(it, id < pieces ? id : -1, gave_up) || id >= pieces) break;
            const Piece w(p, id);
            id = (int)gridDim.x + atomicAdd(p.sched, 1);
            const unsigned char* from = p.ds + (w.hb * p.ds_head + ds_row(p, w.tile)) * kPlaceBytes;
            for (int j = 0; j < w.keys.count; ++j) {
                if (!(go = mbar_wait(empty + 8 * st, phase ^ 1, gave_up))) break;
                const uint32_t to = smem_u32(base + st * G::kStage), bar = full + 8 * st;
                const int tile = w.keys.at(j);
                mbar_expect(bar, G::kStage);
                load_bytes(to, from + (int64_t)ds_col(p, tile) * kPlaceBytes, kPlaceBytes, bar);
                load_kv_tile<DP>(to + kPlaceBytes, &mk, bar, tile * kTile, w.hk, w.b);
                if (++st == G::kStages) st = 0, phase ^= 1;
            }
        }
    } else if (warp == 1) {
        const bool one = elect_one();
        const uint32_t idesc = instr_desc(p.a.dtype == HEDDLE_BF16, true, true, DP);
        int st = 0;
        uint32_t phase = 0, held = 0;
        bool go = true;
        for (int it = 0; go; ++it) {
            const int id = work.get_warp(it, gave_up);
            if (id < 0) break;
            const Piece w(p, id);
            if (!w.keys.count) continue;
            const uint32_t half = held & 1;
            if (!(go = __all_sync(~0u, mbar_wait(freed + 8 * half, (held / 2 & 1) ^ 1, gave_up)))) break;
            for (int j = 0; j < w.keys.count; ++j) {
                if (!(go = __all_sync(~0u, mbar_wait(full + 8 * st, phase, gave_up)))) break;
                unsigned char* ds = base + st * G::kStage;
                const int k0 = w.keys.at(j) * kTile;
                if (w.s.kl < p.a.kv_len && k0 + kTile > w.s.kl) {  // keys past the sequence
#pragma unroll 1
                    for (int r = lane; r < kTile; r += 32) clear_rows<DP>(ds + kPlaceBytes, r, w.s.kl - k0);
                    fence_async_shared();
                    __syncwarp();
                }
                fence_after();
                if (one) {
                    const uint32_t a = smem_u32(ds), b = a + kPlaceBytes;
#pragma unroll
                    for (int k = 0; k < kTile / 16; ++k)
                        mma_ss(tmem + half * DP, smem_desc_units(a + k * 256, 128, kTile * 16),
                               smem_desc(b + k * 2048, 16384), idesc, j | k);
                    commit(empty + 8 * st);
                }
                if (++st == G::kStages) st = 0, phase ^= 1;
            }
            if (go && one) commit(done + 8 * half);
            ++held;
        }
    } else if (warp >= 4) {
        const int row = (warp % 4) * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const float f = 1.0f / ds_factor<T>(p);
        uint32_t held = 0;
        for (int it = 0;; ++it) {
            const int id = work.get_warp(it, gave_up);
            if (id < 0) break;
            const Piece w(p, id);
            const int i = w.t0 + row / p.group, h = w.hk * p.group + row % p.group;
            const bool inside = row < p.group * p.tokens && i < p.a.q_len;
            T* out = static_cast<T*>(p.dq.data) + w.b * p.dq.batch_stride + i * p.dq.token_stride +
                     h * p.dq.head_stride;
            if (!w.keys.count) {
                if (inside) zero_row(out, p.a.head_dim);
                continue;
            }
            const uint32_t half = held & 1;
            if (!__all_sync(~0u, mbar_wait(done + 8 * half, held / 2 & 1, gave_up))) break;
            ++held;
            fence_after();
            store_row<T, DP>(tmem + half * DP + lanes, out, inside, p.a.head_dim, f);
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(freed + 8 * half);
        }
    }
    fence_before();
    __syncthreads();
    if (*gave_up) {
        if (threadIdx.x == 0) atomicOr(p.err, kErrOpWait);
        drain();
        __syncthreads();
    }
    if (threadIdx.x == 0) leave_pieces(p.sched);
    if (warp == 2) tmem_free(tmem, 2 * DP);
}

// Where the sums of a key tile's part go.
__device__ __forceinline__ int64_t dkv_slot(const Params& p, bool lead, int tile, int hb, int part) {
    const int64_t heads = p.a.batch * p.a.kv_heads;
    if (lead) return (tile * heads + hb) * p.lead_parts + part;
    return (p.lead_parts > 1 ? heads * p.lead * p.lead_parts : 0) + (tile * heads + hb) * p.rest_parts + part;
}

// dk and dv of a key tile, over every query tile that sees it (or a part of
// them: the first tokens of a windowed call are seen by every query, and few
// key tiles alone would leave SMs idle), the group's heads among its rows, so
// that no two CTAs add to one result and sums come in one order.  The scores
// are computed transposed, keys along the lanes, so that P^T and dS^T are left
// operands in tensor memory as they come: S^T = K Q^T, dP^T = V dO^T,
// dv += P^T dO, dk += dS^T Q.  The tensor cores are busy half of the time,
// bound by the chain as above: 120 us for two causal sequences of 2048 (32
// heads over 8 of 128), 101 where dS is not kept.  Tiles of 64 queries in two groups of warps by turns
// took 117: products of 64 columns read their left operand twice as often.
template <class T, int DP>
__global__ void __launch_bounds__(kGradThreads, 1)
    attn_dkv_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                    const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo,
                    const __grid_constant__ Params p) {
    using G = GradShape<DP>;
    extern __shared__ unsigned char raw[];
    unsigned char* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    unsigned char *sk = base, *sv = base + G::kTileBytes, *stage = base + 2 * G::kTileBytes;  // Q, dO, Q, dO
    unsigned char* tail = base + 6 * G::kTileBytes;
    const GradBars bar(smem_u32(tail));
    volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(tail + kGradBarBytes);
    uint32_t* tmem_at = const_cast<uint32_t*>(gave_up) + 1;
    float* stat_lse = reinterpret_cast<float*>(tail + kGradBarBytes + 64);  // [3][128] minus lse, in powers of two
    float* stat_delta = stat_lse + 3 * kTile;                               // [3][128] minus scale delta
    uint32_t* stat_place = reinterpret_cast<uint32_t*>(stat_delta + 3 * kTile);  // [3] the query tile's places
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    allow_dependents();
    // the first keys are seen by the most queries
    const int64_t heads = p.hbs, lead_blocks = heads * p.lead * p.lead_parts;
    const bool lead = blockIdx.x < lead_blocks;
    const int parts = lead ? p.lead_parts : p.rest_parts;
    int64_t id = lead ? blockIdx.x : blockIdx.x - lead_blocks;
    const int part = (int)(id % parts);
    id /= parts;
    const int hb = p.hb0 + (int)(id % heads), hk = hb % p.a.kv_heads, b = hb / p.a.kv_heads;
    const int tile = (int)(id / heads);
    const int k0 = (lead ? tile : p.lead + tile) * kTile;
    const int64_t slot = dkv_slot(p, lead, tile, hb, part);
    const Seq s = seq_of(p.a, b);
    // query tiles that see a key of the tile
    int first = 0, n = 0;
    if (k0 < s.kl) {
        const int lo = max(0, k0 - s.off);
        int hi = s.ql;
        if (p.a.window && k0 >= p.a.sinks) hi = (int)min((int64_t)hi, k0 + kTile - 1 + p.a.window - s.off);
        if (lo < hi) {
            first = lo / p.tokens;
            n = (hi - 1) / p.tokens - first + 1;
            const int from = (int)((int64_t)n * part / parts);
            n = (int)((int64_t)n * (part + 1) / parts) - from;
            first += from;
        }
    }

    auto load_tile = [&](int j, const CUtensorMap* m, int second, uint32_t on) {
        mbar_expect(on + 8 * (j & 1), p.group * p.tokens * DP * 2);
        load_q_tile<DP>(smem_u32(stage + (2 * (j & 1) + second) * G::kTileBytes), m, on + 8 * (j & 1), p,
                        (first + j) * p.tokens, hk, b);
    };
    auto load_q = [&](int j) { load_tile(j, &mq, 0, bar.full); };
    auto load_do = [&](int j) { load_tile(j, &mdo, 1, bar.full2); };
    if (threadIdx.x == 0) {
        bar.init();
        *gave_up = 0;
        mbar_fence_init();
        if (n > 0) {  // the first loads run while the CTA gathers
            mbar_expect(bar.held, 2 * G::kTileBytes);
            load_kv_tile<DP>(smem_u32(sk), &mk, bar.held, k0, hk, b);
            load_q(0);
            load_kv_tile<DP>(smem_u32(sv), &mv, bar.held, k0, hk, b);
            load_do(0);
        }
    }
    if (warp == 2) tmem_alloc(smem_u32(tmem_at), 512);
    if (warp >= 2) {  // rows that no copy writes are zero throughout
        const int row = (threadIdx.x - 64) & 127, rows = p.group * p.tokens;
        clear_rows<DP>(stage + (threadIdx.x - 64) / 128 * G::kTileBytes, row, rows);
        fence_async_shared();
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_at;
    const uint32_t at_s = tmem, at_dp = tmem + 128, at_dv = tmem + 256, at_dk = tmem + 256 + DP;

    if (warp == 0 && n > 0 && elect_one()) {
        for (int j = 1; j < n; ++j) {
            if (!mbar_wait(bar.empty + 8 * (j & 1), (j / 2 & 1) ^ 1, gave_up)) break;
            load_q(j);
            load_do(j);
        }
    } else if (warp == 1 && n > 0 && elect_one()) {
        const uint32_t bf = p.a.dtype == HEDDLE_BF16;
        const uint32_t id_s = instr_desc(bf, false, false, kTile), id_d = instr_desc(bf, false, true, DP);
        bool go = mbar_wait(bar.held, 0, gave_up);
        for (int j = -1; go && j < n; ++j) {
            const int st = j & 1, nx = (j + 1) & 1;
            const uint32_t tq = smem_u32(stage + 2 * st * G::kTileBytes), nq = smem_u32(stage + 2 * nx * G::kTileBytes);
            if (j >= 0) {
                if (!(go = mbar_wait(bar.a_ready, j & 1, gave_up))) break;
                fence_after();
                mma_rows<16, 32>(at_dv, at_s, tq + G::kTileBytes, id_d, j > 0);
            }
            if (j + 1 < n) {
                if (!(go = mbar_wait(bar.full + 8 * nx, (j + 1) / 2 & 1, gave_up))) break;
                fence_after();
                mma_dims<DP>(at_s, smem_u32(sk), nq, id_s);
                commit(bar.a_full);
            }
            if (j >= 0) {
                if (!(go = mbar_wait(bar.b_ready, j & 1, gave_up))) break;
                fence_after();
                mma_rows<16, 32>(at_dk, at_dp, tq, id_d, j > 0);
                commit(bar.empty + 8 * st);
            }
            if (j + 1 < n) {
                if (!(go = mbar_wait(bar.full2 + 8 * nx, (j + 1) / 2 & 1, gave_up))) break;
                fence_after();
                mma_dims<DP>(at_dp, smem_u32(sv), nq + G::kTileBytes, id_s);
                commit(bar.b_full);
            }
        }
        if (go) commit(bar.done);
    } else if (warp >= 2) {
        await_previous();  // for delta and the maxima; everything read before is the caller's
        const int side = (warp - 2) / 4, row = (warp % 4) * 32 + lane;  // which 32 of a tile's 128 queries
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const int key = k0 + row;
        const float factor = ds_factor<T>(p), scale = p.a.scale * factor;
        const uint64_t c2 = two(p.scale_log2, p.scale_log2), scale2 = two(scale, scale);

        // where dS goes, less the query tile's part: all of it is below 2^32 bytes
        const uint32_t ds_at = !p.ds ? 0
                                     : (uint32_t)((hb - p.hb0) * p.ds_head + ds_col(p, k0 / kTile)) * kPlaceBytes +
                                           side * (4 * kTile * 16) + row * 16;

        // statistics of query tile j to buffer j % 3, by three of the sides: written
        // a step ahead, while the slowest warp may still read those of the step
        // before
        const int i_row = first * p.tokens + row / p.group;
        const int64_t r_row = ((int64_t)b * p.a.q_heads + hk * p.group + row % p.group) * p.a.q_len;
        const bool in_tile = row < p.group * p.tokens;
        auto put_stats = [&](int j) {
            const int i = i_row + j * p.tokens;
            const bool live = in_tile && i < s.ql;
            const int to = j % 3 * kTile + row;
            if (side == 0) {
                const float l = live ? p.a.lse[r_row + i] : INFINITY;
                stat_lse[to] = l == -INFINITY ? -INFINITY : -l * kLog2e;
            } else if (side == 1) {
                stat_delta[to] = live ? -p.delta[r_row + i] * scale : 0.0f;
            } else if (side == 2 && row == 0 && p.ds) {
                stat_place[j % 3] = (uint32_t)ds_row(p, first + j) * kPlaceBytes;
            }
        };
        // the tile's columns that see the key: query heads of consecutive tokens
        auto seen_by = [&](int t0) {
            const int last = p.a.window && key >= (int)p.a.sinks
                                 ? (int)min((int64_t)s.ql - 1, key + p.a.window - 1 - s.off)
                                 : s.ql - 1;
            const int lo = max(0, min(key - s.off - t0, p.tokens)), hi = max(0, min(last - t0 + 1, p.tokens));
            return bits_between(lo * p.group - side * 32, hi * p.group - 1 - side * 32);
        };
        bool go = true;
        if (n > 0) {
            put_stats(0);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.stats);
        }
        for (int j = 0; j < n; ++j) {
            if (!(go = __all_sync(~0u, mbar_wait(bar.stats, j & 1, gave_up)))) break;
            if (j + 1 < n) {
                put_stats(j + 1);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.stats);
            }
            const int t0 = (first + j) * p.tokens, t1 = t0 + p.tokens;
            const float4* lses = reinterpret_cast<const float4*>(stat_lse + (j % 3) * kTile + side * 32);
            const float4* deltas = reinterpret_cast<const float4*>(stat_delta + (j % 3) * kTile + side * 32);
            const bool whole = t1 <= s.ql && all_visible(p, s, t0, t1, k0);
            if (!(go = __all_sync(~0u, mbar_wait(bar.a_full, j & 1, gave_up)))) break;
            fence_after();
            uint32_t v[32], w[16];
            tmem_ld32(at_s + lanes + side * 32, v);
            wait_ld();
#pragma unroll
            for (int y = 0; y < 32; y += 4) {
                const float4 f = lses[y / 4];
                const float2 z0 = apart(fma_two(two(v[y], v[y + 1]), c2, two(f.x, f.y)));
                const float2 z1 = apart(fma_two(two(v[y + 2], v[y + 3]), c2, two(f.z, f.w)));
                v[y] = __float_as_uint(exp2_fast(z0.x)), v[y + 1] = __float_as_uint(exp2_fast(z0.y));
                v[y + 2] = __float_as_uint(exp2_fast(z1.x)), v[y + 3] = __float_as_uint(exp2_fast(z1.y));
            }
            if (!whole) {
                const uint32_t seen = seen_by(t0);
#pragma unroll
                for (int y = 0; y < 32; ++y)
                    if (!(seen >> y & 1)) v[y] = 0;
            }
#pragma unroll
            for (int y = 0; y < 16; ++y)
                w[y] = pack_two<T>(__uint_as_float(v[2 * y]), __uint_as_float(v[2 * y + 1]));
            tmem_st16(at_s + lanes + side * 32, w);
            if (side < 2 && s.ql < p.a.q_len && t1 > s.ql) {  // queries past the sequence: side 0 clears Q, 1 dO
                const int st2 = j & 1;
                const uint32_t loaded = side ? bar.full2 : bar.full;
                if (!(go = __all_sync(~0u, mbar_wait(loaded + 8 * st2, j / 2 & 1, gave_up)))) break;
                clear_rows<DP>(stage + (2 * st2 + side) * G::kTileBytes, row, (s.ql - t0) * p.group);
                fence_async_shared();
            }
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.a_ready);

            if (!(go = __all_sync(~0u, mbar_wait(bar.b_full, j & 1, gave_up)))) break;
            fence_after();
            uint32_t d[32];
            tmem_ld32(at_dp + lanes + side * 32, d);
            wait_ld();
#pragma unroll
            for (int y = 0; y < 32; y += 4) {
                const float4 f = deltas[y / 4];
                const float2 z0 =
                    apart(mul_two(two(v[y], v[y + 1]), fma_two(two(d[y], d[y + 1]), scale2, two(f.x, f.y))));
                const float2 z1 =
                    apart(mul_two(two(v[y + 2], v[y + 3]), fma_two(two(d[y + 2], d[y + 3]), scale2, two(f.z, f.w))));
                d[y] = __float_as_uint(z0.x), d[y + 1] = __float_as_uint(z0.y);
                d[y + 2] = __float_as_uint(z1.x), d[y + 3] = __float_as_uint(z1.y);
            }
            if (!whole) {  // a product with what lies in hidden places must not count
#pragma unroll
                for (int y = 0; y < 32; ++y)
                    if (__uint_as_float(v[y]) == 0.0f) d[y] = 0;
            }
#pragma unroll
            for (int y = 0; y < 16; ++y)
                w[y] = pack_two<T>(__uint_as_float(d[2 * y]), __uint_as_float(d[2 * y + 1]));
            tmem_st16(at_dp + lanes + side * 32, w);
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.b_ready);
            if (p.ds) {  // units of 8 queries, the keys of each one after another: a warp writes 512 bytes at a time
                unsigned char* to = p.ds + (ds_at + stat_place[j % 3]);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    *reinterpret_cast<uint4*>(to + y * (kTile * 16)) =
                        make_uint4(w[4 * y], w[4 * y + 1], w[4 * y + 2], w[4 * y + 3]);
            }
        }
        if (go && n > 0) go = __all_sync(~0u, mbar_wait(bar.done, 0, gave_up));
        fence_after();
        if (go) {  // two sides for dv, two for dk, half of the columns each
            const bool is_dk = side & 1;
            const int d0 = side / 2 * (DP / 2), D = p.a.head_dim - d0;
            const uint32_t from = (is_dk ? at_dk : at_dv) + lanes + d0;
            const float f = is_dk ? 1.0f / factor : 1.0f;
            const heddle_heads& t = is_dk ? p.dk : p.dv;
            T* out = static_cast<T*>(t.data) + b * t.batch_stride + key * t.token_stride + hk * t.head_stride + d0;
            const bool inside = key < p.a.kv_len;
            if (parts > 1) {
                float* to = (is_dk ? p.part_dk : p.part_dv) + (slot * kTile + row) * p.a.head_dim + d0;
                if (n > 0)
                    store_floats<DP / 2>(from, to, true, D, f);
                else
                    zero_row(to, min(D, DP / 2));
            } else if (n > 0) {
                store_row<T, DP / 2>(from, out, inside, D, f);
            } else if (inside) {
                zero_row(out, min(D, DP / 2));
            }
        }
    }
    fence_before();
    __syncthreads();
    if (*gave_up) {
        if (threadIdx.x == 0) atomicOr(p.err, kErrOpWait);
        drain();
        __syncthreads();
    }
    if (warp == 2) tmem_free(tmem, 512);
}

// Adds up the parts of key tiles, in order: a block for 8 rows of one.  5 us
// for the windowed call of 4095 tokens whose first tiles come in parts.
template <class T>
__global__ void __launch_bounds__(256) attn_dkv_join_kernel(const __grid_constant__ Params p, int is_lead) {
    allow_dependents();
    await_previous();
    const int lane = threadIdx.x % 32, D = p.a.head_dim;
    const int parts = is_lead ? p.lead_parts : p.rest_parts;
    const int64_t heads = p.a.batch * p.a.kv_heads, unit = blockIdx.x / 16;
    const int hb = (int)(unit % heads), tile = (int)(unit / heads);
    const int row = blockIdx.x % 16 * 8 + threadIdx.x / 32;
    const int64_t key = (int64_t)(is_lead ? tile : p.lead + tile) * kTile + row;
    if (key >= p.a.kv_len || lane * 4 >= D) return;
    const int64_t slot = dkv_slot(p, is_lead, tile, hb, 0);
    for (int side = 0; side < 2; ++side) {
        const float* from = (side ? p.part_dk : p.part_dv) + (slot * kTile + row) * D + lane * 4;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int i = 0; i < parts; ++i) {
            const float4 f = *reinterpret_cast<const float4*>(from + (int64_t)i * kTile * D);
            sum.x += f.x, sum.y += f.y, sum.z += f.z, sum.w += f.w;
        }
        const heddle_heads& t = side ? p.dk : p.dv;
        T* out = static_cast<T*>(t.data) + (hb / p.a.kv_heads) * t.batch_stride + key * t.token_stride +
                 (hb % p.a.kv_heads) * t.head_stride + lane * 4;
        out[0] = from_float<T>(sum.x), out[1] = from_float<T>(sum.y);
        out[2] = from_float<T>(sum.z), out[3] = from_float<T>(sum.w);
    }
}

// --------------------------------------------------------------------- host

bool copies(const heddle_heads& t, int64_t b, int64_t n, int64_t h) {
    auto fits = [](int64_t extent, int64_t stride) {
        return extent == 1 || (stride > 0 && stride % 8 == 0 && stride < ((int64_t)1 << 39));
    };
    return (uintptr_t)t.data % 16 == 0 && fits(b, t.batch_stride) && fits(n, t.token_stride) &&
           fits(h, t.head_stride);
}

cudaError_t heads_map(CUtensorMap* m, const heddle_heads& t, const heddle_attention_args& a, int64_t n, int64_t h,
                      int box_heads, int box_tokens) {
    const uint64_t row = (uint64_t)(a.head_dim + 7) / 8 * 16;  // where an axis has one entry
    const uint64_t dims[4] = {(uint64_t)a.head_dim, (uint64_t)h, (uint64_t)n, (uint64_t)a.batch};
    const uint64_t strides[3] = {h == 1 ? row : (uint64_t)t.head_stride * 2,
                                 n == 1 ? row : (uint64_t)t.token_stride * 2,
                                 a.batch == 1 ? row : (uint64_t)t.batch_stride * 2};
    const uint32_t box[4] = {64, (uint32_t)box_heads, (uint32_t)box_tokens, 1};
    return make_map(m, t.data, a.dtype, 4, dims, strides, box);
}

int tiles_per_block(const heddle_attention_args& a) {
    const int group = a.q_heads / a.kv_heads;
    return a.q_len > kTile / group ? 2 : 1;
}

Params params_of(const OpContext& x, const heddle_attention_args& a) {
    Params p{};
    p.a = a;
    p.group = a.q_heads / a.kv_heads;
    p.tokens = kTile / p.group;
    p.q_tiles = (int32_t)ceil_div(a.q_len, p.tokens);
    p.kv_tiles = (int32_t)ceil_div(a.kv_len, kTile);
    p.scale_log2 = a.scale * kLog2e;
    p.err = x.err;
    p.sched = x.sched;
    // Parts along the keys where the query tiles are too few for the SMs: at
    // least two key tiles each, at most 32 (the join holds one a lane).
    const int nt = tiles_per_block(a);
    const int64_t blocks = ceil_div(p.q_tiles, nt) * a.kv_heads * a.batch;
    int64_t keys = a.kv_len;
    if (a.window) {
        const int64_t reach = a.window + (a.q_len < nt * p.tokens ? a.q_len : nt * p.tokens) + a.sinks + 2 * kTile;
        if (reach < keys) keys = reach;
    }
    int64_t parts = x.num_sms / blocks;
    const int64_t most = keys / (2 * kTile);
    parts = parts < most ? parts : most;
    parts = parts < 1 ? 1 : parts > 32 ? 32 : parts;
    p.splits = (int32_t)parts;
    // a single query tile leaves half of a CTA idle: it takes the tile twice
    p.twins = nt == 1 && keys >= 4 * kTile * parts;
    // Backward over keys: blocks enough for the SMs, of four query tiles at
    // least; the tiles of the first tokens, which every query sees, in parts
    // of about the query tiles that a window's key tile has.
    const int64_t heads = (int64_t)a.batch * a.kv_heads;
    const int64_t near = a.window ? ceil_div(a.window + kTile, p.tokens) + 1 : p.q_tiles;
    const int64_t each = near < p.q_tiles ? near : p.q_tiles;
    int64_t rest = 3 * (int64_t)x.num_sms / (2 * heads * p.kv_tiles);
    rest = rest < each / 4 ? rest : each / 4;
    p.rest_parts = (int32_t)(rest < 1 ? 1 : rest > 32 ? 32 : rest);
    const int64_t sinks = a.sinks < a.kv_len ? a.sinks : a.kv_len;
    p.lead = a.window ? (int32_t)ceil_div(sinks, kTile) : 0;
    // at most 64 parts, and no more than make eight CTAs an SM: their sums are
    // 128 KB a part at heads of 128, 0.3 GB in all, however many tokens stay
    // visible (8192 tokens with 2048 first ones, window 256, 32 heads over 8 of
    // 128: 788 us, and 949 in twice the parts)
    int64_t lead = p.rest_parts * p.q_tiles / (each < 8 ? 8 : each);
    const int64_t enough = p.lead ? ceil_div(8 * (int64_t)x.num_sms, heads * p.lead) : 1;
    lead = lead < enough ? lead : enough;
    p.lead_parts = (int32_t)(lead < p.rest_parts ? p.rest_parts : lead > 64 ? 64 : lead);
    return p;
}

// Whether dS is kept for the pass over queries, and its places.  It is where
// they come to at most kMostKept bytes for as many key heads as the SMs need;
// beyond, the scores are computed in both passes.  Kept: two causal sequences
// of 2048 took 175 us in these two kernels, 215 computed twice; one of 8192 the
// whole backward 1230 and 1380.
constexpr int64_t kMostKept = (int64_t)4 << 30;
int64_t keep_ds(const OpContext& x, Params& p) {
    const heddle_attention_args& a = p.a;
    const int64_t heads = a.batch * a.kv_heads;
    p.hb0 = 0, p.hbs = (int32_t)heads;
    p.ds_lead = a.window ? (int32_t)ceil_div(a.sinks < a.kv_len ? a.sinks : a.kv_len, kTile) : 0;
    const int64_t wrap = a.window ? (a.window + p.tokens - 2) / kTile + 2 : p.kv_tiles;
    if (p.ds_lead + wrap >= p.kv_tiles)
        p.ds_lead = 0, p.ds_wrap = p.kv_tiles;
    else
        p.ds_wrap = (int32_t)wrap;
    p.ds_stride = p.ds_lead + p.ds_wrap;
    p.ds_head = ds_row(p, p.q_tiles);
    if (a.q_lens == a.kv_lens) {  // queries end where keys do: at most as many keys ahead as there are more
        Params q = p;
        const int64_t more = a.kv_len > a.q_len ? a.kv_len - a.q_len : 0;
        q.ds_stride = 0, q.ds_lead = 0, q.ds_wrap = p.kv_tiles, q.ds_reach = (int32_t)(p.tokens - 1 + more);
        q.ds_head = ds_row(q, q.q_tiles);
        if (q.ds_head < p.ds_head) p = q;
    }
    int64_t at_once = kMostKept / kPlaceBytes / (p.ds_head < 1 ? 1 : p.ds_head);
    at_once = at_once < heads ? at_once : heads;
    if (at_once < heads && at_once * p.kv_tiles < 2 * x.num_sms) return 0;
    // the launches alike
    if (at_once) p.hbs = (int32_t)ceil_div(heads, ceil_div(heads, at_once));
    return p.hbs * p.ds_head * kPlaceBytes;
}

// Slots of partial sums of the backward pass over keys.
int64_t dkv_slots(const Params& p) {
    const int64_t heads = (int64_t)p.a.batch * p.a.kv_heads;
    return heads * ((p.lead_parts > 1 ? (int64_t)p.lead * p.lead_parts : 0) +
                    (p.rest_parts > 1 ? (int64_t)(p.kv_tiles - p.lead) * p.rest_parts : 0));
}

template <class T, int DP, int NT, bool TWINS>
cudaError_t forward(const OpContext& x, const Params& p, const CUtensorMap& q, const CUtensorMap& k,
                    const CUtensorMap& v,
                    cudaStream_t st) {
    using F = Forward<DP, NT>;
    static_assert(F::kSlots >= 4, "two steps of K and V");
    static_assert(F::kBytes >= kAlone, "see kAlone");
    auto* f = attn_kernel<T, DP, NT, TWINS>;
    static std::atomic<uint64_t> asked{0};
    const cudaError_t e = allow_shared(f, F::kBytes, x.device, asked);
    if (e != cudaSuccess) return e;
    const int64_t pieces = ceil_div(p.q_tiles, TWINS ? 1 : NT) * p.a.batch * p.a.kv_heads * p.splits;
    launch(x, f, dim3((unsigned)pieces), F::kThreads, F::kBytes, st, q, k, v, p);
    if (p.splits > 1) {
        const int64_t rows = p.a.batch * p.a.q_heads * p.a.q_len;
        launch(x, attn_join_kernel<T>, dim3((unsigned)ceil_div(rows, 8)), 256, 0, st, p);
    }
    return cudaGetLastError();
}

template <class T, int DP>
cudaError_t backward(const OpContext& x, Params p, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v,
                     const CUtensorMap& d_o, cudaStream_t st) {
    using G = GradShape<DP>;
    using S = StoredShape<DP>;
    static std::atomic<uint64_t> asked_q{0}, asked_kv{0}, asked_s{0};
    cudaError_t e = allow_shared(attn_dkv_kernel<T, DP>, G::kBytes, x.device, asked_kv);
    if (e == cudaSuccess && !p.ds) e = allow_shared(attn_dq_kernel<T, DP>, G::kBytes, x.device, asked_q);
    if (e == cudaSuccess && p.ds) e = allow_shared(attn_dq_stored_kernel<T, DP>, S::kBytes, x.device, asked_s);
    if (e != cudaSuccess) return e;
    const int64_t heads = p.a.batch * p.a.kv_heads, tiles = p.lead * p.lead_parts +
                                                            (int64_t)(p.kv_tiles - p.lead) * p.rest_parts;
    const int each = p.hbs;
    for (p.hb0 = 0; p.hb0 < heads; p.hb0 += each) {
        p.hbs = (int32_t)(heads - p.hb0 < each ? heads - p.hb0 : each);
        launch(x, attn_dkv_kernel<T, DP>, dim3((unsigned)(p.hbs * tiles)), kGradThreads, G::kBytes, st, q, k, v, d_o,
               p);
        const int64_t pieces = (int64_t)p.q_tiles * p.hbs, grid = pieces < x.num_sms ? pieces : x.num_sms;
        if (p.ds)
            launch(x, attn_dq_stored_kernel<T, DP>, dim3((unsigned)grid), S::kThreads, S::kBytes, st, k, p,
                   (int)pieces);
        else
            launch(x, attn_dq_kernel<T, DP>, dim3((unsigned)grid), kGradThreads, G::kBytes, st, q, k, v, d_o, p,
                   (int)pieces);
    }
    if (p.lead_parts > 1 && p.lead)
        launch(x, attn_dkv_join_kernel<T>, dim3((unsigned)(heads * p.lead * 16)), 256, 0, st, p, 1);
    if (p.rest_parts > 1 && p.kv_tiles > p.lead)
        launch(x, attn_dkv_join_kernel<T>, dim3((unsigned)(heads * (p.kv_tiles - p.lead) * 16)), 256, 0, st, p, 0);
    return cudaGetLastError();
}

template <class T>
cudaError_t forward_of(const OpContext& x, const Params& p, const CUtensorMap& q, const CUtensorMap& k,
                       const CUtensorMap& v,
                       cudaStream_t st) {
    const bool two = tiles_per_block(p.a) == 2;
    if (p.a.head_dim <= 64)
        return two       ? forward<T, 64, 2, false>(x, p, q, k, v, st)
               : p.twins ? forward<T, 64, 2, true>(x, p, q, k, v, st)
                         : forward<T, 64, 1, false>(x, p, q, k, v, st);
    return two       ? forward<T, 128, 2, false>(x, p, q, k, v, st)
           : p.twins ? forward<T, 128, 2, true>(x, p, q, k, v, st)
                     : forward<T, 128, 1, false>(x, p, q, k, v, st);
}

cudaError_t input_maps(const Params& p, CUtensorMap* q, CUtensorMap* k, CUtensorMap* v) {
    const heddle_attention_args& a = p.a;
    cudaError_t e = heads_map(q, a.q, a, a.q_len, a.q_heads, p.group, p.tokens);
    if (e == cudaSuccess) e = heads_map(k, a.k, a, a.kv_len, a.kv_heads, 1, kTile);
    if (e == cudaSuccess) e = heads_map(v, a.v, a, a.kv_len, a.kv_heads, 1, kTile);
    return e;
}

}  // namespace

// head_dim in whole 16-byte units, at most 128, and bases and strides that
// bulk tensor copies take; a scale whose sign keeps the order of scores.
bool attn_tc_takes(const heddle_attention_args& a) {
    return a.q_len <= kMaxLength && a.kv_len <= kMaxLength && a.head_dim % 8 == 0 && a.head_dim <= 128 &&
           a.q_heads / a.kv_heads <= kTile && a.scale > 0.0f &&
           a.q_len > 0 && a.kv_len > 0 && copies(a.q, a.batch, a.q_len, a.q_heads) &&
           copies(a.k, a.batch, a.kv_len, a.kv_heads) && copies(a.v, a.batch, a.kv_len, a.kv_heads);
}
bool attn_tc_takes_grad(const heddle_attention_grad_args& g) {
    return attn_tc_takes(g.fwd) && copies(g.d_o, g.fwd.batch, g.fwd.q_len, g.fwd.q_heads);
}

size_t attn_tc_scratch(const OpContext& x, const heddle_attention_args& a) {
    const Params p = params_of(x, a);
    if (p.splits == 1) return 0;
    const size_t rows = (size_t)(a.batch * a.q_heads * a.q_len) * p.splits;
    return align256(rows * a.head_dim * 4) + align256(rows * 4);
}

cudaError_t launch_attn_tc(const OpContext& x, const heddle_attention_args& a, unsigned char* ws, cudaStream_t st) {
    Params p = params_of(x, a);
    if (p.splits > 1) {
        const size_t rows = (size_t)(a.batch * a.q_heads * a.q_len) * p.splits;
        p.part_o = reinterpret_cast<float*>(ws);
        p.part_lse = reinterpret_cast<float*>(ws + align256(rows * a.head_dim * 4));
    }
    CUtensorMap q, k, v;
    const cudaError_t e = input_maps(p, &q, &k, &v);
    if (e != cudaSuccess) return e;
    return a.dtype == HEDDLE_BF16 ? forward_of<__nv_bfloat16>(x, p, q, k, v, st)
                                  : forward_of<__half>(x, p, q, k, v, st);
}

size_t attn_tc_grad_scratch(const OpContext& x, const heddle_attention_args& a, bool keep) {
    Params p = params_of(x, a);
    const size_t kept = keep_ds(x, p);
    return 2 * align256((size_t)dkv_slots(p) * kTile * a.head_dim * 4) + (keep ? kept : 0);
}

cudaError_t launch_attn_tc_grad(const OpContext& x, const heddle_attention_grad_args& g, const float* delta,
                                unsigned char* ws, bool keep, cudaStream_t st) {
    const heddle_attention_args& a = g.fwd;
    Params p = params_of(x, a);
    const size_t parts = attn_tc_grad_scratch(x, a, false);
    p.part_dk = reinterpret_cast<float*>(ws);
    p.part_dv = reinterpret_cast<float*>(ws + parts / 2);
    const int64_t kept = keep_ds(x, p);
    if (keep && kept)
        p.ds = ws + parts;
    else
        p.hbs = (int32_t)(a.batch * a.kv_heads);
    p.d_o = g.d_o, p.dq = g.dq, p.dk = g.dk, p.dv = g.dv;
    p.delta = delta;
    CUtensorMap q, k, v, d_o;
    cudaError_t e = input_maps(p, &q, &k, &v);
    if (e == cudaSuccess) e = heads_map(&d_o, g.d_o, a, a.q_len, a.q_heads, p.group, p.tokens);
    if (e != cudaSuccess) return e;
    const bool narrow = a.head_dim <= 64;
    if (a.dtype == HEDDLE_BF16)
        return narrow ? backward<__nv_bfloat16, 64>(x, p, q, k, v, d_o, st)
                      : backward<__nv_bfloat16, 128>(x, p, q, k, v, d_o, st);
    return narrow ? backward<__half, 64>(x, p, q, k, v, d_o, st)
                  : backward<__half, 128>(x, p, q, k, v, d_o, st);
}

}  // namespace hd
