// heddle_embedding.cu -- the embedding and the gradient of its table.
//
// Bound by memory: rows are copied, and the gradient's rows are written once
// each.  The gradient sorts (row, token) pairs, by one CTA or a cluster, so that
// a row's terms lie together in the order of their tokens; then blocks add up
// runs of the sorted list, others write zeros to the rows that have no token,
// and the sums of rows that go over several runs are joined in order.
// 16384 tokens as words fall on 131072 rows of 4096 bfloat16 values: 31 us for the
// rows, 205 for the gradient (1.2 GB); launched one by one its kernels take 17 to
// sort, 176 for sums and zeros, 10 to join.

#include <atomic>

#include "heddle_rows.cuh"
#include "heddle_tc.cuh"

namespace hd {
namespace {

// The table's row of a token, -1 for none; a token past the vocabulary says so.
__device__ __forceinline__ int64_t row_of(const heddle_embedding_args& a, int64_t t, bool& past) {
    const int64_t id =
        a.wide_tokens ? static_cast<const int64_t*>(a.token)[t] : static_cast<const int32_t*>(a.token)[t];
    past = id >= a.vocab;
    return id < a.first || id - a.first >= a.table_rows || id < 0 || past ? -1 : id - a.first;
}

constexpr int kThreads = 128;

// GL threads a token's row, U units of 16 bytes a thread: those that the
// output's row is made of; TOKENS of them one after the other, their loads
// together.
// WHOLE: rows of whole units at 16 bytes; else units are put together from the
// two of the table that hold them, and the row's ends go value by value.
template <class T, int GL, int U, int TOKENS, bool WHOLE>
__global__ void __launch_bounds__(kThreads)
    embedding_kernel(const __grid_constant__ heddle_embedding_args a, uint32_t* err) {
    allow_dependents();
    await_previous();
    constexpr int V = 16 / sizeof(T), kGroups = kThreads / GL;
    const int lane = threadIdx.x % GL, cols = (int)a.cols, u0 = blockIdx.y * GL * U + lane;
    const int64_t t0 = (int64_t)blockIdx.x * kGroups * TOKENS + threadIdx.x / GL;
    const float2 scale = both(a.scale);
    const T* table = static_cast<const T*>(a.table);
    T* const y = static_cast<T*>(a.y) + t0 * a.ldy;
    const int64_t y_step = kGroups * a.ldy;
    int row[TOKENS], head[TOKENS];  // the values before the output's first unit
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
        const int64_t t = t0 + j * kGroups;
        bool past = false;
        row[j] = t < a.tokens ? (int)row_of(a, t, past) : -1;
        if (past && blockIdx.y == 0 && lane == 0) atomicOr(err, kErrOpToken);
        head[j] = 0;
        if (!WHOLE) {
            head[j] = (0 - (low_of(y) + (uint32_t)(j * y_step * sizeof(T))) & 15) / (uint32_t)sizeof(T);
            head[j] = head[j] < cols ? head[j] : cols;
        }
    }
    uint4 v[TOKENS][U];
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
        const T* src = table + (row[j] * a.ldt + head[j]);
        const uint32_t skew = WHOLE ? 0 : low_of(src) & 15;
        const unsigned char* from = reinterpret_cast<const unsigned char*>(src) - skew + u0 * 16;
        const int units = row[j] >= 0 ? (cols - head[j]) / V : 0;
#pragma unroll
        for (int k = 0; k < U; ++k)
            v[j][k] = u0 + k * GL < units ? load_skewed(from + k * GL * 16, skew) : make_uint4(0, 0, 0, 0);
    }
    if (!WHOLE && blockIdx.y == 0 && lane < V) {  // the rows' ends: at most V - 1 values on either side
#pragma unroll
        for (int j = 0; j < TOKENS; ++j) {
            if (t0 + j * kGroups >= a.tokens) break;
            const int tail = head[j] + (cols - head[j]) / V * V + lane;
            const T* src = table + row[j] * a.ldt;
            T* dst = y + j * y_step;
            if (lane < head[j]) dst[lane] = from_float<T>(row[j] >= 0 ? to_float(src[lane]) * a.scale : 0.0f);
            if (tail < cols) dst[tail] = from_float<T>(row[j] >= 0 ? to_float(src[tail]) * a.scale : 0.0f);
        }
    }
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
        if (t0 + j * kGroups >= a.tokens) break;
        T* dst = y + j * y_step + head[j] + u0 * V;
        const int units = (cols - head[j]) / V;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (u0 + k * GL >= units) break;
            if (a.scale != 1.0f && row[j] >= 0) {
                uint32_t w[4] = {v[j][k].x, v[j][k].y, v[j][k].z, v[j][k].w};
#pragma unroll
                for (int p = 0; p < V / 2; ++p) set_pair<T>(w, p, mul2(pair_of<T>(w, p), scale));
                v[j][k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            *reinterpret_cast<uint4*>(dst + k * GL * V) = v[j][k];
        }
    }
}

// -------------------------------------------------------------------- sorting

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kDigits = 512;

struct Entry {
    uint32_t row, token;
};

struct Sort {
    heddle_embedding_args a;
    int32_t passes, bits;
    Entry* list[2];  // by turns; the last pass leaves its result in list[passes & 1]
    int64_t* count;  // entries of rows of the table; and of rows that go over several runs, from zero
    uint32_t* err;
};

__device__ __forceinline__ uint32_t load_of_rank(const uint32_t* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(tc::cluster_at(tc::smem_u32(p), rank)) : "memory");
    return v;
}

template <int CTAS>
__device__ __forceinline__ void meet() {
    if constexpr (CTAS > 1)
        tc::cluster_sync();
    else
        __syncthreads();
}

// A stable sort by the row, `bits` bits a pass from the lowest.  Each warp of
// the cluster has a run of the list: it counts its digits, its places in the
// result follow from the counts of all warps before it, and it walks over its
// run again in order.
template <int CTAS>
__device__ __forceinline__ void sort_pass(const Sort& s, int pass, int64_t n, uint32_t (*counts)[kDigits],
                                          uint32_t* total, uint32_t* base, uint32_t* scan) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = CTAS > 1 ? tc::cluster_rank() : 0;
    const Entry* from = s.list[pass & 1];
    Entry* to = s.list[(pass & 1) ^ 1];
    const int shift = pass * s.bits, digits = 1 << s.bits;
    const int64_t run = ceil_div(n, CTAS * kSortWarps), first = (rank * kSortWarps + warp) * run;
    const int64_t end = first + run < n ? first + run : n;
    // entry i; false where it is none of the table's
    auto entry = [&](int64_t i, Entry& e, bool flag) {
        if (i >= end) return false;
        if (pass) {
            e = from[i];
            return true;
        }
        bool past;
        const int64_t row = row_of(s.a, i, past);
        if (past && flag) atomicOr(s.err, kErrOpToken);
        e = {(uint32_t)row, (uint32_t)i};
        return row >= 0;
    };
    for (int d = lane; d < digits; d += 32) counts[warp][d] = 0;
    __syncwarp();
    // a short run stays in registers for the second walk
    constexpr int kHeld = 4;
    Entry held[kHeld];
    bool is_held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) is_held[k] = entry(first + k * 32 + lane, held[k], true);
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (is_held[k]) atomicAdd(&counts[warp][held[k].row >> shift & (digits - 1)], 1u);
    for (int64_t i = first + kHeld * 32 + lane; i < end; i += 32) {
        Entry e;
        if (entry(i, e, true)) atomicAdd(&counts[warp][e.row >> shift & (digits - 1)], 1u);
    }
    __syncthreads();
    // before this warp among the CTA's warps, and the CTA's own count
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
        uint32_t sum = 0;
#pragma unroll 8
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t c = counts[w][d];
            counts[w][d] = sum;
            sum += c;
        }
        total[d] = sum;
    }
    meet<CTAS>();
    // before this CTA: all of the smaller digits, and this digit's of the CTAs before
    uint32_t all = 0, before = 0;
    const int d = threadIdx.x;
    if (d < digits) {
        if constexpr (CTAS > 1) {
#pragma unroll
            for (int r = 0; r < CTAS; ++r) {
                const uint32_t c = load_of_rank(total + d, r);
                before += r < (int)rank ? c : 0;
                all += c;
            }
        } else {
            all = total[d];
        }
    }
    uint32_t up = all;  // inclusive, over the warp, then over warps
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(~0u, up, o);
        up += lane >= o ? v : 0;
    }
    if (lane == 31) scan[warp] = up;
    __syncthreads();
    if (warp == 0) {
        uint32_t v = scan[lane];
        const uint32_t own = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t w = __shfl_up_sync(~0u, v, o);
            v += lane >= o ? w : 0;
        }
        scan[lane] = v - own;
        if (lane == 31 && rank == 0 && pass == 0) s.count[0] = v, s.count[1] = 0;
    }
    __syncthreads();
    if (d < digits) base[d] = scan[warp] + up - all + before;
    __syncthreads();
    auto place = [&](const Entry& e, bool is) {
        const uint32_t digit = is ? e.row >> shift & (digits - 1) : (uint32_t)kDigits;
        const uint32_t same = __match_any_sync(~0u, digit);
        const uint32_t ahead = __popc(same & ((1u << lane) - 1));
        uint32_t at = 0;
        if (is) {
            at = counts[warp][digit];
            to[base[digit] + at + ahead] = e;
        }
        __syncwarp();
        if (is && ahead == 0) counts[warp][digit] = at + __popc(same);
        __syncwarp();
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (first + k * 32 < end) place(held[k], is_held[k]);
    for (int64_t i0 = first + kHeld * 32; i0 < end; i0 += 32) {
        Entry e{};
        const bool is = entry(i0 + lane, e, false);
        place(e, is);
    }
    meet<CTAS>();  // the next pass reads what all wrote, and its counts take these ones' place
}

template <int CTAS>
__global__ void __launch_bounds__(kSortThreads) __cluster_dims__(CTAS, 1, 1)
    embedding_sort_kernel(const __grid_constant__ Sort s) {
    allow_dependents();
    await_previous();
    extern __shared__ uint32_t shared[];
    auto* counts = reinterpret_cast<uint32_t(*)[kDigits]>(shared);
    uint32_t *total = shared + kSortWarps * kDigits, *base = total + kDigits, *scan = base + kDigits;
    int64_t n = s.a.tokens;
    for (int pass = 0; pass < s.passes; ++pass) {
        sort_pass<CTAS>(s, pass, n, counts, total, base, scan);
        if (pass == 0) n = *s.count;
    }
}
constexpr int kSortShared = (kSortWarps * kDigits + 2 * kDigits + 32) * 4;

// ----------------------------------------------------------------------- sums

struct Sums {
    heddle_embedding_args a;  // y: the gradient in
    void* out;
    const Entry* list;
    int64_t* count;      // of entries, and of rows that go over several runs
    uint32_t* crossing;  // the runs that these begin in
    float* partial;      // [chunk][2][cols]
    int32_t chunk;       // entries a block
    int32_t accumulate;
    int32_t out_whole;  // the gradient's rows are whole units at 16 bytes
    // blocks that write zeros to the rows without tokens, behind the others: many
    // small ones even out what memory gives each (two an SM: 404 us where eight
    // take 205, 16384 tokens and 131072 x 4096 bfloat16)
    unsigned fillers;
};

// Zeros to the gradient's rows that the sorted list does not name, a range of
// rows a block: kWindow of them are marked at a time, the others written by
// bulk copies out of shared memory where they lie at 16 bytes.  Entries of the
// window are gone through, or, where they are many for its rows (padding tokens
// of one row), searched for each: 262144 tokens of one row, 32000 rows, took
// 2.9 ms with one thread after the other in place of 0.7.
constexpr int kWindow = 8192, kZeros = 8192;
constexpr int kScan = 8;  // entries of the list that a thread waits for together

// The first entry of lo .. hi whose row is `row` or behind it, hi if there is
// none: 32 probes at a time, by a whole warp.
__device__ __forceinline__ int64_t first_of(const Entry* list, int64_t lo, int64_t hi, int64_t row) {
    const int lane = threadIdx.x % 32;
    while (lo < hi) {
        const int64_t step = ceil_div(hi - lo, 32), at = lo + step * lane;
        const int below = __popc(__ballot_sync(~0u, at < hi && list[at].row < row));
        if (below == 0) break;
        hi = lo + step * below < hi ? lo + step * below : hi;
        lo += step * (below - 1) + 1;
    }
    return lo;
}

template <class TO>
__device__ __noinline__ void fill_rows(const Sums& s, int64_t part) {
    __shared__ uint32_t marks[kWindow / 32];
    __shared__ __align__(128) unsigned char zeros[kZeros];
    const int64_t rows = s.a.table_rows, each = ceil_div(rows, (int64_t)s.fillers), r0 = part * each;
    const int64_t r1 = r0 + each < rows ? r0 + each : rows, n = *s.count;
    TO* out = static_cast<TO*>(s.out);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t bytes = s.a.cols * (int64_t)sizeof(TO);
    const bool bulk = ((uintptr_t)out | (uintptr_t)(s.a.ldt * sizeof(TO)) | (uintptr_t)bytes) % 16 == 0;
    for (int i = threadIdx.x; i < kZeros / 16; i += kThreads)
        reinterpret_cast<uint4*>(zeros)[i] = make_uint4(0, 0, 0, 0);
    tc::fence_async_shared();
    for (int64_t from = r0; from < r1; from += kWindow) {
        const int64_t to = from + kWindow < r1 ? from + kWindow : r1;
        __syncthreads();
        for (int i = threadIdx.x; i < ceil_div(to - from, 32); i += kThreads) marks[i] = 0;
        __syncthreads();
        // its entries; few are gone through, many are searched for its rows
        const int64_t lo = first_of(s.list, 0, n, from), hi = first_of(s.list, lo, n, to);
        auto mark = [&](int64_t row) {
            const uint32_t bit = 1u << ((row - from) % 32);
            uint32_t& word = marks[(row - from) / 32];
            if (!(*(volatile uint32_t*)&word & bit)) atomicOr(&word, bit);
        };
        const int64_t a_row = 64 - __clzll(hi - lo);
        if (ceil_div(hi - lo, kScan * kThreads) <= ceil_div(to - from, kThreads) * a_row) {
            for (int64_t i = lo + threadIdx.x; i < hi; i += kScan * kThreads) {
                uint32_t rows[kScan];
#pragma unroll
                for (int k = 0; k < kScan; ++k)
                    if (i + k * kThreads < hi) rows[k] = s.list[i + k * kThreads].row;
#pragma unroll
                for (int k = 0; k < kScan; ++k)
                    if (i + k * kThreads < hi) mark(rows[k]);
            }
        } else {
            for (int64_t row = from + threadIdx.x; row < to; row += kThreads) {
                int64_t i = lo, end = hi;
                while (i < end) {
                    const int64_t mid = (i + end) / 2;
                    if (s.list[mid].row < row)
                        i = mid + 1;
                    else
                        end = mid;
                }
                if (i < hi && s.list[i].row == row) mark(row);
            }
        }
        __syncthreads();
        if (bulk) {  // a row a thread
            for (int64_t row = from + threadIdx.x; row < to; row += kThreads) {
                if (marks[(row - from) / 32] >> ((row - from) % 32) & 1) continue;
                unsigned char* p = reinterpret_cast<unsigned char*>(out + row * s.a.ldt);
                for (int64_t at = 0; at < bytes; at += kZeros) {
                    const uint32_t size = (uint32_t)(bytes - at < kZeros ? bytes - at : kZeros);
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(
                                     __cvta_generic_to_global(p + at)),
                                 "r"(tc::smem_u32(zeros)), "r"(size)
                                 : "memory");
                }
            }
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            continue;
        }
        for (int64_t row = from + warp; row < to; row += kThreads / 32) {
            if (marks[(row - from) / 32] >> ((row - from) % 32) & 1) continue;
            TO* p = out + row * s.a.ldt;
            // to 16 bytes, whole units, the rest
            const int64_t head = (16 - (uintptr_t)p % 16) % 16 / sizeof(TO);
            const int64_t start = head < s.a.cols ? head : s.a.cols, units = (s.a.cols - start) * sizeof(TO) / 16;
            const int64_t tail = start + units * (16 / sizeof(TO));
            if (lane < start) p[lane] = from_float<TO>(0.0f);
            for (int64_t u = lane; u < units; u += 32) reinterpret_cast<uint4*>(p + start)[u] = make_uint4(0, 0, 0, 0);
            if (tail + lane < s.a.cols) p[tail + lane] = from_float<TO>(0.0f);
        }
    }
    // the copies read shared memory, and the rows are written when the kernel ends
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// A row's sums to the gradient: in 16-byte units, or value by value.
template <class TO, class R>
__device__ __forceinline__ void add_out(const Sums& s, const R& part, int64_t row, int64_t from,
                                        const float (&sum)[R::N]) {
    TO* p = static_cast<TO*>(s.out) + row * s.a.ldt + from;
    if (s.out_whole) {
        if (!part.in(0)) return;
        constexpr int VO = 16 / sizeof(TO);
        uint4* at = reinterpret_cast<uint4*>(p + part.at(0));
        uint4 base[R::N / VO];
#pragma unroll
        for (int u = 0; u < R::N / VO; ++u) base[u] = s.accumulate ? at[u] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < R::N / VO; ++u) {
            float f[VO];
            unpack<TO>(base[u], f);
#pragma unroll
            for (int e = 0; e < VO; ++e) f[e] = fmaf(sum[u * VO + e], s.a.scale, f[e]);
            at[u] = pack<TO>(f);
        }
        return;
    }
    float base[R::N];
#pragma unroll
    for (int e = 0; e < R::N; ++e) base[e] = s.accumulate && part.in(e) ? to_float(p[part.at(e)]) : 0.0f;
#pragma unroll
    for (int e = 0; e < R::N; ++e)
        if (part.in(e)) p[part.at(e)] = from_float<TO>(fmaf(sum[e], s.a.scale, base[e]));
}

constexpr int kAhead = 8;  // rows fetched before any is added
constexpr int kLeastRun = 8, kMostRun = 512;  // entries a block

// A run of the sorted list and a range of columns a block.  A row whose
// entries all lie in the run is written; the sums of one that began before it
// go to partial[.][0], of one that goes on behind it to partial[.][1].  The
// last blocks write zeros to the other rows.
template <class T, class TO, bool WHOLE>
__global__ void __launch_bounds__(kThreads)
    embedding_sums_kernel(const __grid_constant__ Sums s, unsigned slabs) {
    allow_dependents();
    await_previous();
    const unsigned sums = gridDim.x - s.fillers, block = blockIdx.x;
    if (block >= sums) {
        fill_rows<TO>(s, block - sums);
        return;
    }
    using R = RowPart<T, 1, false>;
    constexpr int kCols = kThreads * R::N;
    __shared__ Entry run[kMostRun + 2];  // with the one before and the one behind
    const unsigned chunk = block / slabs, slab = block % slabs;
    const int64_t first = (int64_t)chunk * s.chunk, from = (int64_t)slab * kCols;
    // entries past the last are in the list's place, and not used
    for (int i = threadIdx.x; i < s.chunk + 2; i += kThreads)
        if (first + i >= 1 && first + i <= s.a.tokens) run[i] = s.list[first + i - 1];
    const int64_t n = *s.count;
    if (first >= n) return;
    __syncthreads();
    const int end = (int)(first + s.chunk < n ? s.chunk : n - first);
    const int64_t left = s.a.cols - from;
    const R part{(int)threadIdx.x, kThreads, (int)(left < kCols ? left : kCols)};
    const T* dy = static_cast<const T*>(s.a.y) + from;
    const uint32_t before = first ? run[0].row : ~0u, behind = first + end < n ? run[end + 1].row : ~0u;
    float* partial = s.partial + (int64_t)chunk * 2 * s.a.cols + from;
    float sum[R::N] = {};
    uint32_t row = run[1].row;
    bool began = row == before;
    auto finish = [&](bool goes_on) {
        if (began || goes_on) {
            float* p = partial + (began ? 0 : s.a.cols);
#pragma unroll
            for (int e = 0; e < R::N; ++e)
                if (part.in(e)) p[part.at(e)] = sum[e];
        } else {
            add_out<TO>(s, part, row, from, sum);
        }
    };
    for (int i = 0; i < end; i += kAhead) {
        uint32_t v[kAhead][R::kWords];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= end) break;
            const T* from = dy + (int64_t)run[i + k + 1].token * s.a.ldy;
            if (WHOLE) {
                part.load(v[k], from, true);
            } else if (part.in(0)) {  // what lies past the row's end counts for nothing
                const int valid = part.cols - part.at(0);
                from += part.at(0);
                const uint32_t skew = low_of(from) & 15;
                const uint4 u = load_skewed(reinterpret_cast<const unsigned char*>((uintptr_t)from - skew), skew,
                                            skew + valid * sizeof(T) > 16);
                v[k][0] = u.x, v[k][1] = u.y, v[k][2] = u.z, v[k][3] = u.w;
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= end) break;
            if (run[i + k + 1].row != row) {
                finish(false);
                row = run[i + k + 1].row, began = false;
#pragma unroll
                for (int e = 0; e < R::N; ++e) sum[e] = 0.0f;
            }
#pragma unroll
            for (int p = 0; p < R::N / 2; ++p) {
                const float2 f = pair_of<T>(v[k], p);
                sum[2 * p] += f.x, sum[2 * p + 1] += f.y;
            }
        }
    }
    finish(row == behind);
    if (row == behind && !began && slab == 0 && threadIdx.x == 0)
        s.crossing[atomicAdd(reinterpret_cast<unsigned long long*>(s.count + 1), 1ull)] = chunk;
}

// Rows that go over several runs, 1024 columns of one a block at a time: 262144
// tokens of 1024 values, half of one row, take 234 us, 346 with the runs' parts
// fetched one after the other.  (A block for every run, most of which have
// nothing to do, took 40 us for 16384 tokens where this takes 10; narrow slabs,
// each with the search and its waits, 36.)
constexpr int kJoinThreads = 256, kJoinCols = 4 * kJoinThreads;
constexpr int kJoinAhead = 16;  // runs that a thread waits for together
template <class TO>
__global__ void __launch_bounds__(kJoinThreads)
    embedding_join_kernel(const __grid_constant__ Sums s, unsigned slabs) {
    allow_dependents();
    await_previous();
    const int lane = threadIdx.x % 32;
    const int64_t n = s.count[0], work = s.count[1] * slabs;
    for (int64_t i = blockIdx.x; i < work; i += gridDim.x) {
        const int64_t begin = s.crossing[i / slabs], col = i % slabs * kJoinCols + threadIdx.x;
        const uint32_t row = s.list[(begin + 1) * s.chunk].row;
        // the runs that it goes on into, those that start with it: from `last`
        // on, `none` is not one; 32 probes at a time
        int64_t last = begin + 1, none = ceil_div(n, s.chunk);
        while (none - last > 1) {
            const int64_t step = ceil_div(none - last, 32), at = last + step * lane;
            const unsigned is = __ballot_sync(~0u, at < none && s.list[at * s.chunk].row == row);
            const int64_t found = last + step * (31 - __clz(is));  // the first probe always is
            none = found + step < none ? found + step : none;
            last = found;
        }
        const float* from = s.partial + begin * 2 * s.a.cols + col;
        float sum[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            sum[k] = col + k * kJoinThreads < s.a.cols ? from[s.a.cols + k * kJoinThreads] : 0.0f;
        for (int64_t p = begin + 1; p <= last; p += kJoinAhead) {
            float v[kJoinAhead][4];
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j) {
                from += 2 * s.a.cols;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[j][k] = p + j <= last && col + k * kJoinThreads < s.a.cols ? from[k * kJoinThreads] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j) {
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] += v[j][k];
            }
        }
        TO* p = static_cast<TO*>(s.out) + row * s.a.ldt + col;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (col + k * kJoinThreads >= s.a.cols) break;
            const float base = s.accumulate ? to_float(p[k * kJoinThreads]) : 0.0f;
            p[k * kJoinThreads] = from_float<TO>(fmaf(sum[k], s.a.scale, base));
        }
    }
}

// -------------------------------------------------------------------- launches

template <class T, int GL, int U, int TOKENS, bool WHOLE>
cudaError_t lookup(const OpContext& x, const heddle_embedding_args& a, cudaStream_t st) {
    const int64_t units = ceil_div(a.cols, 16 / (int)sizeof(T));
    const dim3 grid((unsigned)ceil_div(a.tokens, kThreads / GL * TOKENS), (unsigned)ceil_div(units, GL * U));
    return launch(x, embedding_kernel<T, GL, U, TOKENS, WHOLE>, grid, kThreads, 0, st, a, x.err);
}

// Threads a token, units a thread and tokens at a time.  Few tokens take a unit
// a thread (64 of 1024 bfloat16 values: 1.4 us, and 1.65 by four at a time), so
// that more SMs take part.  Others keep several loads of a thread on their way:
// 16384 tokens of 1024 values take 10.3 us, one at a time 17.5; beyond 128 units
// those of one token (512 of 4096 values 2.3 us, four tokens at a time 2.6; 2048
// 4.7 and 5.0; 16384 of 32000 rows, as words fall, 29.5 and 29.2, and any row,
// where it loses, 39.2 and 37.6).
template <class T, bool WHOLE>
cudaError_t lookup_typed(const OpContext& x, const heddle_embedding_args& a, cudaStream_t st) {
    const int64_t units = ceil_div(a.cols, 16 / (int)sizeof(T));
    if (a.tokens * units < (int64_t)x.num_sms * 1024)
        return units <= 16   ? lookup<T, 16, 1, 1, WHOLE>(x, a, st)
               : units <= 32 ? lookup<T, 32, 1, 1, WHOLE>(x, a, st)
                             : lookup<T, 128, 1, 1, WHOLE>(x, a, st);
    if (units <= 16) return lookup<T, 16, 1, 4, WHOLE>(x, a, st);
    if (units <= 32) return lookup<T, 32, 1, 4, WHOLE>(x, a, st);
    if (units <= 64) return lookup<T, 32, 2, 2, WHOLE>(x, a, st);
    if (units <= 128) return lookup<T, 128, 1, 4, WHOLE>(x, a, st);
    return lookup<T, 128, 4, 1, WHOLE>(x, a, st);
}

template <class T>
cudaError_t lookup_any(const OpContext& x, const heddle_embedding_args& a, cudaStream_t st) {
    constexpr int size = sizeof(T);
    const bool whole = a.cols % (16 / size) == 0 && rows_whole(a.table, a.ldt, a.table_rows, size) &&
                       rows_whole(a.y, a.ldy, a.tokens, size);
    return whole ? lookup_typed<T, true>(x, a, st) : lookup_typed<T, false>(x, a, st);
}

// Columns of a block of the sums: a unit a thread.
int64_t slabs_of(const heddle_embedding_args& a) {
    return ceil_div(a.cols, kThreads * (a.dtype == HEDDLE_FP32 ? 4 : 8));
}

// Entries a block of the sums takes: as many as leave 1024 blocks for the
// table's share of the tokens, so that few rows go over several runs.  (16384
// tokens of 4096 bfloat16 values, half of them of one row, into 32000 rows of
// 32 bits: 142 us, 2048 blocks 159, 512 137; 262144 tokens of 1024 values, any
// row: 217, 227 and 237.)  At least 8, and more from 6400 tokens on, whose
// joining grows with the runs (with the lookup, 12867 tokens of 256 float16
// values, 687 rows: 29 us by 16, 34 by 8; 4096 of 1023, 6251 rows: 52 and 50).
// More beyond 8192 runs, which bounds the parts that a row of up to four million
// tokens is joined from.
int64_t chunk_of(const heddle_embedding_args& a) {
    const int64_t slabs = slabs_of(a);
    const int64_t own = (int64_t)((double)a.tokens * ((double)a.table_rows / (double)a.vocab));
    int64_t c = kMostRun, least = kLeastRun;
    while (least < kMostRun && 100 * least * least <= own) least *= 2;
    while (c > least && ceil_div(own, c) * slabs < 1024) c /= 2;
    while (c < kMostRun && ceil_div(a.tokens, c) > 8192) c *= 2;
    return c;
}

struct Places {
    size_t list, crossing, partial, total;
};
Places places(const heddle_embedding_args& a) {
    Places p;
    p.list = 256;
    const size_t chunks = (size_t)ceil_div(a.tokens, chunk_of(a));
    p.crossing = p.list + 2 * align256(sizeof(Entry) * (size_t)a.tokens);
    p.partial = p.crossing + align256(sizeof(uint32_t) * chunks);
    p.total = p.partial + align256(sizeof(float) * 2 * chunks * a.cols);
    return p;
}

template <class T, class TO>
cudaError_t sums(const OpContext& x, const Sums& s, cudaStream_t st) {
    const int64_t chunks = ceil_div(s.a.tokens, s.chunk), slabs = slabs_of(s.a);
    const bool whole = s.a.cols % (16 / (int)sizeof(T)) == 0 && rows_whole(s.a.y, s.a.ldy, s.a.tokens, sizeof(T));
    auto* kernel = whole ? embedding_sums_kernel<T, TO, true> : embedding_sums_kernel<T, TO, false>;
    cudaError_t e =
        launch(x, kernel, dim3((unsigned)(s.fillers + chunks * slabs)), kThreads, 0, st, s, (unsigned)slabs);
    const int64_t parts = ceil_div(s.a.cols, kJoinCols), want = (chunks - 1) * parts, most = (int64_t)x.num_sms * 8;
    if (e == cudaSuccess && chunks > 1)
        e = launch(x, embedding_join_kernel<TO>, dim3((unsigned)(want < most ? want : most)), kJoinThreads, 0, st, s,
                   (unsigned)parts);
    return e;
}

// Up to so many are sorted by one CTA, others by a cluster of eight (the gradient
// of 256 bfloat16 values, 1000 rows: 512 tokens 12.9 us, by a cluster 14.3; 2048:
// 17.5 and 16.9).
constexpr int64_t kFewTokens = 512;
template <int CTAS>
cudaError_t sort(const OpContext& x, const Sort& s, cudaStream_t st) {
    static std::atomic<uint64_t> asked{0};
    const cudaError_t e = allow_shared(embedding_sort_kernel<CTAS>, kSortShared, x.device, asked);
    if (e != cudaSuccess) return e;
    return launch(x, embedding_sort_kernel<CTAS>, dim3(CTAS), kSortThreads, kSortShared, st, s);
}

template <class T, class TO>
cudaError_t backward(const OpContext& x, const heddle_embedding_grad_args& g, unsigned char* ws, cudaStream_t st) {
    const heddle_embedding_args& a = g.fwd;
    const Places at = places(a);
    Sort s{};
    s.a = a;
    int bits = 1;
    while (bits < 31 && (int64_t)1 << bits < a.table_rows) ++bits;
    s.passes = (bits + 8) / 9;
    s.bits = (bits + s.passes - 1) / s.passes;
    s.list[0] = reinterpret_cast<Entry*>(ws + at.list);
    s.list[1] = reinterpret_cast<Entry*>(ws + at.list + align256(sizeof(Entry) * (size_t)a.tokens));
    s.count = reinterpret_cast<int64_t*>(ws);
    s.err = x.err;
    cudaError_t e = a.tokens <= kFewTokens ? sort<1>(x, s, st) : sort<8>(x, s, st);
    if (e != cudaSuccess) return e;
    Sums m{};
    m.a = a;
    m.out = const_cast<void*>(a.table);
    m.list = s.list[s.passes & 1];
    m.count = s.count;
    m.crossing = reinterpret_cast<uint32_t*>(ws + at.crossing);
    m.partial = reinterpret_cast<float*>(ws + at.partial);
    m.chunk = (int32_t)chunk_of(a);
    m.accumulate = g.accumulate;
    m.out_whole = a.cols % (16 / (int)sizeof(T)) == 0 && rows_whole(a.table, a.ldt, a.table_rows, sizeof(TO));
    const int64_t most = (int64_t)x.num_sms * 8;
    m.fillers = g.accumulate ? 0 : (unsigned)(a.table_rows < most ? a.table_rows : most);
    return sums<T, TO>(x, m, st);
}

}  // namespace

cudaError_t launch_embedding(const OpContext& x, const heddle_embedding_args& a, cudaStream_t st) {
    switch (a.dtype) {
        case HEDDLE_BF16: return lookup_any<__nv_bfloat16>(x, a, st);
        case HEDDLE_FP16: return lookup_any<__half>(x, a, st);
        default: return lookup_any<float>(x, a, st);
    }
}

size_t embedding_grad_scratch(const OpContext&, const heddle_embedding_grad_args& g) { return places(g.fwd).total; }

cudaError_t launch_embedding_grad(const OpContext& x, const heddle_embedding_grad_args& g, unsigned char* ws,
                                  cudaStream_t st) {
    const bool wide = g.grad_dtype == HEDDLE_FP32;
    switch (g.fwd.dtype) {
        case HEDDLE_BF16:
            return wide ? backward<__nv_bfloat16, float>(x, g, ws, st)
                        : backward<__nv_bfloat16, __nv_bfloat16>(x, g, ws, st);
        case HEDDLE_FP16: return wide ? backward<__half, float>(x, g, ws, st) : backward<__half, __half>(x, g, ws, st);
        default: return backward<float, float>(x, g, ws, st);
    }
}

}  // namespace hd
