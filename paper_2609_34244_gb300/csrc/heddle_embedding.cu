// heddle_embedding.cu -- the embedding and the gradient of its table.
//
// Bound by memory: rows are copied, and the gradient's rows are written once
// each.  The gradient sorts (row, token) pairs, so that a row's terms lie
// together in the order of their tokens: one cluster of CTAs sorts while the
// others write zeros to the rows that have no token.  Then blocks add up runs
// of the sorted list, and the sums of rows that go over several blocks' parts
// are joined in order.

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

// GL threads a token's row, U units of 16 bytes a thread at a time.
template <class T, int GL, int U, bool STRIDED>
__global__ void __launch_bounds__(kThreads)
    embedding_kernel(const __grid_constant__ heddle_embedding_args a, bool whole, uint32_t* err) {
    allow_dependents();
    await_previous();
    using R = RowPart<T, U, STRIDED>;
    constexpr int kTokens = kThreads / GL, kCols = GL * R::N;
    const int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / GL, from = (int64_t)blockIdx.y * kCols;
    if (t >= a.tokens) return;
    bool past;
    const int64_t row = row_of(a, t, past);
    if (past && from == 0 && threadIdx.x % GL == 0) atomicOr(err, kErrOpToken);
    const int64_t left = a.cols - from;
    const R part{(int)(threadIdx.x % GL), GL, (int)(left < kCols ? left : kCols)};
    uint32_t v[R::kWords] = {};
    if (row >= 0) {
        part.load(v, static_cast<const T*>(a.table) + row * a.ldt + from, whole);
        if (a.scale != 1.0f) {
#pragma unroll
            for (int p = 0; p < R::N / 2; ++p) set_pair<T>(v, p, mul2(pair_of<T>(v, p), both(a.scale)));
        }
    }
    part.store(static_cast<T*>(a.y) + t * a.ldy + from, v, whole);
}

// -------------------------------------------------------------------- sorting

constexpr int kCluster = 8;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kDigits = 512;

struct Entry {
    uint32_t row, token;
};

struct Sort {
    heddle_embedding_args a;
    void* out;          // the gradient
    int64_t out_bytes;  // of an element
    int32_t passes, bits;
    int32_t fill;       // rows without tokens are written
    Entry* list[2];     // by turns; the last pass leaves its result in list[passes & 1]
    int64_t* count;     // entries of rows of the table
    uint32_t* err;
};

__device__ __forceinline__ uint32_t load_of_rank(const uint32_t* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(tc::cluster_at(tc::smem_u32(p), rank)) : "memory");
    return v;
}

// A stable sort by the row, `bits` bits a pass from the lowest.  Each warp of
// the cluster has a run of the list: it counts its digits, its places in the
// result follow from the counts of all warps before it, and it walks over its
// run again in order.
__device__ void sort_pass(const Sort& s, int pass, int64_t n, uint32_t (*counts)[kDigits], uint32_t* total,
                          uint32_t* scan) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = tc::cluster_rank();
    const Entry* from = s.list[pass & 1];
    Entry* to = s.list[(pass & 1) ^ 1];
    const int shift = pass * s.bits, digits = 1 << s.bits;
    const int64_t run = ceil_div(n, kCluster * kSortWarps) , first = (rank * kSortWarps + warp) * run;
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
    for (int64_t i = first + lane; i < end; i += 32) {
        Entry e;
        if (entry(i, e, true)) atomicAdd(&counts[warp][e.row >> shift & (digits - 1)], 1u);
    }
    __syncthreads();
    // before this warp among the CTA's warps, and the CTA's own count
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
        uint32_t sum = 0;
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t c = counts[w][d];
            counts[w][d] = sum;
            sum += c;
        }
        total[d] = sum;
    }
    tc::cluster_sync();
    // before this CTA: all of the smaller digits, and this digit's of the CTAs before
    uint32_t all = 0, before = 0;
    const int d = threadIdx.x;
    if (d < digits) {
#pragma unroll
        for (uint32_t r = 0; r < kCluster; ++r) {
            const uint32_t c = load_of_rank(total + d, r);
            before += r < rank ? c : 0;
            all += c;
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
        if (lane == 31 && rank == 0 && pass == 0) *s.count = v;
    }
    __syncthreads();
    if (d < digits) {
        const uint32_t base = scan[warp] + up - all + before;
        for (int w = 0; w < kSortWarps; ++w) counts[w][d] += base;
    }
    __syncthreads();
    for (int64_t i0 = first; i0 < end; i0 += 32) {
        Entry e{};
        const bool is = entry(i0 + lane, e, false);
        const uint32_t digit = is ? e.row >> shift & (digits - 1) : (uint32_t)kDigits;
        const uint32_t same = __match_any_sync(~0u, digit);
        const uint32_t ahead = __popc(same & ((1u << lane) - 1));
        if (is) {
            const uint32_t at = counts[warp][digit] + ahead;
            to[at] = e;
        }
        __syncwarp();
        if (is && ahead == 0) counts[warp][digit] += __popc(same);
        __syncwarp();
    }
    __threadfence();
    tc::cluster_sync();  // the next pass reads what all wrote, and its counts take these ones' place
}

// Zeros to the rows of the gradient without tokens: a CTA has a range of rows,
// `kMark` at a time, marks those that the tokens name, and writes the others.
constexpr int kMark = 1 << 16;
template <class TO>
__device__ void fill_rows(const Sort& s, int64_t part, int64_t parts, uint32_t* marks) {
    const int64_t rows = s.a.table_rows, each = ceil_div(rows, parts), r0 = part * each;
    const int64_t r1 = r0 + each < rows ? r0 + each : rows;
    TO* out = static_cast<TO*>(s.out);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int64_t from = r0; from < r1; from += kMark) {
        const int64_t to = from + kMark < r1 ? from + kMark : r1;
        __syncthreads();
        for (int i = threadIdx.x; i < ceil_div(to - from, 32); i += kSortThreads) marks[i] = 0;
        __syncthreads();
        for (int64_t t = threadIdx.x; t < s.a.tokens; t += kSortThreads) {
            bool past;
            const int64_t row = row_of(s.a, t, past);
            if (row >= from && row < to) atomicOr(&marks[(row - from) / 32], 1u << ((row - from) % 32));
        }
        __syncthreads();
        for (int64_t row = from + warp; row < to; row += kSortWarps) {
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
}

template <class TO>
__global__ void __launch_bounds__(kSortThreads) __cluster_dims__(kCluster, 1, 1)
    embedding_sort_kernel(const __grid_constant__ Sort s) {
    allow_dependents();
    await_previous();
    extern __shared__ uint32_t shared[];
    if (blockIdx.x < kCluster) {
        auto* counts = reinterpret_cast<uint32_t(*)[kDigits]>(shared);
        uint32_t *total = shared + kSortWarps * kDigits, *scan = total + kDigits;
        int64_t n = s.a.tokens;
        for (int pass = 0; pass < s.passes; ++pass) {
            sort_pass(s, pass, n, counts, total, scan);
            if (pass == 0) n = *s.count;
        }
    } else if (s.fill) {
        fill_rows<TO>(s, blockIdx.x - kCluster, gridDim.x - kCluster, shared);
    }
}
constexpr int kSortShared = (kSortWarps * kDigits + kDigits + 32) * 4;

// ----------------------------------------------------------------------- sums

struct Sums {
    heddle_embedding_args a;  // y: the gradient in
    void* out;
    const Entry* list;
    const int64_t* count;
    float* partial;  // [chunk][2][cols]
    int32_t chunk;   // entries a block
    int32_t accumulate;
};

template <class TO, class R>
__device__ __forceinline__ void add_out(const Sums& s, const R& part, int64_t row, int64_t from,
                                        const float (&sum)[R::N]) {
    TO* p = static_cast<TO*>(s.out) + row * s.a.ldt + from;
#pragma unroll
    for (int e = 0; e < R::N; ++e)
        if (part.in(e)) {
            float v = sum[e] * s.a.scale;
            if (s.accumulate) v += to_float(p[part.at(e)]);
            p[part.at(e)] = from_float<TO>(v);
        }
}

constexpr int kAhead = 8;  // rows fetched before any is added

// A run of the sorted list and a range of columns a block.  A row whose
// entries all lie in the run is written; the sums of one that began before it
// go to partial[.][0], of one that goes on behind it to partial[.][1].
template <class T, class TO, int U, bool STRIDED>
__global__ void __launch_bounds__(kThreads)
    embedding_sums_kernel(const __grid_constant__ Sums s, bool whole) {
    allow_dependents();
    await_previous();
    using R = RowPart<T, U, STRIDED>;
    constexpr int kCols = kThreads * R::N;
    const int64_t n = *s.count, first = (int64_t)blockIdx.x * s.chunk;
    if (first >= n) return;
    const int64_t end = first + s.chunk < n ? first + s.chunk : n, from = (int64_t)blockIdx.y * kCols;
    const int64_t left = s.a.cols - from;
    const R part{(int)threadIdx.x, kThreads, (int)(left < kCols ? left : kCols)};
    const T* dy = static_cast<const T*>(s.a.y) + from;
    const uint32_t before = first ? s.list[first - 1].row : ~0u, behind = end < n ? s.list[end].row : ~0u;
    float* partial = s.partial + ((int64_t)blockIdx.x * 2) * s.a.cols + from;
    float sum[R::N] = {};
    uint32_t row = s.list[first].row;
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
    for (int64_t i = first; i < end; i += kAhead) {
        uint32_t v[kAhead][R::kWords];
        uint32_t rows[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const Entry e = s.list[i + k < end ? i + k : end - 1];
            rows[k] = e.row;
            if (i + k < end) part.load(v[k], dy + (int64_t)e.token * s.a.ldy, whole);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= end) break;
            if (rows[k] != row) {
                finish(false);
                row = rows[k], began = false;
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
}

// Rows that go over several runs, by the block of the one that they begin in.
template <class TO>
__global__ void __launch_bounds__(kThreads) embedding_join_kernel(const __grid_constant__ Sums s) {
    allow_dependents();
    await_previous();
    const int64_t n = *s.count, end = ((int64_t)blockIdx.x + 1) * s.chunk, first = end - s.chunk;
    if (end >= n) return;
    const uint32_t row = s.list[end].row;
    if (s.list[end - 1].row != row || (first && s.list[first].row == row && s.list[first - 1].row == row)) return;
    const int64_t i = (int64_t)blockIdx.y * kThreads + threadIdx.x;
    if (i >= s.a.cols) return;
    // the runs that it goes on into: those that start with it
    int64_t last = blockIdx.x + 1, none = ceil_div(n, s.chunk);
    while (none - last > 1) {
        const int64_t mid = (last + none) / 2;
        if (s.list[mid * s.chunk].row == row)
            last = mid;
        else
            none = mid;
    }
    float sum = s.partial[((int64_t)blockIdx.x * 2 + 1) * s.a.cols + i];
#pragma unroll 8
    for (int64_t c = blockIdx.x + 1; c <= last; ++c) sum += s.partial[c * 2 * s.a.cols + i];
    TO* p = static_cast<TO*>(s.out) + row * s.a.ldt + i;
    float v = sum * s.a.scale;
    if (s.accumulate) v += to_float(*p);
    *p = from_float<TO>(v);
}

// -------------------------------------------------------------------- launches

int size_of(int32_t dtype) { return dtype == HEDDLE_FP32 ? 4 : 2; }

template <class T, int GL, int U, bool STRIDED>
cudaError_t lookup(const OpContext& x, const heddle_embedding_args& a, bool whole, cudaStream_t st) {
    constexpr int kCols = RowPart<T, U, STRIDED>::N * GL;
    const dim3 grid((unsigned)ceil_div(a.tokens, kThreads / GL), (unsigned)ceil_div(a.cols, kCols));
    return launch(x, embedding_kernel<T, GL, U, STRIDED>, grid, kThreads, 0, st, a, whole, x.err);
}

template <class T, bool STRIDED>
cudaError_t lookup_typed(const OpContext& x, const heddle_embedding_args& a, cudaStream_t st) {
    const int size = sizeof(T);
    const int64_t units = ceil_div(a.cols, 16 / size);
    const bool whole = rows_whole(a.table, a.ldt, a.table_rows, size) && rows_whole(a.y, a.ldy, a.tokens, size);
    if (units <= 16) return lookup<T, 16, 1, STRIDED>(x, a, whole, st);
    if (units <= 32) return lookup<T, 32, 1, STRIDED>(x, a, whole, st);
    if (units <= 128 || a.tokens * units < (int64_t)x.num_sms * 1024)
        return lookup<T, 128, 1, STRIDED>(x, a, whole, st);
    return lookup<T, 128, 4, STRIDED>(x, a, whole, st);
}

// Entries a block of the sums takes: few, and no more than 2048 blocks of them,
// which bounds the parts that a row can be joined from.
constexpr int64_t kMostChunks = 2048;
int64_t chunk_of(int64_t tokens) {
    int64_t c = 16;
    while (ceil_div(tokens, c) > kMostChunks) c *= 2;
    return c;
}

struct Places {
    size_t list, partial, total;
};
Places places(const heddle_embedding_args& a) {
    Places p;
    p.list = 256;
    p.partial = p.list + 2 * align256(sizeof(Entry) * (size_t)a.tokens);
    p.total = p.partial + align256(sizeof(float) * 2 * (size_t)ceil_div(a.tokens, chunk_of(a.tokens)) * a.cols);
    return p;
}

template <class T, class TO, bool STRIDED>
cudaError_t sums(const OpContext& x, const Sums& s, cudaStream_t st) {
    constexpr int kCols = RowPart<T, 1, STRIDED>::N * kThreads;
    const unsigned chunks = (unsigned)ceil_div(s.a.tokens, s.chunk);
    const bool whole = rows_whole(s.a.y, s.a.ldy, s.a.tokens, sizeof(T));
    cudaError_t e = launch(x, embedding_sums_kernel<T, TO, 1, STRIDED>,
                           dim3(chunks, (unsigned)ceil_div(s.a.cols, kCols)), kThreads, 0, st, s, whole);
    if (e == cudaSuccess && chunks > 1)
        e = launch(x, embedding_join_kernel<TO>, dim3(chunks - 1, (unsigned)ceil_div(s.a.cols, kThreads)), kThreads, 0,
                   st, s);
    return e;
}

template <class T, class TO>
cudaError_t backward(const OpContext& x, const heddle_embedding_grad_args& g, unsigned char* ws, cudaStream_t st) {
    const heddle_embedding_args& a = g.fwd;
    const Places at = places(a);
    Sort s{};
    s.a = a;
    s.out = const_cast<void*>(a.table);
    int bits = 1;
    while (bits < 31 && (int64_t)1 << bits < a.table_rows) ++bits;
    s.passes = (bits + 8) / 9;
    s.bits = (bits + s.passes - 1) / s.passes;
    s.fill = !g.accumulate;
    s.list[0] = reinterpret_cast<Entry*>(ws + at.list);
    s.list[1] = reinterpret_cast<Entry*>(ws + at.list + align256(sizeof(Entry) * (size_t)a.tokens));
    s.count = reinterpret_cast<int64_t*>(ws);
    s.err = x.err;
    auto* kernel = embedding_sort_kernel<TO>;
    static std::atomic<uint64_t> asked{0};
    cudaError_t e = allow_shared(kernel, kSortShared, x.device, asked);
    if (e != cudaSuccess) return e;
    const unsigned clusters = 1 + (s.fill ? (unsigned)(x.num_sms / kCluster) : 0);
    e = launch(x, kernel, dim3(clusters * kCluster), kSortThreads, kSortShared, st, s);
    if (e != cudaSuccess || a.tokens == 0) return e;
    Sums m{};
    m.a = a;
    m.out = s.out;
    m.list = s.list[s.passes & 1];
    m.count = s.count;
    m.partial = reinterpret_cast<float*>(ws + at.partial);
    m.chunk = (int32_t)chunk_of(a.tokens);
    m.accumulate = g.accumulate;
    return a.cols % (16 / (int)sizeof(T)) ? sums<T, TO, true>(x, m, st) : sums<T, TO, false>(x, m, st);
}

}  // namespace

cudaError_t launch_embedding(const OpContext& x, const heddle_embedding_args& a, cudaStream_t st) {
    const bool strided = a.cols % (16 / size_of(a.dtype)) != 0;
    switch (a.dtype) {
        case HEDDLE_BF16:
            return strided ? lookup_typed<__nv_bfloat16, true>(x, a, st) : lookup_typed<__nv_bfloat16, false>(x, a, st);
        case HEDDLE_FP16: return strided ? lookup_typed<__half, true>(x, a, st) : lookup_typed<__half, false>(x, a, st);
        default: return strided ? lookup_typed<float, true>(x, a, st) : lookup_typed<float, false>(x, a, st);
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
