// heddle_rows.cuh -- rows of values dealt out over groups of threads, and a
// ring of rows in shared memory that bulk copies fill ahead of their use.
#pragma once

#include <type_traits>

#include "heddle_ops.cuh"
#include "heddle_tc.cuh"

namespace hd {

// ------------------------------------------------------ two floats at a time

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\t"
        "mov.b64 {%0, %1}, a;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\t"
        "mov.b64 {%0, %1}, a;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

template <class T>
__device__ __forceinline__ float2 pair_of(const uint32_t* w, int p) {
    if constexpr (sizeof(T) == 4)
        return make_float2(__uint_as_float(w[2 * p]), __uint_as_float(w[2 * p + 1]));
    else
        return to_floats<T>(w[p]);
}
template <class T>
__device__ __forceinline__ void set_pair(uint32_t* w, int p, float2 v) {
    if constexpr (sizeof(T) == 4)
        w[2 * p] = __float_as_uint(v.x), w[2 * p + 1] = __float_as_uint(v.y);
    else
        w[p] = from_floats<T>(v.x, v.y);
}

// Values of 16 bits as they lie in their words, added to 32 bits and multiplied
// into them in one instruction each: nothing is taken out of a word first.
#define HEDDLE_PLUS(type)                                                                             \
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.f32." type " %0, l, %3;\n\tadd.f32." type \
        " %1, h, %4;\n\t}"                                                                            \
        : "=f"(r.x), "=f"(r.y)                                                                        \
        : "r"(w[p]), "f"(c.x), "f"(c.y))
#define HEDDLE_TIMES(type)                                                                                  \
    asm("{\n\t.reg .b16 l, h, m, n;\n\tmov.b32 {l, h}, %2;\n\tmov.b32 {m, n}, %3;\n\tfma.rn.f32." type      \
        " %0, l, m, 0f00000000;\n\tfma.rn.f32." type " %1, h, n, 0f00000000;\n\t}"                          \
        : "=f"(r.x), "=f"(r.y)                                                                              \
        : "r"(a[p]), "r"(b[p]))
template <class T>
__device__ __forceinline__ float2 plus(const uint32_t* w, int p, float2 c) {
    float2 r;
    if constexpr (sizeof(T) == 4)
        r = add2(pair_of<T>(w, p), c);
    else if constexpr (std::is_same<T, __half>::value)
        HEDDLE_PLUS("f16");
    else
        HEDDLE_PLUS("bf16");
    return r;
}
template <class T>
__device__ __forceinline__ float2 times(const uint32_t* a, const uint32_t* b, int p) {
    float2 r;
    if constexpr (sizeof(T) == 4)
        r = mul2(pair_of<T>(a, p), pair_of<T>(b, p));
    else if constexpr (std::is_same<T, __half>::value)
        HEDDLE_TIMES("f16");
    else
        HEDDLE_TIMES("bf16");
    return r;
}
#undef HEDDLE_PLUS
#undef HEDDLE_TIMES

// ---------------------------------------------------------------------- rows

// A row of `cols` values in the registers of `group` threads, U 16-byte units
// each.  Rows of whole units: thread `lane` has units lane, lane + group, ..;
// where they do not lie at 16 bytes they are read and written value by value,
// with the same results.  Others (STRIDED): values lane, lane + group, .., so
// that neighbours are read together.  Which one a row takes goes by its size
// alone.  Values past the row's end are zeros.
template <class T, int U, bool STRIDED>
struct RowPart {
    static constexpr int V = 16 / sizeof(T), N = U * V, kWords = 4 * U;
    int lane, group, cols;

    __device__ __forceinline__ int at(int e) const {
        return STRIDED ? lane + group * e : (lane + group * (e / V)) * V + e % V;
    }
    __device__ __forceinline__ bool in(int e) const { return at(e) < cols; }

    __device__ __forceinline__ void load(uint32_t (&r)[kWords], const T* p, bool whole) const {
        if (!STRIDED && whole) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (in(u * V)) v = *reinterpret_cast<const uint4*>(p + at(u * V));
                r[4 * u] = v.x, r[4 * u + 1] = v.y, r[4 * u + 2] = v.z, r[4 * u + 3] = v.w;
            }
        } else {
            T* t = reinterpret_cast<T*>(r);
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = in(e) ? p[at(e)] : from_float<T>(0.0f);
        }
    }
    __device__ __forceinline__ void store(T* p, const uint32_t (&r)[kWords], bool whole) const {
        if (!STRIDED && whole) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (in(u * V))
                    *reinterpret_cast<uint4*>(p + at(u * V)) =
                        make_uint4(r[4 * u], r[4 * u + 1], r[4 * u + 2], r[4 * u + 3]);
        } else {
            const T* t = reinterpret_cast<const T*>(r);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (in(e)) p[at(e)] = t[e];
        }
    }
};

// Whether rows at p, ld elements apart, lie at 16 bytes (null: does not matter).
inline bool rows_whole(const void* p, int64_t ld, int64_t rows, int size) {
    return !p || ((uintptr_t)p % 16 == 0 && (rows <= 1 || ld * size % 16 == 0));
}

// ---------------------------------------------------------------------- ring

// Rows of several arrays in `stages` slots of shared memory.  A copy takes the
// 16-byte units that hold a row, whatever its alignment; the row then starts
// at (address % 16) of its place.  One thread issues.  A wait that runs out
// ends all others; the values are then not valid, nothing more is issued, and
// the kernel says so at its end (leave).
constexpr int kRingStages = 8;
struct __align__(128) RingBars {  // the slots follow it: bulk copies start at 16 bytes
    uint64_t full[kRingStages];
    uint32_t gave_up;
};
static_assert(sizeof(RingBars) % 16 == 0, "slots at 16 bytes");
__host__ __device__ inline int row_place(int64_t row_bytes) { return (int)((row_bytes + 15) / 16 * 16 + 16); }

struct Ring {
    unsigned char* slots;
    RingBars* bars;
    int arrays, stages, place, row_bytes;  // of a slot: its arrays, an array's place, a row
    int first = 0, in = 0;                 // the slots of the row at hand and of the next one to fetch
    uint32_t phase = 0;                    // of the row at hand
    bool go = true;

    __device__ __forceinline__ Ring(unsigned char* slots_, RingBars* bars_, int arrays_, int stages_, int row_bytes_)
        : slots(slots_),
          bars(bars_),
          arrays(arrays_),
          stages(stages_),
          place(row_place(row_bytes_)),
          row_bytes(row_bytes_) {
        if (threadIdx.x == 0) {
            for (int s = 0; s < stages; ++s) tc::mbar_init(tc::smem_u32(&bars->full[s]), 1);
            bars->gave_up = 0;
            tc::mbar_fence_init();
        }
        __syncthreads();
    }
    // The next row into the next slot, from where it lies in each array (null:
    // not in this one).  Every thread calls it, one issues.
    __device__ __forceinline__ void fetch(const void* a, const void* b, const void* c) {
        if (threadIdx.x == 0 && go) {
            const uint32_t bar = tc::smem_u32(&bars->full[in]);
            const void* rows[3] = {a, b, c};
            uint32_t bytes[3], sum = 0;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const uintptr_t p = (uintptr_t)rows[i];
                bytes[i] = rows[i] ? (uint32_t)(((p + row_bytes + 15) & ~(uintptr_t)15) - (p & ~(uintptr_t)15)) : 0;
                sum += bytes[i];
            }
            tc::mbar_expect(bar, sum);
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (bytes[i])
                    tc::load_bytes(tc::smem_u32(slots + (in * arrays + i) * place),
                                   (const void*)((uintptr_t)rows[i] & ~(uintptr_t)15), bytes[i], bar);
        }
        in = in + 1 == stages ? 0 : in + 1;
    }
    // `ahead` (0, 1) of the row at hand: its slot, and its arrival
    __device__ __forceinline__ int slot(int ahead) const {
        return first + ahead < stages ? first + ahead : first + ahead - stages;
    }
    __device__ __forceinline__ void wait(int ahead) {
        const uint32_t p = first + ahead < stages ? phase : phase ^ 1;
        go = go && tc::mbar_wait(tc::smem_u32(&bars->full[slot(ahead)]), p, &bars->gave_up);
    }
    __device__ __forceinline__ void advance(int rows) {
        first += rows;
        if (first >= stages) first -= stages, phase ^= 1;
    }
    __device__ __forceinline__ void leave(uint32_t* err) const {
        __syncthreads();
        if (*(volatile uint32_t*)&bars->gave_up) {
            if (threadIdx.x == 0) atomicOr(err, kErrOpWait);
            tc::drain();
        }
    }
    // Where an array's row is: its address in memory modulo 16 bytes further on.
    __device__ __forceinline__ const unsigned char* row(int ahead, int array) const {
        return slots + (slot(ahead) * arrays + array) * place;
    }
};
__device__ __forceinline__ uint32_t low_of(const void* p) { return (uint32_t)(uintptr_t)p; }

// 16 bytes at p + skew, p at 16 bytes, skew below 16 and the same for a row; an
// element's size divides it.  `second`: whether the next 16 bytes are needed.
__device__ __forceinline__ uint4 load_skewed(const unsigned char* p, uint32_t skew, bool second = true) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    if (skew == 0) return a;
    const uint4 b = second ? *reinterpret_cast<const uint4*>(p + 16) : make_uint4(0, 0, 0, 0);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (skew & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (skew & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (skew & 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row that lies in shared memory, `skew` bytes into its place; values past the
// row's end are zeros.  WHOLE: no skew, and whole units alone.
template <bool WHOLE, class T, int U, bool STRIDED>
__device__ __forceinline__ void load_units(uint32_t (&r)[4 * U], const RowPart<T, U, STRIDED>& part,
                                           const unsigned char* place, uint32_t skew) {
    constexpr int V = 16 / sizeof(T);
    if constexpr (WHOLE || STRIDED) {
        part.load(r, reinterpret_cast<const T*>(place + (WHOLE ? 0 : skew)), WHOLE);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int left = part.cols - part.at(u * V);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (left > 0) v = load_skewed(place + part.at(u * V) * sizeof(T), skew);
            r[4 * u] = v.x, r[4 * u + 1] = v.y, r[4 * u + 2] = v.z, r[4 * u + 3] = v.w;
            if (left > 0 && left < V) {
                T* t = reinterpret_cast<T*>(r + 4 * u);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e >= left) t[e] = from_float<T>(0.0f);
            }
        }
    }
}
// A row to memory: at 16 bytes at once, else by way of shared memory (a place
// of its own at 16 bytes), whole units and the ends value by value; value by
// value where there is no place.  The block calls it together; between two
// calls it meets at a barrier.
template <bool WHOLE, class T, int U, bool STRIDED>
__device__ __forceinline__ void store_units(T* dst, const RowPart<T, U, STRIDED>& part, const uint32_t (&r)[4 * U],
                                            unsigned char* place) {
    constexpr int V = 16 / sizeof(T);
    if (WHOLE) {
        part.store(dst, r, true);
        return;
    }
    const uint32_t off = low_of(dst) & 15;
    const int cols = part.cols;
    if (!place || (off == 0 && cols % V == 0)) {
        part.store(dst, r, off == 0 && cols % V == 0);
        return;
    }
    // its last unit whole: the place has room for it
    if constexpr (STRIDED) {
        part.store(reinterpret_cast<T*>(place), r, false);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (part.in(u * V))
                *reinterpret_cast<uint4*>(place + part.at(u * V) * sizeof(T)) =
                    make_uint4(r[4 * u], r[4 * u + 1], r[4 * u + 2], r[4 * u + 3]);
    }
    __syncthreads();
    const int skip = off / sizeof(T), head = skip ? (V - skip < cols ? V - skip : cols) : 0;
    const T* src = reinterpret_cast<const T*>(place);
    const int units = (cols - head) / V, tail = head + units * V;
    if (part.lane < head) dst[part.lane] = src[part.lane];
    for (int u = part.lane; u < units; u += part.group)
        *reinterpret_cast<uint4*>(dst + head + u * V) = load_skewed(place + u * 16, head * sizeof(T));
    if (tail + part.lane < cols) dst[tail + part.lane] = src[tail + part.lane];
}

}  // namespace hd
