// heddle_rows.cuh -- a row of values dealt out over a group of threads.
#pragma once

#include "heddle_ops.cuh"

namespace hd {

// A row of `cols` values in the registers of G threads, U 16-byte units each.
// Rows of whole units: thread `lane` has units lane, lane + G, ..; where they
// do not lie at 16 bytes they are read and written value by value, with the
// same results.  Others (STRIDED): values lane, lane + G, .., so that
// neighbours are read together.  Which one a row takes goes by its size alone.
template <class T, int G, int U, bool STRIDED>
struct RowPart {
    static constexpr int V = 16 / sizeof(T), N = U * V;
    int lane, cols;

    __device__ __forceinline__ int at(int e) const {
        return STRIDED ? lane + G * e : (lane + G * (e / V)) * V + e % V;
    }
    __device__ __forceinline__ bool in(int e) const { return at(e) < cols; }

    // zeros past the row's end
    __device__ __forceinline__ void load(uint4 (&r)[U], const T* p, bool whole) const {
        T* t = reinterpret_cast<T*>(&r);
        if (!STRIDED && whole) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                r[u] = in(u * V) ? *reinterpret_cast<const uint4*>(p + at(u * V)) : make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = in(e) ? p[at(e)] : from_float<T>(0.0f);
        }
    }
    __device__ __forceinline__ void store(T* p, const uint4 (&r)[U], bool whole) const {
        const T* t = reinterpret_cast<const T*>(&r);
        if (!STRIDED && whole) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (in(u * V)) *reinterpret_cast<uint4*>(p + at(u * V)) = r[u];
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (in(e)) p[at(e)] = t[e];
        }
    }
    static __device__ __forceinline__ float get(const uint4 (&r)[U], int e) {
        return to_float(reinterpret_cast<const T*>(&r)[e]);
    }
    static __device__ __forceinline__ void set(uint4 (&r)[U], int e, float v) {
        reinterpret_cast<T*>(&r)[e] = from_float<T>(v);
    }
};

// Whether rows at p, ld elements apart, lie at 16 bytes (null: does not matter).
inline bool rows_whole(const void* p, int64_t ld, int64_t rows, int size) {
    return !p || ((uintptr_t)p % 16 == 0 && (rows <= 1 || ld * size % 16 == 0));
}

}  // namespace hd
