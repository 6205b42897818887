// Rows of fp32 or bf16 elements as fp32 values, and sums over the lanes or the workgroup that share a row.
#pragma once

#include "sp_internal.h"

namespace sp {

typedef uint16_t bf16_t;

__device__ __forceinline__ float elem(float v) { return v; }
__device__ __forceinline__ float elem(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }

// fp32 -> storage, to nearest even; NaN stays NaN
template <typename T>
__device__ __forceinline__ T to_elem(float v);
template <>
__device__ __forceinline__ float to_elem<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t to_elem<bf16_t>(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }

// V consecutive elements as they lie in memory: a 16-byte piece, or one element
template <typename T, int V>
struct Piece {
    static_assert(V * sizeof(T) == 16 || V == 1, "a 16-byte piece or one element");
    T e[V];
};
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> load_piece(const T* p) {
    Piece<T, V> r;
    if constexpr (V == 1) r.e[0] = *p;
    else r = __builtin_bit_cast(Piece<T, V>, *reinterpret_cast<const uint4*>(p));
    return r;
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, V>& r) {
    if constexpr (V == 1) *p = r.e[0];
    else *reinterpret_cast<uint4*>(p) = __builtin_bit_cast(uint4, r);
}

struct Add {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
    static constexpr float none = 0.f;
};
struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
    static constexpr float none = -INFINITY;
};

// N <= 2 values reduced over LANES threads that share a row: neighbouring lanes of a wavefront, or a whole workgroup of LANES
// threads (then `room` has kReduceRoom<LANES> floats, used in halves by turns, so that one barrier a call is enough).  Every lane
// gets the results, in an order of operations that does not change.
template <int LANES>
constexpr int kReduceRoom = LANES > 64 ? 4 * LANES / 64 : 1;
template <int LANES, typename Op, int N>
__device__ __forceinline__ void reduce_lanes(float (&v)[N], float* room, int* turn) {
    static_assert(N <= 2, "room for two values a wavefront");
#pragma unroll
    for (int s = (LANES < 64 ? LANES : 64) / 2; s > 0; s >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = Op::of(v[i], __shfl_xor(v[i], s));
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        float* r = room + *turn * 2 * kWaves;
        *turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) r[i * kWaves + (threadIdx.x >> 6)] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = r[i * kWaves];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v[i] = Op::of(v[i], r[i * kWaves + w]);
        }
    }
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace sp
