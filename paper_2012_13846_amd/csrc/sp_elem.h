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

// for what is not read again soon: leaves the chip's last cache to others
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T, int V>
__device__ __forceinline__ void store_piece_past(T* p, const Piece<T, V>& r) {
    if constexpr (V == 1) __builtin_nontemporal_store(r.e[0], p);
    else __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<u32x4*>(p));
}

struct Add {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
    static constexpr float none = 0.f;
};
struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
    static constexpr float none = -INFINITY;
};

// A value from another lane of the same 4, 8 or 16, without LDS.  All of them must be active.
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// v reduced over LANES (4 to 64) neighbouring lanes, in all of them
template <int LANES, typename Op>
__device__ __forceinline__ float lanes_reduce(float v) {
    v = Op::of(v, from_lane<0xB1>(v));                        // the neighbour (quad_perm 1 0 3 2)
    v = Op::of(v, from_lane<0x4E>(v));                        // the other pair (2 3 0 1)
    if constexpr (LANES >= 8) v = Op::of(v, from_lane<0x141>(v));   // the other half of 8 (mirrored)
    if constexpr (LANES >= 16) v = Op::of(v, from_lane<0x140>(v));  // of 16
    if constexpr (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = Op::of(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (LANES >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = Op::of(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}

// N <= 2 values reduced over LANES threads that share a row: neighbouring lanes of a wavefront, or a whole workgroup of LANES
// threads (then `room` has kReduceRoom<LANES> floats, used in halves by turns, so that one barrier a call is enough).  Every lane
// gets the results, in an order of operations that does not change.
template <int LANES>
constexpr int kReduceRoom = LANES > 64 ? 4 * LANES / 64 : 1;
template <int LANES, typename Op, int N>
__device__ __forceinline__ void reduce_lanes(float (&v)[N], float* room, int* turn) {
    static_assert(N <= 2, "room for two values a wavefront");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_reduce<(LANES < 64 ? LANES : 64), Op>(v[i]);
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
