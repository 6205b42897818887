// Tiles of rows in LDS and their products on the matrix cores, for the windowed attention's kernels.
//
// All products are 32 x 32 blocks (v_mfma_f32_32x32x16_bf16, v_mfma_f32_32x32x2_f32).  A block's accumulators hold, in lane l, column
// l % 32 and rows 8 g + 4 (l / 32) + i (g, i < 4).  Scores are computed so that a lane holds 16 keys of one query (or 16 queries of one
// key), and the second product contracts over just these: any order of the contraction is right as long as both operands have it, so a
// lane's accumulators are, rounded, its second operand, and no value moves between lanes.
//   rows of a tile as they lie ("direct", the first operand of scores): lane l reads 16 bytes of row l % 32, piece 2 s + l / 32 in step s;
//   rows of a tile transposed (the first operand of the second product): element l % 32 of rows 8 g + 4 (l / 32) + i; bf16: a 64-bit
//   transposing LDS read gives a lane 4 rows of its column.
// A tile's row is C pieces of 16 bytes (a power of two); piece p of row r lies at p ^ swizzle(r), so that 16 rows' same piece, and four
// consecutive rows' same 64 bytes, fall on different banks.
#pragma once

#include <type_traits>

#include "sp_attn.h"

namespace sp {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
#define SP_LDS __attribute__((address_space(3)))

constexpr int pieces_of(int bytes) { return bytes <= 64 ? 4 : bytes <= 128 ? 8 : bytes <= 256 ? 16 : 32; }

template <int C>
__device__ __forceinline__ int swizzle(int row) {
    if constexpr (C >= 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    else if constexpr (C == 8) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    else return (row >> 2) & 3;
}

// A sum over rows adds, for rows that do not take part, 0 times their elements: NaN where these are infinities or NaN.  A workgroup whose
// sums are not finite therefore takes them again in parts: of the elements that are finite; and how often those that do take part are +infinity
// or NaN, and -infinity or NaN (1 for each), for infinity to be added with that sign where there are any; or are either.
enum Part { kFinite, kPlus, kMinus, kEither };

// NT: head width in 32s, rounded up.  What is beyond `dim` is zero in LDS and registers.
template <typename T, int NT>
struct Tile {
    static constexpr bool kBf16 = sizeof(T) == 2;
    static constexpr int kC = pieces_of(NT * 32 * (int)sizeof(T));  // pieces a row of LDS
    static constexpr int kRowBytes = kC * 16;
    static constexpr int kPer = 16 / (int)sizeof(T);                // elements a piece
    static constexpr int kSteps = NT * 32 / (2 * kPer);             // pairs of pieces in a head
    static constexpr int kTSteps = kBf16 ? 2 : 4;                   // steps of a contraction over 32 rows
    using Raw = Piece<T, kPer>;
    using Frag = typename std::conditional<kBf16, bf16x8, f32x4>::type;

    static __device__ __forceinline__ f32x16 mma(const Frag& a, const Frag& b, f32x16 acc) {
        if constexpr (kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], acc, 0, 0, 0);
            return acc;
        }
    }

    // A lane's place in a tile: `direct` for step 0 of rows l % 32, `turned[j]` for element l % 32 and the rows of its half
    struct Place {
        int direct, turned[kBf16 ? 2 : 1];
    };
    static __device__ __forceinline__ Place place() {
        const int l = threadIdx.x & 63, h = l >> 5;
        Place p;
        p.direct = (l & 31) * kRowBytes + ((h ^ swizzle<kC>(l & 31)) << 4);
        if constexpr (kBf16) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = 8 * j + 4 * h + ((l & 15) >> 2), piece = ((l & 16) >> 3) + ((l & 3) >> 1);
                p.turned[j] = row * kRowBytes + ((piece ^ swizzle<kC>(row)) << 4) + ((l & 1) << 3);
            }
        } else {
            p.turned[0] = 4 * h * kRowBytes + ((((l & 31) >> 2) ^ swizzle<kC>(4 * h)) << 4) + ((l & 3) << 2);
        }
        return p;
    }
    // step s of rows 32 blk + l % 32
    static __device__ __forceinline__ Frag direct(const char* tile, const Place& p, int blk, int s) {
        return __builtin_bit_cast(Frag, *reinterpret_cast<const uint4*>(tile + (p.direct ^ (2 * s << 4)) + blk * 32 * kRowBytes));
    }
    // step s of the contraction over rows 32 blk .., element 32 dt + l % 32
    static __device__ __forceinline__ Frag turned(const char* tile, const Place& p, int blk, int s, int dt) {
        if constexpr (kBf16) {
            const char* at = tile + (blk * 32 + 16 * s) * kRowBytes;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SP_LDS s16x4*)(at + (p.turned[0] ^ (dt << 6))));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SP_LDS s16x4*)(at + (p.turned[1] ^ (dt << 6))));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // swizzle(8 s + 4 h + i) without h's part, which `turned` holds
                const int row = 8 * s + i, x = (dt << 3) ^ swizzle<kC>(row);
                v[i] = *reinterpret_cast<const float*>(tile + (blk * 32 + row) * kRowBytes + (p.turned[0] ^ (x << 4)));
            }
            return v;
        }
    }
    // what `part` of a first operand's elements are (Part)
    static __device__ __forceinline__ Frag part_of(Frag v, int part, bool* bad) {
        using Bits = typename std::conditional<kBf16, uint16_t, uint32_t>::type;
        constexpr int kMantissa = kBf16 ? 7 : 23;
        constexpr Bits kInf = (Bits)(0xffu << kMantissa), kOne = (Bits)(0x7fu << kMantissa), kSign = (Bits)(0x100u << kMantissa);
        struct All { Bits e[kPer]; } b = __builtin_bit_cast(All, v);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const Bits size = b.e[i] & (Bits)~kSign;
            const bool other = size >= kInf, counts = size > kInf || part == kEither || (b.e[i] == kInf) == (part == kPlus);
            *bad |= other;
            b.e[i] = part == kFinite ? (other ? (Bits)0 : b.e[i]) : other && counts ? kOne : (Bits)0;
        }
        return __builtin_bit_cast(Frag, b);
    }
    // accumulators of 32 rows as the second operand of step s of a contraction over them
    static __device__ __forceinline__ Frag operand(const f32x16& v, int s) {
        Frag r;
#pragma unroll
        for (int i = 0; i < (kBf16 ? 8 : 4); ++i) {
            if constexpr (kBf16) r[i] = (__bf16)v[8 * s + i];
            else r[i] = v[4 * s + i];
        }
        return r;
    }
    // a lane's pieces of one row in global memory, as operands: piece 2 s + l / 32 in step s
    template <bool VEC>
    static __device__ __forceinline__ void load_row(Frag (&f)[kSteps], const T* row, int dim, bool there, bool negate) {
        const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = (2 * s + h) * kPer;
            Frag v = {};
            if constexpr (VEC) {
                if (there && at < dim) v = __builtin_bit_cast(Frag, *reinterpret_cast<const uint4*>(row + at));
            } else {
                Piece<T, kPer> e{};
                if (there)
                    for (int i = 0; i < kPer; ++i)
                        if (at + i < dim) e.e[i] = row[at + i];
                v = __builtin_bit_cast(Frag, e);
            }
            if (negate)
#pragma unroll
                for (int i = 0; i < kPer; ++i) v[i] = -v[i];
            f[s] = v;
        }
    }
};

constexpr uint32_t kOutside = 0x80000000u;  // behind every tile's bytes: the load writes zeros
// The last row of a tile's bytes must lie below kOutside, for which rows are at most this far apart
constexpr int64_t kMostRowBytes = 1 << 24;

// Memory as far as `bytes` behind `base` (scalars), for loads that check their offset against it
__device__ __forceinline__ u32x4 memory_of(const void* base, uint32_t bytes) {
    const uint64_t at = (uint64_t)base;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xffffu),
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}
// 16 bytes a lane from memory to LDS, past the registers; lane l writes at `lds` + 16 l (a scalar).  There after wait_tiles().
__device__ __forceinline__ void memory_to_lds(u32x4 memory, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(memory) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(SP_LDS const char*)p; }

// What a thread loads of a tile of ROWS rows: piece p = thread, thread + THREADS, ... of its ROWS * kC, which lies at byte 16 p of the
// tile.  THREADS: of the workgroup, or 64 for a wavefront with a tile of its own.
template <typename T, int NT, int ROWS, int THREADS>
struct TileLoads {
    using Tl = Tile<T, NT>;
    static constexpr int kLoads = (ROWS * Tl::kC + THREADS - 1) / THREADS;
    uint32_t off[kLoads];
    static __device__ __forceinline__ int at(int k) { return k * THREADS + (int)(threadIdx.x % THREADS); }
    static __device__ __forceinline__ int row(int k) { return at(k) / Tl::kC; }
    static __device__ __forceinline__ int piece(int k) { return (at(k) % Tl::kC) ^ swizzle<Tl::kC>(row(k)); }
    // row r of the tile lies `row_at(r)` bytes behind the tile's memory
    template <typename RowAt>
    __device__ __forceinline__ void place(int dim, RowAt row_at) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) off[k] = piece(k) * Tl::kPer < dim ? row_at(row(k)) + piece(k) * 16 : kOutside;
    }
    static __device__ __forceinline__ uint32_t lds_of(uint32_t tile, int k) {
        return tile + k * THREADS * 16 + __builtin_amdgcn_readfirstlane((threadIdx.x % THREADS) >> 6) * 1024;
    }
    static __device__ __forceinline__ bool mine(int k) { return ROWS * Tl::kC % THREADS == 0 || at(k) < ROWS * Tl::kC; }
    __device__ __forceinline__ void load(uint32_t tile, u32x4 memory) const {
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (mine(k)) memory_to_lds(memory, off[k], lds_of(tile, k));
    }
    // the first `split` rows from one place, the others from another, as if it began `back` bytes earlier
    __device__ __forceinline__ void load_two(uint32_t tile, u32x4 one, int split, u32x4 two, uint32_t back) const {
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (mine(k)) {
                if (row(k) < split) memory_to_lds(one, off[k], lds_of(tile, k));
                else memory_to_lds(two, off[k] - back, lds_of(tile, k));
            }
    }
};

// Rows that are no 16-byte pieces, element by element: row r of the tile from where at(r) says, zeros for nullptr.
template <typename T, int NT, int ROWS, int THREADS, typename At>
__device__ __forceinline__ void load_elements(char* tile, int dim, At at) {
    using Tl = Tile<T, NT>;
    using Ld = TileLoads<T, NT, ROWS, THREADS>;
#pragma unroll 1
    for (int k = 0; k < Ld::kLoads; ++k) {
        if (!Ld::mine(k)) continue;
        const int e0 = Ld::piece(k) * Tl::kPer;
        const T* from = e0 < dim ? at(Ld::row(k)) : nullptr;
        Piece<T, Tl::kPer> e{};
        if (from)
            for (int i = 0; i < Tl::kPer; ++i)
                if (e0 + i < dim) e.e[i] = from[e0 + i];
        *reinterpret_cast<uint4*>(tile + Ld::at(k) * 16) = __builtin_bit_cast(uint4, e);
    }
}
// All of a workgroup's loads into LDS are there, for every thread
__device__ __forceinline__ void wait_tiles() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
}
// Whether any thread of the workgroup says so: a scalar, so that nothing is kept for the other way
__device__ __forceinline__ bool any_of_workgroup(bool x) { return __builtin_amdgcn_readfirstlane(__syncthreads_or(x)) != 0; }
// A wavefront's loads into LDS of its own
__device__ __forceinline__ void wait_own_tiles() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// the two halves of a wavefront combined, in both
template <typename Op>
__device__ __forceinline__ float halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return Op::of(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Accumulators whose column is a row of the result: elements 32 d + 8 g + 4 (l / 32) + i, four at a time
template <typename T, int NT, bool VEC>
__device__ __forceinline__ void put_column(T* row, const f32x16 (&acc)[NT], int dim) {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int d = 0; d < NT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = d * 32 + 8 * g + 4 * h;
            if constexpr (VEC) {
                struct alignas(4 * sizeof(T)) Four { T e[4]; } v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v.e[i] = to_elem<T>(acc[d][4 * g + i]);
                if (at < dim) *reinterpret_cast<Four*>(row + at) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (at + i < dim) row[at + i] = to_elem<T>(acc[d][4 * g + i]);
            }
        }
}

// Whether a column of accumulators holds an infinity or NaN.  After they are stored, so that they need not be kept for it.
template <int NT, typename... More>
__device__ __forceinline__ bool other_than_finite(const f32x16 (&acc)[NT], const More&... more) {
    float check = 0.f;
    auto add = [&](const f32x16 (&a)[NT]) {
#pragma unroll
        for (int d = 0; d < NT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) check = fmaf(a[d][i], 0.f, check);
    };
    add(acc);
    (add(more), ...);
    return halves<Add>(check) != 0.f;
}
// `other` (an infinity, NaN) joins a row of the result where `counts` (Part) are not zero.  The thread itself has written these elements.
template <typename T, int NT>
__device__ __forceinline__ void join_column(T* row, const f32x16 (&counts)[NT], int dim, float other) {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int d = 0; d < NT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = d * 32 + 8 * (i / 4) + 4 * h + i % 4;
            if (at < dim && counts[d][i] != 0.f) row[at] = to_elem<T>(elem(row[at]) + other);
        }
}

// Workgroups go to the 8 XCDs by turns: neighbouring items, which read the same rows, to one XCD.
__device__ __forceinline__ uint32_t item_of_block(uint32_t block, uint32_t items) {
    const uint32_t each = items / 8, extra = items % 8, x = block % 8;
    return x * each + min(x, extra) + block / 8;
}

}  // namespace sp
