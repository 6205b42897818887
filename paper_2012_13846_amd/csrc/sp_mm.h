// Products of matrices on the matrix cores with a last step of their own, for the feed-forward block and for rows in 8 bits.
//
// out[n][m] = sum over k of first(m, k) * second(n, k).  An operand is "direct" if its contraction runs along its rows in memory ([m][k]), and
// "turned" if it runs across them ([k][m]).  A workgroup makes BM x BN results (first x second): in steps of 128 bytes of a direct operand's rows
// it takes both operands' tiles from memory to LDS past the registers, ST tiles deep, and multiplies 32 x 32 blocks; turned bf16 tiles are read
// by the transposing LDS read, so no operand is ever copied transposed.  The first operand are the results' columns: a lane's accumulators are
// then four neighbouring columns of one row at a time.  Pieces of LDS rows are swizzled (sp_attn_tile.h) so that reads are free of bank conflicts.
// Few results are split along the contraction; the parts' sums are added in order by a second kernel, which takes the same last step.
// Operands that are no whole, aligned 16-byte pieces go through registers by unaligned loads, with zeros behind their ends.
#pragma once

#include <type_traits>

#include "sp_attn_tile.h"
#include "sp_q8.h"

namespace sp {

struct q8_t {  // an e4m3 code
    uint8_t code;
};
typedef int i32x8 __attribute__((ext_vector_type(8)));

enum Last { kStore, kPartial, kGate, kGateBack };

struct Mm {
    const void *first, *second;
    int64_t ld_first, ld_second;  // bytes a row in memory
    int m, n, k;                  // results' columns and rows, contraction (elements)
    int steps, per_split, splits; // steps of 128 bytes; of each part
    int tiles_m, tiles_n;
    // kStore: out [n][m] in rows of ld elements.  kGate: m is the hidden width; first has rows of gates, then as many of ups; out = act(g) * u,
    // and, if not NULL, kept [n][kKept * m] gets g and u.  kGateBack: results are the gradient of act(g) * u; kept is read, dgu [n][2 m] written.
    Last last;
    void* out;
    int64_t ld;
    void *kept, *dgu;
    int act;
    bool out_f32;                 // kStore: of 8-bit operands
    bool four;                    // results' rows may be written four columns at a time
    float* part;                  // kPartial: [splits][n][m]
    const uint8_t *first_scales, *second_scales;
    int scales;                   // bytes a row of them
};

// ---- the last step ---------------------------------------------------------------------------------------------
struct Four {
    float e[4];
};
template <typename T>
__device__ __forceinline__ void put_four(T* p, const Four& v, int left, bool four) {
    struct alignas(4 * sizeof(T)) Quad { T e[4]; } q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.e[i] = to_elem<T>(v.e[i]);
    if (four) *reinterpret_cast<Quad*>(p) = q;
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = q.e[i];
}
template <typename T>
__device__ __forceinline__ Four get_four(const T* p, int left, bool four) {
    struct alignas(4 * sizeof(T)) Quad { T e[4]; } q{};
    if (four) q = *reinterpret_cast<const Quad*>(p);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) q.e[i] = p[i];
    return Four{{elem(q.e[0]), elem(q.e[1]), elem(q.e[2]), elem(q.e[3])}};
}

// act(g) and its derivative
__device__ __forceinline__ float2 gate_of(float g, int act) {
    if (act == SP_GATE_SILU) {
        const float p = 1.f / (1.f + expf(-g));
        return float2{g * p, p * (1.f + g * (1.f - p))};
    }
    const float p = 0.5f * (1.f + erff(g * 0.70710678f));
    return float2{g * p, p + g * 0.39894228f * expf(-0.5f * g * g)};
}

// What the backward pass reads of a row, m values each: g | u | act(g) * u, in bf16 g and u cut off behind 16 bits and the next 8 bits of both in a
// fourth part.  Rounded to bf16 alone they would put as much error into dx and dW_in as all that is rounded after them (0.0030 of the norm against
// 0.0024, and 0.0017 for the one rounding that cannot be done without).
template <typename T>
constexpr int kKept = sizeof(T) == 2 ? 4 : 3;

template <typename T>
__device__ __forceinline__ void keep(const Mm& a, int64_t row, int col, const Four& g, const Four& u) {
    const int left = a.m - col;
    T* to = static_cast<T*>(a.kept) + row * kKept<T> * a.m + col;
    if constexpr (sizeof(T) == 4) {
        put_four(to, g, left, a.four);
        put_four(to + a.m, u, left, a.four);
    } else {
        uint16_t hg[4], hu[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = __float_as_uint(g.e[i]), y = __float_as_uint(u.e[i]);
            hg[i] = (uint16_t)(x >> 16), hu[i] = (uint16_t)(y >> 16), lo[i] = (uint16_t)((x >> 8 & 255u) | (y & 0xff00u));
        }
        auto put = [&](T* p, const uint16_t (&v)[4]) {
            if (a.four) *reinterpret_cast<uint2*>(p) = uint2{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16};
            else
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) p[i] = v[i];
        };
        put(to, hg), put(to + a.m, hu), put(to + 3 * (int64_t)a.m, lo);
    }
}
template <typename T>
__device__ __forceinline__ void kept_of(const Mm& a, int64_t row, int col, Four& g, Four& u) {
    const int left = a.m - col;
    const T* from = static_cast<const T*>(a.kept) + row * kKept<T> * a.m + col;
    if constexpr (sizeof(T) == 4) {
        g = get_four(from, left, a.four), u = get_four(from + a.m, left, a.four);
    } else {
        auto get = [&](const T* p, uint32_t (&v)[4]) {
            if (a.four) {
                const uint2 w = *reinterpret_cast<const uint2*>(p);
                v[0] = w.x & 0xffffu, v[1] = w.x >> 16, v[2] = w.y & 0xffffu, v[3] = w.y >> 16;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = i < left ? p[i] : 0u;
            }
        };
        uint32_t hg[4], hu[4], lo[4];
        get(from, hg), get(from + a.m, hu), get(from + 3 * (int64_t)a.m, lo);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            g.e[i] = __uint_as_float(hg[i] << 16 | (lo[i] & 255u) << 8);
            u.e[i] = __uint_as_float(hu[i] << 16 | (lo[i] & 0xff00u));
        }
    }
}

template <typename T>
__device__ __forceinline__ void put_gate(const Mm& a, int64_t row, int col, const Four& g, const Four& u) {
    Four h;
#pragma unroll
    for (int i = 0; i < 4; ++i) h.e[i] = gate_of(g.e[i], a.act).x * u.e[i];
    put_four(static_cast<T*>(a.out) + row * a.ld + col, h, a.m - col, a.four);
    if (a.kept) keep<T>(a, row, col, g, u);
}
template <typename T>
__device__ __forceinline__ void put_gate_back(const Mm& a, int64_t row, int col, const Four& dh) {
    const int left = a.m - col;
    Four g, u, dg, du;
    kept_of<T>(a, row, col, g, u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = gate_of(g.e[i], a.act);
        dg.e[i] = dh.e[i] * u.e[i] * p.y;
        du.e[i] = dh.e[i] * p.x;
    }
    T* dgu = static_cast<T*>(a.dgu) + row * 2 * a.m + col;
    put_four(dgu, dg, left, a.four);
    put_four(dgu + a.m, du, left, a.four);
}
template <typename T>
__device__ __forceinline__ void put_out(const Mm& a, int64_t row, int col, const Four& v) {
    const int left = a.m - col;
    if constexpr (sizeof(T) == 1) {
        if (a.out_f32) put_four(static_cast<float*>(a.out) + row * a.ld + col, v, left, a.four);
        else put_four(static_cast<bf16_t*>(a.out) + row * a.ld + col, v, left, a.four);
    } else {
        put_four(static_cast<T*>(a.out) + row * a.ld + col, v, left, a.four);
    }
}

// Codes 8 e .. 8 e + 7 of a lane's 32, times their scale (the word's lowest byte)
__device__ __forceinline__ bf16x8 q8_values(const i32x8& codes, int e, int scale) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const uint32_t code = (uint32_t)scale & 255u;
    const float times = __uint_as_float(code == 0 ? 0x00400000u : code << 23);
    bf16x8 r;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * e + w], times, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * e + w], times, true);
        r[4 * w] = lo[0], r[4 * w + 1] = lo[1], r[4 * w + 2] = hi[0], r[4 * w + 3] = hi[1];
    }
    return r;
}

// ---- tiles -----------------------------------------------------------------------------------------------------
constexpr int kStepBytes = 128;

template <typename T>
struct Kind {
    static constexpr int kPer = 16 / (int)sizeof(T);           // elements a piece
    static constexpr int kElems = kStepBytes / (int)sizeof(T);  // elements of the contraction a step
    static constexpr int kSub = sizeof(T) == 1 ? 2 : 4;        // products of a block a step
    using Frag = std::conditional_t<sizeof(T) == 1, i32x8, std::conditional_t<sizeof(T) == 2, bf16x8, f32x4>>;
};

// One operand's tile: ROWS results of kElems elements each.
template <typename T, int ROWS, bool TURNED, int THREADS>
struct Side {
    using K = Kind<T>;
    static constexpr int kBytes = ROWS * kStepBytes;
    static constexpr int kC = TURNED ? ROWS / K::kPer : kStepBytes / 16;  // pieces of an LDS row
    static constexpr int kRowBytes = kC * 16;
    static constexpr int kLoads = kBytes / 16 / THREADS;
    static_assert(kBytes / 16 % THREADS == 0, "every thread loads equally many pieces");
    static __device__ __forceinline__ int at(int j) { return j * THREADS + (int)threadIdx.x; }
    static __device__ __forceinline__ int row(int j) { return at(j) / kC; }  // of LDS: a result, or an element of the contraction if turned
    static __device__ __forceinline__ int piece(int j) { return (at(j) % kC) ^ swizzle<kC>(row(j)); }

    // A lane's place in fragments: of step 0 and block 0
    int place[TURNED && sizeof(T) == 2 ? 2 : 1];
    __device__ __forceinline__ void aim() {
        const int l = threadIdx.x & 63, h = l >> 5;
        if constexpr (!TURNED) {
            place[0] = (l & 31) * kRowBytes + ((h ^ swizzle<kC>(l & 31)) << 4);
        } else if constexpr (sizeof(T) == 2) {
            // 4 elements of the contraction by a transposing read: the lane's half has elements 8 h .. 8 h + 7 of each 16, as in a direct tile
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 8 * h + 4 * j + ((l & 15) >> 2), p = ((l & 16) >> 3) + ((l & 3) >> 1);
                place[j] = r * kRowBytes + ((p ^ swizzle<kC>(r)) << 4) + ((l & 1) << 3);
            }
        } else {
            place[0] = 4 * h * kRowBytes + ((((l & 31) >> 2) ^ swizzle<kC>(4 * h)) << 4) + ((l & 3) << 2);
        }
    }
    // results 32 blk .., step s
    __device__ __forceinline__ typename K::Frag frag(const char* tile, int blk, int s) const {
        if constexpr (sizeof(T) == 1) {
            const uint4 lo = *reinterpret_cast<const uint4*>(tile + (place[0] ^ (4 * s << 4)) + blk * 32 * kRowBytes);
            const uint4 hi = *reinterpret_cast<const uint4*>(tile + (place[0] ^ ((4 * s + 2) << 4)) + blk * 32 * kRowBytes);
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        } else if constexpr (!TURNED) {
            return __builtin_bit_cast(typename K::Frag, *reinterpret_cast<const uint4*>(tile + (place[0] ^ (2 * s << 4)) + blk * 32 * kRowBytes));
        } else if constexpr (sizeof(T) == 2) {
            const char* from = tile + 16 * s * kRowBytes;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SP_LDS s16x4*)(from + (place[0] ^ (blk << 6))));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SP_LDS s16x4*)(from + (place[1] ^ (blk << 6))));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 8 * s + i, x = (blk << 3) ^ swizzle<kC>(r);  // without the half's part of the swizzle, which `place` has
                v[i] = *reinterpret_cast<const float*>(tile + r * kRowBytes + (place[0] ^ (x << 4)));
            }
            return v;
        }
    }
};

// The tile of an operand in memory: results from `first` on (of `count`), contraction from `k0` on (of `k`).  Rows of a direct gate tile: the first
// half of each wavefront's are gates, the second half ups, `ups` rows behind.
struct Place {
    const char* p;
    int64_t ld;
    int first, count, k;
};

// By checked loads, past the registers
template <typename T, int ROWS, bool TURNED, int THREADS>
struct Direct {
    using S = Side<T, ROWS, TURNED, THREADS>;
    uint32_t off[S::kLoads];
    __device__ __forceinline__ void aim(const Place& o, bool gate) {
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            const int r = S::row(j);
            if constexpr (TURNED) {
                const int col = S::piece(j) * S::K::kPer;
                off[j] = o.first + col < o.count ? (uint32_t)(r * o.ld + S::piece(j) * 16) : kOutside;
            } else {
                const int half = THREADS / 8, q = gate ? r % half + (j >> 1) * half : r;
                off[j] = o.first + q < o.count ? (uint32_t)(q * o.ld + S::piece(j) * 16) : kOutside;
            }
        }
    }
    // step: of the whole contraction; ups: of a gate tile, bytes from gates to ups
    __device__ __forceinline__ void load(const Place& o, int step, bool gate, int64_t ups, uint32_t lds) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t to = lds + wave * 1024;
        if constexpr (TURNED) {
            const int64_t k0 = (int64_t)step * S::K::kElems, bytes = (o.k - k0) * o.ld;
            const u32x4 mem = memory_of(o.p + k0 * o.ld + (int64_t)o.first * sizeof(T), (uint32_t)min(bytes, (int64_t)0x7fffffff));
#pragma unroll
            for (int j = 0; j < S::kLoads; ++j) memory_to_lds(mem, off[j], to + j * THREADS * 16);
        } else {
            const char* at = o.p + (int64_t)o.first * o.ld + (int64_t)step * kStepBytes;
            const u32x4 mem = memory_of(at, 0x7fffffffu), up = gate ? memory_of(at + ups, 0x7fffffffu) : mem;
            const int left = (int)min((int64_t)kStepBytes, (int64_t)o.k * (int)sizeof(T) - (int64_t)step * kStepBytes);
#pragma unroll
            for (int j = 0; j < S::kLoads; ++j) {
                const uint32_t from = left == kStepBytes || S::piece(j) * 16 < left ? off[j] : kOutside;
                memory_to_lds(j & 1 ? up : mem, from, to + j * THREADS * 16);
            }
        }
    }
};

// Through registers, element by element where a row ends
template <typename T, int ROWS, bool TURNED, int THREADS>
struct Through {
    using S = Side<T, ROWS, TURNED, THREADS>;
    uint4 held[S::kLoads];
    __device__ __forceinline__ void load(const Place& o, int step, bool gate, int64_t ups) {
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            const int r = S::row(j), e = S::piece(j) * S::K::kPer;
            const int64_t k0 = (int64_t)step * S::K::kElems;
            const char* from;
            int64_t left;
            if constexpr (TURNED) {
                from = o.p + (k0 + r) * o.ld + (int64_t)(o.first + e) * sizeof(T);
                left = k0 + r < o.k ? o.count - o.first - e : 0;
            } else {
                const int half = THREADS / 8, q = gate ? r % half + (j >> 1) * half : r;
                from = o.p + (int64_t)(o.first + q) * o.ld + (k0 + e) * sizeof(T) + (gate && (j & 1) ? ups : 0);
                left = o.first + q < o.count ? o.k - k0 - e : 0;
            }
            Piece<T, S::K::kPer> v{};
            if (left >= S::K::kPer) __builtin_memcpy(&v, from, 16);
            else
#pragma unroll
                for (int i = 0; i < S::K::kPer; ++i)
                    if (i < left) v.e[i] = reinterpret_cast<const T*>(from)[i];
            held[j] = __builtin_bit_cast(uint4, v);
        }
    }
    __device__ __forceinline__ void store(char* tile) const {
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) *reinterpret_cast<uint4*>(tile + S::at(j) * 16) = held[j];
    }
};

// four bytes a lane from memory to LDS, past the registers; lane l writes at `lds` + 4 l
__device__ __forceinline__ void word_to_lds(u32x4 memory, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(memory) : "memory");
}

template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// BM x BN results a workgroup, WM x WN wavefronts, ST tiles in LDS.
template <int BM_, int BN_, int WM_, int WN_, int ST_>
struct Shape2 {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, ST = ST_, kThreads = WM_ * WN_ * 64;
};
using Large = Shape2<256, 256, 2, 4, 2>;
using Middle = Shape2<128, 128, 2, 2, 2>;
using Narrow = Shape2<64, 128, 1, 4, 3>;
using Few = Shape2<128, 32, 4, 1, 4>;

// Tiles in LDS: two workgroups of Few a CU
template <typename T, typename Sh>
constexpr int depth_of() {
    return sizeof(T) == 1 && Sh::ST == 4 ? 3 : Sh::ST;
}

// EXACT (8-bit operands): codes become bf16, which holds them and their scales exactly, for the bf16 products.  The 8-bit products themselves take
// eight neighbouring elements at a time and cut their products off at 2^-13 of the largest's power of two (found by cancelling that one); of
// random rows 1.5e-5 of the result, whatever their length, against 1e-8: far below a bf16 result's rounding (1.7e-3), but not an fp32 one's.
template <typename T, typename Sh, bool TA, bool TB, bool VEC, bool EXACT>
__global__ __launch_bounds__(Sh::kThreads) void mm_kernel(Mm a) {
    using K = Kind<T>;
    constexpr int kThreads = Sh::kThreads, MT = Sh::BM / Sh::WM / 32, NT = Sh::BN / Sh::WN / 32;
    constexpr int kScaleLoads = sizeof(T) == 1 ? (Sh::BM + Sh::BN + kThreads - 1) / kThreads : 0;
    constexpr int kScaleBytes = kScaleLoads * kThreads * 4;
    constexpr int kStage = (Sh::BM + Sh::BN) * kStepBytes + kScaleBytes;
    constexpr int ST = VEC ? depth_of<T, Sh>() : 2;
    using A = Side<T, Sh::BM, TA, kThreads>;
    using B = Side<T, Sh::BN, TB, kThreads>;
    __shared__ char room[ST * kStage] __attribute__((aligned(16)));  // [ST][tile of the first operand, of the second, their scales]
    const bool gate = a.last == kGate;
    // neighbouring workgroups of an XCD: up to eight tiles of rows, then the next tile of columns, so that its L2 serves both operands
    const uint32_t tiles = (uint32_t)a.tiles_m * a.tiles_n, item = item_of_block(blockIdx.x, tiles * a.splits);
    const uint32_t split = item / tiles, t = item - split * tiles;
    const uint32_t band = 8u * a.tiles_m, b = t / band, in = t - b * band, high = min(8u, a.tiles_n - 8u * b);
    const int tm = (int)(in / high), tn = (int)(8u * b + in % high);
    const int begin = (int)split * a.per_split, count = min(a.steps - begin, a.per_split);
    const int cols = gate ? Sh::BM / 2 : Sh::BM;  // results' columns of a tile
    const Place pa{static_cast<const char*>(a.first), a.ld_first, tm * cols, a.m, a.k};
    const Place pb{static_cast<const char*>(a.second), a.ld_second, tn * Sh::BN, a.n, a.k};
    const int64_t ups = (int64_t)a.m * a.ld_first;
    const int wave = threadIdx.x >> 6, wm = wave / Sh::WN, wn = wave % Sh::WN, l = threadIdx.x & 63;

    f32x16 acc[MT][NT] = {};
    A fa;
    B fb;
    fa.aim(), fb.aim();
    auto multiply = [&](const char* stage, int step) {
        const char *ta = stage, *tb = stage + A::kBytes;
        int sa[MT], sb[NT];
        if constexpr (sizeof(T) == 1) {
            // this step's scales: one byte of the four steps that a row's word has
            const int shift = 8 * (step & 3);
            const uint32_t* words = reinterpret_cast<const uint32_t*>(tb + B::kBytes);
#pragma unroll
            for (int i = 0; i < MT; ++i) sa[i] = (int)(words[(wm * MT + i) * 32 + (l & 31)] >> shift);
#pragma unroll
            for (int i = 0; i < NT; ++i) sb[i] = (int)(words[Sh::BM + (wn * NT + i) * 32 + (l & 31)] >> shift);
        }
#pragma unroll
        for (int s = 0; s < K::kSub; ++s) {
            typename K::Frag x[MT], y[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) x[i] = fa.frag(ta, wm * MT + i, s);
#pragma unroll
            for (int i = 0; i < NT; ++i) y[i] = fb.frag(tb, wn * NT + i, s);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if constexpr (EXACT) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q8_values(x[i], e, sa[i]), q8_values(y[j], e, sb[j]), acc[i][j], 0, 0, 0);
                    } else if constexpr (sizeof(T) == 1) {
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[i], y[j], acc[i][j], 0, 0, 0, sa[i], 0, sb[j]);
                    } else if constexpr (sizeof(T) == 2) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y[j], acc[i][j], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i][e], y[j][e], acc[i][j], 0, 0, 0);
                    }
                }
        }
    };

    if constexpr (VEC) {
        Direct<T, Sh::BM, TA, kThreads> la;
        Direct<T, Sh::BN, TB, kThreads> lb;
        la.aim(pa, gate), lb.aim(pb, false);
        constexpr int kLoads = A::kLoads + B::kLoads + kScaleLoads;  // of a wavefront a step
        const uint32_t lds = lds_address(room);
        auto load = [&](int step, int stage) {
            const uint32_t to = lds + stage * kStage;
            la.load(pa, step, gate, ups, to);
            lb.load(pb, step, false, 0, to + A::kBytes);
            if constexpr (sizeof(T) == 1) {
                // a word a row: four steps' scales.  Every wavefront loads equally often, so that waits can count (zeros behind the rows).
#pragma unroll
                for (int j = 0; j < kScaleLoads; ++j) {
                    const int base = __builtin_amdgcn_readfirstlane(j * kThreads + (int)(threadIdx.x & ~63u));
                    const Place& o = base < Sh::BM ? pa : pb;
                    const int q = (base < Sh::BM ? base : base - Sh::BM) + l, rows = base < Sh::BM ? Sh::BM : Sh::BN;
                    const uint8_t* from = (base < Sh::BM ? a.first_scales : a.second_scales) + (int64_t)o.first * a.scales + (step >> 2) * 4;
                    const uint32_t off = q < rows && o.first + q < o.count ? (uint32_t)(q * a.scales) : kOutside;
                    word_to_lds(memory_of(from, 0x7fffffffu), off, to + A::kBytes + B::kBytes + base * 4);
                }
            }
        };
#pragma unroll
        for (int s = 0; s < ST - 1; ++s)
            if (s < count) load(begin + s, s);
        int stage = 0, next = ST - 1;
#pragma unroll 1
        for (int k = 0; k < count; ++k) {
            // this step's tiles are there; the ones behind it may still be under way
            if (k + ST - 1 <= count) wait_loads<(ST - 2) * kLoads>();
            else wait_loads<0>();
            meet();
            if (k + ST - 1 < count) load(begin + k + ST - 1, next);
            multiply(room + stage * kStage, begin + k);
            stage = stage + 1 == ST ? 0 : stage + 1;
            next = next + 1 == ST ? 0 : next + 1;
        }
    } else {
        Through<T, Sh::BM, TA, kThreads> la;
        Through<T, Sh::BN, TB, kThreads> lb;
        if (count > 0) la.load(pa, begin, gate, ups), lb.load(pb, begin, false, 0);
#pragma unroll 1
        for (int k = 0; k < count; ++k) {
            char* stage = room + (k & 1) * kStage;
            la.store(stage), lb.store(stage + A::kBytes);
            wait_loads<0>();
            meet();
            if (k + 1 < count) la.load(pa, begin + k + 1, gate, ups), lb.load(pb, begin + k + 1, false, 0);
            multiply(stage, begin + k);
        }
    }

    const int h = l >> 5;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t row = (int64_t)pb.first + (wn * NT + j) * 32 + (l & 31);
        if (row >= a.n) continue;
        auto four = [&](int i, int g) { return Four{{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]}}; };
        if (gate) {
            if constexpr (sizeof(T) > 1 && MT > 1 && !TA && !TB)
#pragma unroll
                for (int i = 0; i < MT / 2; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int col = pa.first + (wm * MT / 2 + i) * 32 + 8 * g + 4 * h;
                        if (col < a.m) put_gate<T>(a, row, col, four(i, g), four(i + MT / 2, g));
                    }
            continue;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = pa.first + (wm * MT + i) * 32 + 8 * g + 4 * h;
                if (col >= a.m) continue;
                if (a.last == kPartial) put_four(a.part + ((int64_t)split * a.n + row) * a.m + col, four(i, g), a.m - col, a.m % 4 == 0);
                else if (a.last == kStore) put_out<T>(a, row, col, four(i, g));
                else if constexpr (sizeof(T) > 1 && TA && !TB) put_gate_back<T>(a, row, col, four(i, g));
            }
    }
}

// ---- the parts' sums, and the last step ---------------------------------------------------------------------------
// a.m: the results' columns (of a gate: the hidden width, parts have 2 m columns)
template <typename T>
__global__ __launch_bounds__(256) void mm_join_kernel(Mm a) {
    const int each = (a.m + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / each;
    if (row >= a.n) return;
    const int col = (int)(i - row * each) * 4, wide = a.last == kGate ? 2 * a.m : a.m;
    auto sum = [&](int at, int left) {
        Four s{};
        for (int p = 0; p < a.splits; ++p) {
            const Four v = get_four(a.part + ((int64_t)p * a.n + row) * wide + at, left, a.m % 4 == 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) s.e[e] += v.e[e];
        }
        return s;
    };
    const Four s = sum(col, a.m - col);
    if constexpr (sizeof(T) > 1) {
        if (a.last == kGate) return put_gate<T>(a, row, col, s, sum(a.m + col, a.m - col));
        if (a.last == kGateBack) return put_gate_back<T>(a, row, col, s);
    }
    put_out<T>(a, row, col, s);
}

// ---- which workgroups, how many parts --------------------------------------------------------------------------
enum ShapeName { kLarge, kMiddle, kNarrow, kFew };
struct Plan {
    ShapeName shape;
    int splits, per_split, tiles_m, tiles_n;
};
// rows: of the first operand (a gate: 2 m); k_bytes: of a row of the contraction; gate: the results are made from pairs of rows
Plan mm_plan(int64_t rows, int64_t n, int64_t k_bytes, int size, bool gate, bool pieces);
// Bytes of the parts' sums (0: none)
inline int64_t mm_work(int64_t rows, int64_t n, int64_t k_bytes, int size, bool gate, bool pieces) {
    const Plan p = mm_plan(rows, n, k_bytes, size, gate, pieces);
    return p.splits > 1 || (gate && p.shape == kFew) ? (int64_t)p.splits * rows * n * 4 : 0;
}

template <typename T, typename Sh, bool TA, bool TB, bool VEC, bool EXACT>
int mm_launch(const Mm& a, hipStream_t s) {
    const int64_t blocks = (int64_t)a.tiles_m * a.tiles_n * a.splits;
    if (blocks > 0x7fffffff) return fail(SP_ERR_UNSUPPORTED, "too many tiles");
    hipLaunchKernelGGL((mm_kernel<T, Sh, TA, TB, VEC, EXACT>), dim3((unsigned)blocks), dim3(Sh::kThreads), 0, s, a);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

// Fills in what is left of `a` (steps, tiles, parts) and enqueues the product.  pieces: both operands are whole, aligned 16-byte pieces; part:
// mm_work() bytes.
template <typename T, bool TA, bool TB>
int mm(Mm a, bool pieces, float* part, hipStream_t s) {
    const bool gate = a.last == kGate;
    const int64_t k_bytes = (int64_t)a.k * (int)sizeof(T);
    const Plan p = mm_plan(gate ? (int64_t)2 * a.m : a.m, a.n, k_bytes, sizeof(T), gate, pieces);
    a.steps = (int)((k_bytes + kStepBytes - 1) / kStepBytes);
    a.per_split = p.per_split, a.splits = p.splits, a.tiles_m = p.tiles_m, a.tiles_n = p.tiles_n;
    Mm last = a;
    const bool join = p.splits > 1 || (gate && p.shape == kFew);
    if (join) {
        a.last = kPartial, a.part = last.part = part;
        if (gate) a.m *= 2;
    }
    auto go = [&](auto vec, auto exact) -> int {
        constexpr bool V = decltype(vec)::value, X = decltype(exact)::value;
        switch (p.shape) {
            case kLarge:
                if constexpr (V) return mm_launch<T, Large, TA, TB, V, X>(a, s);
                break;
            case kMiddle: return mm_launch<T, Middle, TA, TB, V, X>(a, s);
            case kNarrow: return mm_launch<T, Narrow, TA, TB, V, X>(a, s);
            case kFew: return mm_launch<T, Few, TA, TB, V, X>(a, s);
        }
        return fail(SP_ERR_UNSUPPORTED, "no kernel for this product");
    };
    if constexpr (sizeof(T) == 1) {
        SP_TRY(a.out_f32 ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{}));
    } else {
        SP_TRY(pieces ? go(std::true_type{}, std::false_type{}) : go(std::false_type{}, std::false_type{}));
    }
    if (join) {
        const int64_t blocks = ((int64_t)((last.m + 3) / 4) * last.n + 255) / 256;
        if (blocks > 0x7fffffff) return fail(SP_ERR_UNSUPPORTED, "too many results");
        hipLaunchKernelGGL(mm_join_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, s, last);
        SP_HIP(hipGetLastError());
    }
    return SP_OK;
}

inline int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }

// the feed-forward block's products (sp_ffn_f32.hip, sp_ffn_bf16.hip)
struct Ffn {
    int64_t n;
    int c, m, act;
    const void *x, *w_in, *w_out, *dy;
    void *kept, *y, *dx, *dw_in, *dw_out;
    char* work;
};
template <typename T>
int ffn_fwd(const Ffn& f, hipStream_t s);
template <typename T>
int ffn_bwd(const Ffn& f, hipStream_t s);

}  // namespace sp
