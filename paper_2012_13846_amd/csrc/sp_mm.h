// Products of matrices on the matrix cores with a last step of their own, for the feed-forward block and for rows in 8 bits.
//
// out[n][m] = sum over k of first(m, k) * second(n, k).  An operand is "direct" if its contraction runs along its rows in memory ([m][k]), and
// "turned" if it runs across them ([k][m]).  A workgroup makes BM x BN results (first x second): in steps of 128 bytes of a direct operand's rows
// it takes both operands' tiles from memory to LDS past the registers, ST tiles deep, and multiplies 16 x 16 blocks; turned bf16 tiles are read
// by the transposing LDS read, so no operand is ever copied transposed.  The first operand are the results' columns; at the end groups of 16 lanes
// swap halves of two neighbouring blocks, and a lane has eight neighbouring columns of one row: 16 bytes a store in bf16.  Pieces of LDS rows are
// swizzled so that reads are free of bank conflicts.
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
    float* part;                  // kPartial: [splits][n][m]
    const uint8_t *first_scales, *second_scales;
    int scales;                   // bytes a row of them
};

// ---- the last step ---------------------------------------------------------------------------------------------
// Eight neighbouring columns, of which `left` (1 or more) exist.
template <typename T>
struct EightOf {
    T e[8];
};
using Eight = EightOf<float>;
template <typename T>
__device__ __forceinline__ void put_eight(T* p, const EightOf<T>& v, int left) {
    if (left >= 8) __builtin_memcpy(p, &v, sizeof v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = v.e[i];
}
template <typename T>
__device__ __forceinline__ void put_rounded(T* p, const Eight& v, int left) {
    EightOf<T> q;
#pragma unroll
    for (int i = 0; i < 8; ++i) q.e[i] = to_elem<T>(v.e[i]);
    put_eight(p, q, left);
}
template <typename T>
__device__ __forceinline__ EightOf<T> get_piece(const T* p, int left) {
    EightOf<T> q{};
    if (left >= 8) __builtin_memcpy(&q, p, sizeof q);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) q.e[i] = p[i];
    return q;
}
template <typename T>
__device__ __forceinline__ Eight get_eight(const T* p, int left) {
    const EightOf<T> q = get_piece(p, left);
    Eight v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.e[i] = elem(q.e[i]);
    return v;
}

// act(g) and its derivative.  For bf16 by the exponential and reciprocal instructions (an ulp each; the exponential's argument is off by |g| 2^-24,
// as its result is then in relation): 2^-20 where the gate is not yet 2^-16 of g, against the 2^-8 of a rounding.  The normal distribution's tail
// beyond |g| is then exp(-g^2 / 2) t q(t) with t = 1 / (1 + 0.28 |g|) and q of degree 8, fitted to erfcx in fp64 with the least largest relative
// error, 1.8e-7: its exponential is the derivative's, too.
template <typename T, int ACT>
__device__ __forceinline__ float2 gate_of(float g) {
    constexpr bool kQuick = sizeof(T) == 2;
    if constexpr (ACT == SP_GATE_SILU) {
        const float p = kQuick ? __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * g)) : 1.f / (1.f + expf(-g));
        return float2{g * p, p * (1.f + g * (1.f - p))};
    } else if constexpr (kQuick) {
        const float e = __builtin_amdgcn_exp2f(-0.72134752f * g * g), t = __builtin_amdgcn_rcpf(fmaf(0.28f, fabsf(g), 1.f));
        constexpr float q[9] = {0.111703858f, 0.111699802f, 0.103084684f, 0.0836305994f, 0.072775931f, -0.00645151077f, 0.0924313212f, -0.093595375f, 0.0247206059f};
        float v = q[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) v = fmaf(v, t, q[i]);
        v *= e * t;
        const float p = g < 0.f ? v : 1.f - v;
        return float2{g * p, p + g * 0.39894228f * e};
    } else {
        const float p = 0.5f * erfcf(g * -0.70710678f);  // (of 1 + erf the tail would be what cancels)
        return float2{g * p, p + g * 0.39894228f * expf(-0.5f * g * g)};
    }
}
// f(std::integral_constant): of the gate, once for many values (a question at each is a third of the last step's instructions)
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    if (act == SP_GATE_SILU) f(std::integral_constant<int, SP_GATE_SILU>{});
    else f(std::integral_constant<int, SP_GATE_GELU>{});
}

// What the backward pass reads of a row, m values each: g | u | act(g) * u, in bf16 g and u cut off behind 16 bits and the next 8 bits of both in a
// fourth part.  Rounded to bf16 alone they would put as much error into dx and dW_in as all that is rounded after them (0.0030 of the norm against
// 0.0024, and 0.0017 for the one rounding that cannot be done without).
template <typename T>
constexpr int kKept = sizeof(T) == 2 ? 4 : 3;

template <typename T>
__device__ __forceinline__ void keep(const Mm& a, int64_t row, int col, const Eight& g, const Eight& u, int left) {
    T* to = static_cast<T*>(a.kept) + row * kKept<T> * a.m + col;
    if constexpr (sizeof(T) == 4) {
        put_eight(to, g, left);
        put_eight(to + a.m, u, left);
    } else {
        EightOf<T> hg, hu, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t x = __float_as_uint(g.e[i]), y = __float_as_uint(u.e[i]);
            hg.e[i] = (uint16_t)(x >> 16), hu.e[i] = (uint16_t)(y >> 16), lo.e[i] = (uint16_t)((x >> 8 & 255u) | (y & 0xff00u));
        }
        put_eight(to, hg, left), put_eight(to + a.m, hu, left), put_eight(to + 3 * (int64_t)a.m, lo, left);
    }
}
// The same as it lies in memory, in whole words: 16-bit elements by themselves take a register each
template <typename T>
struct KeptOf {
    static constexpr int kWords = 2 * (int)sizeof(T);
    uint32_t g[kWords], u[kWords], lo[kWords];  // lo: bf16 only
};
template <typename T>
__device__ __forceinline__ void get_words(const T* p, int left, uint32_t (&w)[2 * sizeof(T)]) {
    if (left >= 8) {
        __builtin_memcpy(w, p, sizeof w);
        return;
    }
#pragma unroll
    for (int i = 0; i < (int)(2 * sizeof(T)); ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[i]);
            else w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
        }
}
template <typename T>
__device__ __forceinline__ KeptOf<T> kept_at(const Mm& a, int64_t row, int col, int left) {
    const T* from = static_cast<const T*>(a.kept) + row * kKept<T> * a.m + col;
    KeptOf<T> k;
    get_words(from, left, k.g), get_words(from + a.m, left, k.u);
    if constexpr (sizeof(T) == 2) get_words(from + 3 * (int64_t)a.m, left, k.lo);
    return k;
}
template <typename T>
__device__ __forceinline__ float2 gate_and_up(const KeptOf<T>& k, int i) {
    if constexpr (sizeof(T) == 4) {
        return float2{__uint_as_float(k.g[i]), __uint_as_float(k.u[i])};
    } else {
        const uint32_t g = k.g[i / 2], u = k.u[i / 2], lo = k.lo[i / 2];
        return i & 1 ? float2{__uint_as_float((g & 0xffff0000u) | (lo >> 8 & 0xff00u)), __uint_as_float((u & 0xffff0000u) | (lo >> 16 & 0xff00u))}
                     : float2{__uint_as_float(g << 16 | (lo << 8 & 0xff00u)), __uint_as_float(u << 16 | (lo & 0xff00u))};
    }
}

template <typename T, int ACT>
__device__ __forceinline__ void put_gate(const Mm& a, int64_t row, int col, const Eight& g, const Eight& u, int left) {
    Eight h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h.e[i] = gate_of<T, ACT>(g.e[i]).x * u.e[i];
    put_rounded(static_cast<T*>(a.out) + row * a.ld + col, h, left);
    if (a.kept) keep<T>(a, row, col, g, u, left);
}
template <typename T, int ACT>
__device__ __forceinline__ void put_gate_back(const Mm& a, int64_t row, int col, const Eight& dh, const KeptOf<T>& kept, int left) {
    Eight dg, du;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 gu = gate_and_up(kept, i), p = gate_of<T, ACT>(gu.x);
        dg.e[i] = dh.e[i] * gu.y * p.y;
        du.e[i] = dh.e[i] * p.x;
    }
    T* dgu = static_cast<T*>(a.dgu) + row * 2 * a.m + col;
    put_rounded(dgu, dg, left);
    put_rounded(dgu + a.m, du, left);
}
template <typename T>
__device__ __forceinline__ void put_out(const Mm& a, int64_t row, int col, const Eight& v, int left) {
    if constexpr (sizeof(T) == 1) {
        if (a.out_f32) put_eight(static_cast<float*>(a.out) + row * a.ld + col, v, left);
        else put_rounded(static_cast<bf16_t*>(a.out) + row * a.ld + col, v, left);
    } else {
        put_rounded(static_cast<T*>(a.out) + row * a.ld + col, v, left);
    }
}

// 8-bit products as bf16.  A code times its scale is a bf16 value if the scale's code is 64 to 191 (3 to 246 would do, but of these exactly
// one of the two highest bits is set).  Smaller scales would lose codes' bits and larger ones make them infinite; there a step's sum of codes
// alone gets both scales' exponents, together, since one by itself may take the sum beyond fp32.
constexpr uint32_t kPlain = 0x80808080u;
__device__ __forceinline__ uint32_t q8_plain(uint32_t word) { return word ^ word << 1; }  // has all of kPlain's bits if a word's four scales are such
// Codes 8 e .. 8 e + 7 of a lane's 32, times `times`, a power of two or what a scale of 255 stands for
__device__ __forceinline__ bf16x8 q8_values(const i32x8& codes, int e, float times) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    bf16x8 r;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * e + w], times, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * e + w], times, true);
        r[4 * w] = lo[0], r[4 * w + 1] = lo[1], r[4 * w + 2] = hi[0], r[4 * w + 3] = hi[1];
    }
    return r;
}
__device__ __forceinline__ float q8_all(int scale) { return __uint_as_float(((uint32_t)scale & 255u) << 23); }  // a plain scale (a word's lowest byte)
__device__ __forceinline__ float q8_none(int scale) { return __uint_as_float((scale & 255) == (int)kQ8NaN ? 0x7f800000u : 0x3f800000u); }
__device__ __forceinline__ float q8_scaled(float sum, int first, int second) { return ldexpf(sum, (first & 255) + (second & 255) - 254); }

// ---- tiles -----------------------------------------------------------------------------------------------------
constexpr int kStepBytes = 128;

template <typename T>
struct Kind {
    static constexpr int kPer = 16 / (int)sizeof(T);            // elements a piece
    static constexpr int kElems = kStepBytes / (int)sizeof(T);  // elements of the contraction a step
    static constexpr int kSub = sizeof(T) == 1 ? 1 : 2;         // fragments of a block a step
    using Frag = std::conditional_t<sizeof(T) == 1, i32x8, std::conditional_t<sizeof(T) == 2, bf16x8, f32x4>>;
};

// One operand's tile: ROWS results of kElems elements each.  Lane l has row l % 16 of a block's fragment; of the contraction, 16 bytes a fragment
// (8 bits: 32, the whole step), those of group l / 16.
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
    static __device__ __forceinline__ int piece(int j) { return (at(j) % kC) ^ swizzled(row(j)); }
    // 64 banks are 16 pieces.  Direct: 16 lanes read the same piece of 16 rows, of which neighbours lie 32 banks apart.  Turned bf16: 32 lanes read 2
    // neighbouring pieces of rows 0 .. 3 and 8 .. 11; turned fp32: 64 lanes 4 pieces of rows 0, 4, 8 and 12.
    static __device__ __forceinline__ int swizzled(int r) {
        if constexpr (!TURNED) return r >> 1 & 7;
        else if constexpr (sizeof(T) == 2) return kC >= 16 ? (r & 3) << 1 | (r >> 3 & 1) << 3 : kC == 8 ? (r >> 1 & 1) << 1 | (r >> 3 & 1) << 2 : (r >> 3 & 1) << 1;
        else return kC >= 16 ? (r >> 2 & 3) << 2 : (r >> 2 & 1) << 2;
    }

    // A lane's place in the first fragment of a wavefront's pairs of blocks `from` ..
    int place;
    __device__ __forceinline__ void aim(int from) {
        const int l = threadIdx.x & 63, h = l >> 4, q = l >> 2 & 3, e = l & 3;
        if constexpr (!TURNED) {
            const int r = 32 * from + (l & 15);
            place = r * kRowBytes + ((h ^ swizzled(r)) << 4);
        } else if constexpr (sizeof(T) == 2) {
            // a transposing read: lanes 4 q + e of a group address columns 4 e .. of a block in row q, and get column 4 q + e of all four rows
            const int r = 8 * h + q;
            place = r * kRowBytes + (((4 * from + (e >> 1)) ^ swizzled(r)) << 4) + ((e & 1) << 3);
        } else {
            place = 4 * h * kRowBytes + (((8 * from + q) ^ swizzled(4 * h)) << 4) + (e << 2);
        }
    }
    // Bytes from a direct tile's block 0 to block i; `half`: rows from gates to ups, which blocks MT / 2 .. are (0: no gate)
    template <int MT>
    static __device__ __forceinline__ constexpr int block(int i, int half) {
        const int b = half && i >= MT / 2 ? i - MT / 2 : i;
        return ((half && i >= MT / 2 ? half : 0) + 16 * b) * kRowBytes;
    }
    // block i of the wavefront (a direct tile: `off` bytes behind its first), fragment s
    __device__ __forceinline__ typename K::Frag frag(const char* tile, int i, int off, int s) const {
        if constexpr (sizeof(T) == 1) {
            const uint4 lo = *reinterpret_cast<const uint4*>(tile + place + off);
            const uint4 hi = *reinterpret_cast<const uint4*>(tile + (place ^ 64) + off);
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        } else if constexpr (!TURNED) {
            return __builtin_bit_cast(typename K::Frag, *reinterpret_cast<const uint4*>(tile + (place ^ (s << 6)) + off));
        } else if constexpr (sizeof(T) == 2) {
            const char* from = tile + 32 * s * kRowBytes + (place ^ (i << 5));
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SP_LDS s16x4*)from);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SP_LDS s16x4*)(from + 4 * kRowBytes));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const char* from = tile + 16 * s * kRowBytes + (place ^ (i << 6));
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const float*>(from + e * kRowBytes);
            return v;
        }
    }
};

// The tile of an operand in memory: results from `first` on (of `count`), contraction from `k0` on (of `k`).  The second half of a direct gate
// tile are ups, as many rows as there are gates behind them.
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
                const int q = gate && j >= S::kLoads / 2 ? r - ROWS / 2 : r;
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
                memory_to_lds(j >= S::kLoads / 2 ? up : mem, from, to + j * THREADS * 16);
            }
        }
    }
};

// Through registers, by unaligned loads.  Steps but the last need no care: a direct operand's pieces lie within their rows, a turned one's may hold
// elements of the next row, behind its own, which reach only results that there are not; rows and columns that there are not have another's
// elements.  The last step is loaded with zeros behind the contraction's end, element by element where a row ends.
template <typename T, int ROWS, bool TURNED, int THREADS>
struct Through {
    using S = Side<T, ROWS, TURNED, THREADS>;
    uint4 held[S::kLoads];
    uint32_t off[S::kLoads];
    bool quick;
    __device__ __forceinline__ void aim(const Place& o, bool gate) {
        // (a turned piece of the last row but one, which may begin in the last column, ends within the last row)
        quick = !TURNED || o.ld >= (S::K::kPer - 1) * (int64_t)sizeof(T);
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            const int r = S::row(j), e = S::piece(j) * S::K::kPer;
            if constexpr (TURNED) {
                off[j] = (uint32_t)(r * o.ld + (o.first + e < o.count ? e : 0) * (int)sizeof(T));
            } else {
                const int q = gate && j >= S::kLoads / 2 ? r - ROWS / 2 : r;
                off[j] = (uint32_t)(min(q, o.count - 1 - o.first) * o.ld + e * (int)sizeof(T));
            }
        }
    }
    __device__ __forceinline__ void load(const Place& o, int step, bool gate, int64_t ups) {
        if (quick && (step + 1) * (int64_t)S::K::kElems < o.k) {
            const char* at = TURNED ? o.p + (int64_t)step * S::K::kElems * o.ld + (int64_t)o.first * sizeof(T) : o.p + (int64_t)o.first * o.ld + (int64_t)step * kStepBytes;
#pragma unroll
            for (int j = 0; j < S::kLoads; ++j) __builtin_memcpy(&held[j], at + (gate && j >= S::kLoads / 2 ? ups : 0) + off[j], 16);
        } else {
            load_last(o, step, gate, ups);
        }
    }
    __device__ __forceinline__ void load_last(const Place& o, int step, bool gate, int64_t ups) {
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
                const int q = gate && j >= S::kLoads / 2 ? r - ROWS / 2 : r;
                from = o.p + (int64_t)(o.first + q) * o.ld + (k0 + e) * sizeof(T) + (gate && j >= S::kLoads / 2 ? ups : 0);
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
// Middle where a workgroup has its CU to itself: twice the wavefronts, and all of the LDS for tiles further ahead.  bf16, 256 workgroups of 32 steps: 24.7
// against 20.4 us, 216 of 51 steps 49.8 against 36.6; 8 bits 50.2 against 47.6; fp32, whose steps are longer than a load's way, the same.  (Narrow, six
// tiles deep: the same, too.)
using MiddleDeep = Shape2<128, 128, 2, 4, 4>;
constexpr int64_t kCUs = 256;

template <typename T, typename Sh, bool VEC>
struct Room {  // LDS: [ST][tile of the first operand, of the second], [2][scales]
    static constexpr int kStage = (Sh::BM + Sh::BN) * kStepBytes, kWords = sizeof(T) == 1 ? Sh::BM + Sh::BN : 0;
    static constexpr int ST = VEC ? Sh::ST : 2, kBytes = ST * kStage + 2 * kWords * 4;
};

// The loop, bound by the matrix cores and the power they take.  bf16 and fp32 (kAhead): a step's two fragments are read while the ones before them are
// multiplied, an LDS read for every two products; one barrier a step, between them, behind which this step's tiles are free and the next one's are
// there.  Large has 8 wavefronts of 128 x 64 results: 2048 x 8192 of 8192 in bf16 takes 184 us alone (1500 TFLOP/s; 16 wavefronts of 64 x 64, which read
// a third more from LDS and nothing ahead, 214), 212 in the block, where the memory still writes what was kept.  8 bits: fragments are twice as long and
// only registers for one set are left; 16384 x 4096 x 6144 at 2500 TFLOP/s.  fp32: 134 TFLOP/s in 8192 x 1024 x 2048, of 152.
// Last steps: 8 bytes a result of the gate and 10 of its gradient are memory's, 8192 x 2048 x 8192: 493 us for 370 of products, 331 for 190
// (what is kept and read ahead leaves its last step six registers short: 28 bytes of scratch a lane).
// EXACT (8-bit operands): codes and their scales become bf16, exactly (q8_plain), for the bf16 products.  The 8-bit products themselves take
// eight neighbouring elements at a time and cut their products off at 2^-13 of the largest's power of two (found by cancelling that one); of
// random rows 1.5e-5 of the result, whatever their length, against 1e-8: far below a bf16 result's rounding (1.7e-3), but not an fp32 one's.
// 16384 x 4096 x 6144: 706 us, 1170 TFLOP/s (686 without a way for scales that bf16 does not take).
template <typename T, typename Sh, bool TA, bool TB, bool VEC, bool EXACT, Last LAST>
__device__ __forceinline__ void mm_body(const Mm& a, uint32_t block, char* room) {
    using K = Kind<T>;
    constexpr int kThreads = Sh::kThreads, MT = Sh::BM / Sh::WM / 16, NT = Sh::BN / Sh::WN / 16;
    static_assert(MT % 2 == 0 && NT % 2 == 0, "blocks come in pairs");
    constexpr bool gate = LAST == kGate;
    static_assert(!gate || (MT % 4 == 0 && !TA), "a wavefront has as many pairs of gates as of ups");
    constexpr int kStage = Room<T, Sh, VEC>::kStage, kWords = Room<T, Sh, VEC>::kWords, ST = Room<T, Sh, VEC>::ST;
    constexpr bool kAhead = VEC && sizeof(T) > 1;
    using A = Side<T, Sh::BM, TA, kThreads>;
    using B = Side<T, Sh::BN, TB, kThreads>;
    // Neighbouring workgroups of an XCD: up to kBand tiles of rows, then the next tile of columns, so that its L2 serves both operands.  Each band begins
    // 5/8 of the columns behind the last: XCDs that go through equal columns of their rows at a time write to, and read the first operand from, the same
    // memory channels where rows are a power of two apart (8192 x 16384 results of 2048 in bf16, bands of 8 that all begin at column 0: 456 us, so: 403).
    constexpr uint32_t kBand = 6;
    const uint32_t tiles = (uint32_t)a.tiles_m * a.tiles_n, item = item_of_block(block, tiles * a.splits);
    const uint32_t split = item / tiles, t = item - split * tiles;
    const uint32_t band = kBand * a.tiles_m, b = t / band, in = t - b * band, high = min(kBand, a.tiles_n - kBand * b);
    const uint32_t turned = in / high + b % 8 * 5 * a.tiles_m / 8;
    const int tm = (int)(turned % a.tiles_m), tn = (int)(kBand * b + in % high);
    const int begin = (int)split * a.per_split, count = min(a.steps - begin, a.per_split);
    constexpr int cols = gate ? Sh::BM / 2 : Sh::BM, half = gate ? Sh::BM / 2 : 0;  // results' columns of a tile; rows from gates to ups
    constexpr int MP = gate ? MT / 4 : MT / 2, NP = NT / 2;                          // pairs of blocks of a wavefront
    const Place pa{static_cast<const char*>(a.first), a.ld_first, tm * cols, a.m, a.k};
    const Place pb{static_cast<const char*>(a.second), a.ld_second, tn * Sh::BN, a.n, a.k};
    const int64_t ups = (int64_t)a.m * a.ld_first;
    const int wave = threadIdx.x >> 6, wm = wave / Sh::WN, wn = wave % Sh::WN, l = threadIdx.x & 63;

    f32x4 acc[MT][NT] = {};
    A fa;
    B fb;
    fa.aim(wm * MP), fb.aim(wn * NP);
    using Frag = typename K::Frag;
    // of an LDS read and products in turn
    auto alternate = [] {
        constexpr int kReads = (MT * (TA ? 2 : 1) + NT * (TB ? 2 : 1)) * (sizeof(T) == 4 && (TA || TB) ? 2 : 1);
        constexpr int kEach = MT * NT / kReads > 1 ? 2 : 1;
#pragma unroll
        for (int i = 0; i < kReads; ++i) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0), __builtin_amdgcn_sched_group_barrier(0x8, kEach, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, MT * NT * 4, 0);
    };
    auto take = [&](const char* stage, int s, Frag (&x)[MT], Frag (&y)[NT]) {
#pragma unroll
        for (int i = 0; i < NT; ++i) y[i] = fb.frag(stage + A::kBytes, i, B::template block<NT>(i, 0), s);
#pragma unroll
        for (int i = 0; i < MT; ++i) x[i] = fa.frag(stage, i, A::template block<MT>(i, half), s);
    };
    auto product_of = [&](const Frag (&x)[MT], const Frag (&y)[NT], auto from, auto to) {
#pragma unroll
        for (int i = decltype(from)::value; i < decltype(to)::value; ++i)
#pragma unroll
            for (int v = 0; v < NT; ++v) {
                const int j = i & 1 ? NT - 1 - v : v;  // (back and forth: 2% in a product of 2048 x 8192 x 8192)
                if constexpr (sizeof(T) == 2) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], y[j], acc[i][j], 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i][e], y[j][e], acc[i][j], 0, 0, 0);
                }
            }
    };
    auto product = [&](const Frag (&x)[MT], const Frag (&y)[NT]) { product_of(x, y, std::integral_constant<int, 0>{}, std::integral_constant<int, MT>{}); };
    // 8 bits: the scales of a row's next four steps, a byte each; step u's (opsel) is a constant of the matrix instruction
    int sa[MT], sb[NT];
    bool plain = true;  // (EXACT) these scales, of the rows that there are
    auto take_scales = [&](int step) {
        const int* words = reinterpret_cast<const int*>(room + ST * kStage) + (step >> 2 & 1) * kWords + (l & 15);
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = words[32 * wm * MP + 16 * i];
#pragma unroll
        for (int i = 0; i < NT; ++i) sb[i] = words[Sh::BM + 32 * wn * NP + 16 * i];
        if constexpr (EXACT) {
            uint32_t all = kPlain;
#pragma unroll
            for (int i = 0; i < MT; ++i) all &= pa.first + 32 * wm * MP + 16 * i + (l & 15) >= a.m ? kPlain : q8_plain((uint32_t)sa[i]);
#pragma unroll
            for (int i = 0; i < NT; ++i) all &= pb.first + 32 * wn * NP + 16 * i + (l & 15) >= a.n ? kPlain : q8_plain((uint32_t)sb[i]);
            plain = __all(all == kPlain);
        }
    };
    auto multiply = [&](const char* stage, auto opsel) {
        constexpr int U = decltype(opsel)::value;
#pragma unroll
        for (int s = 0; s < K::kSub; ++s) {
            if constexpr (EXACT) if (!plain) {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    asm volatile("" ::: "memory");  // blocks are read one by one: all of them, as bf16, are more registers than two workgroups a CU have
                    const Frag x = fa.frag(stage, i, A::template block<MT>(i, half), s);
                    int scale[4];                   // of rows 4 (l / 16) ..: the lanes of those rows have them
#pragma unroll
                    for (int e = 0; e < 4; ++e) scale[e] = __shfl(sa[i], 4 * (l >> 4) + e) >> (8 * U);
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const Frag y = fb.frag(stage + A::kBytes, j, B::template block<NT>(j, 0), s);
                        f32x4 t = {};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q8_values(x, e, q8_none(sa[i] >> (8 * U))), q8_values(y, e, q8_none(sb[j] >> (8 * U))), t, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] += q8_scaled(t[e], scale[e], sb[j] >> (8 * U));
                    }
                }
                continue;
            }
            Frag x[MT], y[NT];
            take(stage, s, x, y);
            if constexpr (EXACT) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    bf16x8 u[MT], v[NT];
#pragma unroll
                    for (int i = 0; i < MT; ++i) u[i] = q8_values(x[i], e, q8_all(sa[i] >> (8 * U)));
#pragma unroll
                    for (int j = 0; j < NT; ++j) v[j] = q8_values(y[j], e, q8_all(sb[j] >> (8 * U)));
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u[i], v[j], acc[i][j], 0, 0, 0);
                }
            } else if constexpr (sizeof(T) == 1) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[i], y[j], acc[i][j], 0, 0, U, sa[i], U, sb[j]);
            } else {
                product(x, y);
            }
        }
    };

    if constexpr (VEC) {
        Direct<T, Sh::BM, TA, kThreads> la;
        Direct<T, Sh::BN, TB, kThreads> lb;
        la.aim(pa, gate), lb.aim(pb, false);
        constexpr int kLoads = A::kLoads + B::kLoads;  // of a wavefront a step (8 bits: at least)
        const uint32_t lds = lds_address(room);
        auto load_first = [&](int step, int stage) { la.load(pa, step, gate, ups, lds + stage * kStage); };
        auto load_second = [&](int step, int stage) { lb.load(pb, step, false, 0, lds + stage * kStage + A::kBytes); };
        auto load = [&](int step, int stage) {
            load_first(step, stage), load_second(step, stage);
            if constexpr (sizeof(T) == 1) {
                // a word a row, four steps' scales (zeros behind the rows)
                if ((step & 3) == 0 || step == begin) {
#pragma unroll
                    for (int j = 0; j < (kWords + kThreads - 1) / kThreads; ++j) {
                        const int base = __builtin_amdgcn_readfirstlane(j * kThreads + (int)(threadIdx.x & ~63u));
                        if (base >= kWords) continue;
                        const Place& o = base < Sh::BM ? pa : pb;
                        const int q = (base < Sh::BM ? base : base - Sh::BM) + l;
                        const uint8_t* from = (base < Sh::BM ? a.first_scales : a.second_scales) + (int64_t)o.first * a.scales + (step >> 2) * 4;
                        word_to_lds(memory_of(from, 0x7fffffffu), o.first + q < o.count ? (uint32_t)(q * a.scales) : kOutside,
                                    lds + ST * kStage + ((step >> 2 & 1) * kWords + base) * 4);
                    }
                }
            }
        };
        if constexpr (kAhead) {
            // Fragments are read while the ones before them are multiplied.  One meeting a step, between its two fragments: behind it nobody reads this
            // step's tiles any more, and the next step's are there.
            // One operand's loads come between the halves of a step's products, of 8192 x 2048 x 8192 18 - 25 us less for the gate; which one, 2 - 3 % less.
            static_assert(K::kSub == 2, "two fragments a step");
            constexpr bool kFirstFirst = (TA && TB) || LAST == kGateBack;
            Frag x[2][MT], y[2][NT];
#pragma unroll
            for (int i = 0; i < ST; ++i)
                if (i < count) load(begin + i, i);
            if (ST <= count) wait_loads<(ST - 1) * kLoads>();
            else wait_loads<0>();
            meet();
            take(room, 0, x[0], y[0]);
            int stage = 0;
#pragma unroll 1
            for (int k = 0; k < count; ++k) {
                take(room + stage * kStage, 1, x[1], y[1]);
                product(x[0], y[0]);
                alternate();
                if (k + ST <= count) wait_loads<(ST - 2) * kLoads>();
                else wait_loads<0>();
                meet();
                const int free = stage;
                if (k + ST < count) kFirstFirst ? load_first(begin + k + ST, free) : load_second(begin + k + ST, free);
                stage = stage + 1 == ST ? 0 : stage + 1;
                take(room + stage * kStage, 0, x[0], y[0]);  // (behind the last step: a tile that is not used)
                product_of(x[1], y[1], std::integral_constant<int, 0>{}, std::integral_constant<int, MT / 2>{});
                alternate();
                if (k + ST < count) kFirstFirst ? load_second(begin + k + ST, free) : load_first(begin + k + ST, free);
                product_of(x[1], y[1], std::integral_constant<int, MT / 2>{}, std::integral_constant<int, MT>{});
            }
        } else {
#pragma unroll
            for (int s = 0; s < ST - 1; ++s)
                if (s < count) load(begin + s, s);
            int stage = 0, next = ST - 1;
            // (a part begins at a step whose scales are a word's first)
            auto step = [&](int k, auto opsel) {
                // this step's tiles are there; the ones behind it may still be under way
                if (k + ST - 1 <= count) wait_loads<(ST - 2) * kLoads>();
                else wait_loads<0>();
                meet();
                if (k + ST - 1 < count) load(begin + k + ST - 1, next);
                if constexpr (decltype(opsel)::value == 0) take_scales(begin + k);
                multiply(room + stage * kStage, opsel);
                stage = stage + 1 == ST ? 0 : stage + 1;
                next = next + 1 == ST ? 0 : next + 1;
            };
#pragma unroll 1
            for (int k = 0; k < count; k += 4) {
                step(k, std::integral_constant<int, 0>{});
                if (k + 1 < count) step(k + 1, std::integral_constant<int, 1>{});
                if (k + 2 < count) step(k + 2, std::integral_constant<int, 2>{});
                if (k + 3 < count) step(k + 3, std::integral_constant<int, 3>{});
            }
        }
    } else {
        Through<T, Sh::BM, TA, kThreads> la;
        Through<T, Sh::BN, TB, kThreads> lb;
        la.aim(pa, gate), lb.aim(pb, false);
        if (count > 0) la.load(pa, begin, gate, ups), lb.load(pb, begin, false, 0);
#pragma unroll 1
        for (int k = 0; k < count; ++k) {
            char* stage = room + (k & 1) * kStage;
            la.store(stage), lb.store(stage + A::kBytes);
            wait_loads<0>();
            meet();
            if (k + 1 < count) la.load(pa, begin + k + 1, gate, ups), lb.load(pb, begin + k + 1, false, 0);
            multiply(stage, std::integral_constant<int, 0>{});
        }
    }

    // Blocks 2 p and 2 p + 1 hold columns 4 h .. of 32 p and 32 p + 16, h the lane's group; lanes of odd groups swap the first's with the second's of
    // the group before: 8 (h >> 1) .. of the first, or of the second.
#pragma unroll
    for (int i = 0; i < MT; i += 2)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][j][e]), __float_as_uint(acc[i + 1][j][e]), false, false);
                acc[i][j][e] = __uint_as_float(both[0]), acc[i + 1][j][e] = __uint_as_float(both[1]);
            }
    // The last step's items of a lane: eight columns of a row each, item t = (t / MP)'s block of rows.  In 16 bits lanes r and r + 8 of a block swap a
    // pair's half, so that a store writes 128 bytes of 8 rows instead of 64 of 16.
    constexpr bool kWhole = sizeof(T) <= 2 && MP % 2 == 0;
    auto row_at = [&](int t) { return (int64_t)pb.first + 32 * wn * NP + 16 * (t / MP) + (kWhole ? 8 * (t & 1) + (l & 7) : l & 15); };
    auto col_at = [&](int t) {
        return pa.first + 32 * (wm * MP + (kWhole ? t % MP / 2 * 2 + (l >> 3 & 1) : t % MP)) + 16 * (l >> 4 & 1) + 8 * (l >> 5);
    };
    auto values = [&](int t, int from) {  // from: the first block of these columns
        const int j = t / MP, p = t % MP;
        Eight v;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (kWhole) {
                const float lo = acc[from + 2 * (p & ~1) + (e >> 2)][j][e & 3], hi = acc[from + 2 * (p | 1) + (e >> 2)][j][e & 3];
                const bool high = l & 8;
                const float swapped = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, high ? lo : hi), 0x128, 0xf, 0xf, false));
                v.e[e] = t & 1 ? (high ? hi : swapped) : (high ? swapped : lo);
            } else {
                v.e[e] = acc[from + 2 * p + (e >> 2)][j][e & 3];
            }
        }
        return v;
    };
    // Tiles that lie within the results, nearly all, have code of their own: with a way out for each of eight columns behind every store the last step
    // is so long that it is fetched from memory again and again.
    constexpr int kItems = NT * MP, kMostAhead = LAST == kGateBack ? sizeof(T) == 2 ? 4 : 2 : 1, kAheadBy = kMostAhead < kItems ? kMostAhead : kItems;
    static_assert(kAheadBy <= kItems, "an item that is read ahead is one of the lane's: the rows behind a tile may be none of the matrix");
    auto items = [&](auto inside, auto act) {
        constexpr bool kInside = decltype(inside)::value;
        constexpr int kAct = decltype(act)::value;
        auto left = [&](int col) { return kInside ? 8 : a.m - col; };
        KeptOf<std::conditional_t<sizeof(T) == 1, float, T>> kept[kAheadBy];  // (kGateBack) what was kept is read some items ahead
        auto fetch = [&](int t) {
            if constexpr (LAST == kGateBack) {
                const int col = col_at(t);
                if (left(col) > 0) kept[t % kAheadBy] = kept_at<T>(a, kInside ? row_at(t) : min(row_at(t), (int64_t)a.n - 1), col, left(col));
            }
        };
#pragma unroll
        for (int t = 0; t < kAheadBy; ++t) fetch(t);
#pragma unroll
        for (int t = 0; t < kItems; ++t) {
            const int64_t row = row_at(t);
            const int col = col_at(t);
            const Eight v = values(t, 0);
            Eight u;
            if constexpr (gate) u = values(t, MT / 2);
            if (kInside || (row < a.n && col < a.m)) {
                if constexpr (gate) put_gate<T, kAct>(a, row, col, v, u, left(col));
                else if constexpr (LAST == kGateBack) put_gate_back<T, kAct>(a, row, col, v, kept[t % kAheadBy], left(col));
                else if (a.last == kPartial) put_eight(a.part + ((int64_t)split * a.n + row) * a.m + col, v, left(col));
                else put_out<T>(a, row, col, v, left(col));
            }
            if constexpr (LAST == kGateBack) {
                if (t + kAheadBy < kItems) fetch(t + kAheadBy);
                __builtin_amdgcn_sched_barrier(0);  // what is ahead stays ahead: the compiler would move it to where it is used, to save registers
            }
        }
    };
    auto with = [&](auto act) {
        if (pa.first + cols <= a.m && pb.first + Sh::BN <= a.n) items(std::true_type{}, act);
        else items(std::false_type{}, act);
    };
    if constexpr (gate || LAST == kGateBack) with_act(a.act, with);
    else with(std::integral_constant<int, 0>{});
}

template <typename T, typename Sh, bool TA, bool TB, bool VEC, bool EXACT, Last LAST>
__global__ __launch_bounds__(Sh::kThreads) void mm_kernel(Mm a) {
    __shared__ char room[Room<T, Sh, VEC>::kBytes] __attribute__((aligned(16)));
    mm_body<T, Sh, TA, TB, VEC, EXACT, LAST>(a, blockIdx.x, room);
}

// Three products that do not wait for each other, the first of a turned and a direct operand, the others of turned ones, in one launch: small ones
// leave most of the chip idle, and a launch takes the host 2.7 us.
struct Three {
    Mm p[3];
    uint32_t end[3];  // workgroups up to and with each
};
template <typename T, typename Sh, bool VEC0, bool VEC>
__global__ __launch_bounds__(Sh::kThreads) void mm_three_kernel(Three t) {
    constexpr int kRoom = Room<T, Sh, VEC0>::kBytes > Room<T, Sh, VEC>::kBytes ? Room<T, Sh, VEC0>::kBytes : Room<T, Sh, VEC>::kBytes;
    __shared__ char room[kRoom] __attribute__((aligned(16)));
    const uint32_t block = blockIdx.x;
    if (block < t.end[0]) return mm_body<T, Sh, true, false, VEC0, false, kStore>(t.p[0], block, room);
    const int i = block < t.end[1] ? 1 : 2;
    mm_body<T, Sh, true, true, VEC, false, kStore>(t.p[i], block - t.end[i - 1], room);
}

// ---- the parts' sums, and the last step ---------------------------------------------------------------------------
// a.m: the results' columns (of a gate: the hidden width, parts have 2 m columns).  GROUPS threads share the parts of eight columns, each GROUPS-th of
// them in order, and the threads' sums are added in order: 42 parts of 540 x 100 results one after another took 20 us.
template <typename T, int GROUPS>
__device__ __forceinline__ void mm_join(const Mm& a, uint32_t block, Eight* room) {
    constexpr int kItems = 256 / GROUPS;
    const int each = (a.m + 7) / 8, item = threadIdx.x % kItems, group = threadIdx.x / kItems;
    const int64_t i = (int64_t)block * kItems + item, row = i / each;
    const bool there = row < a.n, gate = a.last == kGate;
    const int col = (int)(i - row * each) * 8, wide = gate ? 2 * a.m : a.m;
    auto sum = [&](int at) {
        Eight s{};
        if (there)
#pragma unroll 4
            for (int p = group; p < a.splits; p += GROUPS) {
                const Eight v = get_eight(a.part + ((int64_t)p * a.n + row) * wide + at, a.m - col);
#pragma unroll
                for (int e = 0; e < 8; ++e) s.e[e] += v.e[e];
            }
        return s;
    };
    Eight s = sum(col), u = gate ? sum(a.m + col) : Eight{};
    if constexpr (GROUPS > 1) {
        room[threadIdx.x] = s, room[256 + threadIdx.x] = u;
        __syncthreads();
        if (group) return;
        for (int g = 1; g < GROUPS; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) s.e[e] += room[g * kItems + item].e[e], u.e[e] += room[256 + g * kItems + item].e[e];
    }
    if (!there) return;
    if constexpr (sizeof(T) > 1) {
        if (gate || a.last == kGateBack)
            return with_act(a.act, [&](auto act) {
                if (gate) put_gate<T, decltype(act)::value>(a, row, col, s, u, a.m - col);
                else put_gate_back<T, decltype(act)::value>(a, row, col, s, kept_at<T>(a, row, col, a.m - col), a.m - col);
            });
    }
    put_out<T>(a, row, col, s, a.m - col);
}

template <typename T, int GROUPS>
__global__ __launch_bounds__(256) void mm_join_kernel(Mm a) {
    __shared__ Eight room[GROUPS > 1 ? 2 * 256 : 1];
    mm_join<T, GROUPS>(a, blockIdx.x, room);
}
template <typename T>
__global__ __launch_bounds__(256) void mm_join_three_kernel(Three t) {
    __shared__ Eight room[2 * 256];
    const uint32_t block = blockIdx.x;
    const int i = block < t.end[0] ? 0 : block < t.end[1] ? 1 : 2;
    mm_join<T, 8>(t.p[i], i ? block - t.end[i - 1] : block, room);
}

// ---- few rows --------------------------------------------------------------------------------------------------------
// Up to 16 * NB rows (a serving batch's tokens): bound by reading the first operand once, from memory to registers.  A workgroup makes 16 columns
// (of a gate: 16 gates and their ups) of all rows; its wavefronts share the contraction and add their sums through LDS, in order, so that the last
// step needs no second kernel.  8 x 4096 x 8192 in bf16, gated: 25 us for 134 MB (5.4 TB/s) where parts joined by a second
// kernel took 33.
template <typename T, int NB, bool GATE, bool VEC, bool EXACT>
__global__ __launch_bounds__(1024) void mm_thin_kernel(Mm a) {
    using K = Kind<T>;
    using Frag = typename K::Frag;
    constexpr int kBytes = sizeof(T) == 1 ? 128 : 64, kSides = GATE ? 2 : 1, kAtOnce = (VEC ? sizeof(T) == 1 ? 4 : 8 : 2) / NB;  // bytes of a row a fragment
    constexpr int kWhole = sizeof(T) == 1 ? 4 : 1;  // a word has four steps' scales: wavefronts begin at one
    extern __shared__ float sums[];  // [wavefront][gates, ups][block][row of 16][16 columns]
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, l = threadIdx.x & 63, h = l >> 4, r = l & 15;
    const int col0 = blockIdx.x * 16, all = (int)(((int64_t)a.k * (int)sizeof(T) + kBytes - 1) / kBytes);
    const int each = ((all + waves - 1) / waves + kWhole - 1) / kWhole * kWhole;
    const int begin = wave * each, end = min(all, begin + each);
    // rows that there are not have another's values: their results are not stored
    const char* from[kSides + NB];
    const uint8_t* scales[kSides + NB];
#pragma unroll
    for (int i = 0; i < kSides + NB; ++i) {
        const bool first = i < kSides;
        const int64_t row = first ? (int64_t)min(col0 + r, a.m - 1) + (int64_t)i * a.m : min((i - kSides) * 16 + r, a.n - 1);
        from[i] = static_cast<const char*>(first ? a.first : a.second) + row * (first ? a.ld_first : a.ld_second);
        if constexpr (sizeof(T) == 1) scales[i] = (first ? a.first_scales : a.second_scales) + row * a.scales;
    }
    auto piece = [&](const char* row, int64_t at) {
        const int64_t left = (int64_t)a.k * (int)sizeof(T) - at;
        if constexpr (VEC) return left > 0 ? *reinterpret_cast<const uint4*>(row + at) : uint4{};
        Piece<T, K::kPer> v{};
        if (left >= 16) __builtin_memcpy(&v, row + at, 16);
        else
#pragma unroll
            for (int i = 0; i < K::kPer; ++i)
                if (i * (int)sizeof(T) < left) v.e[i] = reinterpret_cast<const T*>(row + at)[i];
        return __builtin_bit_cast(uint4, v);
    };
    auto fragment = [&](const char* row, int s) {
        const int64_t at = (int64_t)s * kBytes + 16 * h;
        if constexpr (sizeof(T) == 1) {
            const uint4 lo = piece(row, at), hi = piece(row, at + 64);
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        } else {
            return __builtin_bit_cast(Frag, piece(row, at));
        }
    };
    f32x4 acc[kSides][NB] = {};
    auto some = [&](int s0, int count) {  // `count` fragments, up to kAtOnce: all are asked for before the first is used
        Frag x[kAtOnce][kSides], y[kAtOnce][NB];
        uint32_t sx[kSides], sy[NB];
        if constexpr (sizeof(T) == 1) {
            static_assert(kAtOnce <= kWhole, "one word");
#pragma unroll
            for (int i = 0; i < kSides; ++i) sx[i] = *reinterpret_cast<const uint32_t*>(scales[i] + (s0 & ~3));
#pragma unroll
            for (int j = 0; j < NB; ++j) sy[j] = *reinterpret_cast<const uint32_t*>(scales[kSides + j] + (s0 & ~3));
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (u >= count) break;
#pragma unroll
            for (int i = 0; i < kSides; ++i) x[u][i] = fragment(from[i], s0 + u);
#pragma unroll
            for (int j = 0; j < NB; ++j) y[u][j] = fragment(from[kSides + j], s0 + u);
        }
        bool plain = true;
        if constexpr (sizeof(T) == 1) {
            if constexpr (EXACT) {
                uint32_t all = kPlain;
#pragma unroll
                for (int i = 0; i < kSides; ++i) all &= q8_plain(sx[i]);
#pragma unroll
                for (int j = 0; j < NB; ++j) all &= q8_plain(sy[j]);
                plain = __all(all == kPlain);
            }
#pragma unroll
            for (int i = 0; i < kSides; ++i) sx[i] >>= 8 * (s0 & 3);
#pragma unroll
            for (int j = 0; j < NB; ++j) sy[j] >>= 8 * (s0 & 3);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (u >= count) break;
#pragma unroll
            for (int i = 0; i < kSides; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    if constexpr (EXACT) {
                        if (plain) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q8_values(x[u][i], e, q8_all((int)(sx[i] >> (8 * u)))), q8_values(y[u][j], e, q8_all((int)(sy[j] >> (8 * u)))), acc[i][j], 0, 0, 0);
                        } else {
                            f32x4 t = {};
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q8_values(x[u][i], e, q8_none((int)(sx[i] >> (8 * u)))), q8_values(y[u][j], e, q8_none((int)(sy[j] >> (8 * u)))), t, 0, 0, 0);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][e] += q8_scaled(t[e], __shfl((int)sx[i], 4 * h + e) >> (8 * u), (int)(sy[j] >> (8 * u)));
                        }
                    } else if constexpr (sizeof(T) == 1) {
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[u][i], y[u][j], acc[i][j], 0, 0, 0, (int)(sx[i] >> (8 * u)), 0, (int)(sy[j] >> (8 * u)));
                    } else if constexpr (sizeof(T) == 2) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[u][i], y[u][j], acc[i][j], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[u][i][e], y[u][j][e], acc[i][j], 0, 0, 0);
                    }
                }
        }
    };
    int s = begin;
#pragma unroll 1
    for (; s + kAtOnce <= end; s += kAtOnce) some(s, kAtOnce);
#pragma unroll 1
    for (; s < end; ++s) some(s, 1);
#pragma unroll
    for (int i = 0; i < kSides; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4*>(sums + ((wave * kSides + i) * NB + j) * 256 + r * 16 + 4 * h) = acc[i][j];
    __syncthreads();
    // eight columns a thread
    const int row = threadIdx.x >> 1, col = col0 + 8 * (threadIdx.x & 1);
    if (row >= a.n || col >= a.m) return;
    auto sum = [&](int i) {
        Eight v{};
        const float* p = sums + (i * NB + row / 16) * 256 + row % 16 * 16 + 8 * (threadIdx.x & 1);
#pragma unroll 4
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) v.e[e] += p[w * kSides * NB * 256 + e];
        return v;
    };
    if constexpr (GATE) with_act(a.act, [&](auto act) { put_gate<T, decltype(act)::value>(a, row, col, sum(0), sum(1), a.m - col); });
    else put_out<T>(a, row, col, sum(0), a.m - col);
}

constexpr int kThinRows = 32;
// Wavefronts of a workgroup: 16 a CU, while each has two fragments to read; enough threads for the last step.
inline int thin_waves(int64_t groups, int64_t fragments) {
    int waves = 16;
    while (waves > 1 && ((groups * waves > 4096 && waves > 4) || 2 * (waves - 1) >= fragments)) waves /= 2;
    return waves;
}
template <typename T, bool GATE, bool VEC, bool EXACT>
int mm_thin(Mm a, hipStream_t s) {
    const int64_t groups = ((int64_t)a.m + 15) / 16, bytes = sizeof(T) == 1 ? 128 : 64;
    const int waves = thin_waves(groups, ((int64_t)a.k * (int)sizeof(T) + bytes - 1) / bytes);
    const size_t room = (size_t)waves * (GATE ? 2 : 1) * (a.n > 16 ? 2 : 1) * 1024;
    // (of gates there are at most 2^14 groups, one launch)
    const int64_t most = ((int64_t)1 << 26) / (waves * 64);
    for (int64_t group = 0; group < groups; group += most) {
        const dim3 grid((unsigned)(groups - group < most ? groups - group : most));
        if (a.n <= 16) hipLaunchKernelGGL((mm_thin_kernel<T, 1, GATE, VEC, EXACT>), grid, dim3(waves * 64), room, s, a);
        else hipLaunchKernelGGL((mm_thin_kernel<T, 2, GATE, VEC, EXACT>), grid, dim3(waves * 64), room, s, a);
        SP_HIP(hipGetLastError());
        a.m -= (int)(most * 16);
        a.first = static_cast<const char*>(a.first) + most * 16 * a.ld_first;
        a.first_scales += most * 16 * a.scales;
        a.out = static_cast<char*>(a.out) + most * 16 * (sizeof(T) > 1 ? (int)sizeof(T) : a.out_f32 ? 4 : 2);
    }
    return SP_OK;
}

// ---- which workgroups, how many parts --------------------------------------------------------------------------
enum ShapeName { kLarge, kMiddle, kNarrow, kFew };
struct Plan {
    ShapeName shape;
    int splits, per_split, tiles_m, tiles_n;
    double time;  // us, about
};
constexpr double kNoPlan = 1e300;                           // (time) more tiles than a launch has threads for
constexpr int64_t kNoWork = (int64_t)1 << 62;
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1;  // a launch of more is cut short without an error
// rows: of the first operand (a gate: 2 m); k_bytes: of a row of the contraction
enum MmType { kF32, kBf16, kQ8, kQ8Exact };
Plan mm_plan(int64_t rows, int64_t n, int64_t k_bytes, MmType type, bool pieces);
// Bytes of the parts' sums (0: none).  direct: both operands are.
inline int64_t mm_work(int64_t rows, int64_t n, int64_t k_bytes, MmType type, bool direct, bool pieces) {
    if (direct && n <= kThinRows) return 0;
    const Plan p = mm_plan(rows, n, k_bytes, type, pieces);
    if (p.time == kNoPlan) return kNoWork;
    return p.splits > 1 ? (int64_t)p.splits * rows * n * 4 : 0;
}

template <typename T, typename Sh, bool TA, bool TB, bool VEC, bool EXACT, Last LAST>
int mm_launch(const Mm& a, hipStream_t s) {
    const int64_t blocks = (int64_t)a.tiles_m * a.tiles_n * a.splits;
    hipLaunchKernelGGL((mm_kernel<T, Sh, TA, TB, VEC, EXACT, LAST>), dim3((unsigned)blocks), dim3(Sh::kThreads), 0, s, a);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

// Are both operands' rows whole, aligned 16-byte pieces?
template <typename T>
bool mm_whole(const Mm& a, bool turned_first, bool turned_second) {
    auto whole = [](const void* p, int64_t ld, int64_t row) { return aligned16(p) && ld % 16 == 0 && row * (int64_t)sizeof(T) % 16 == 0; };
    return whole(a.first, a.ld_first, turned_first ? a.m : a.k) && whole(a.second, a.ld_second, turned_second ? a.n : a.k);
}

// Fills in what is left of `a` (steps, tiles, parts) and enqueues the product.  part: mm_work() bytes.
template <typename T, bool TA, bool TB>
int mm(Mm a, float* part, hipStream_t s) {
    const bool gate = a.last == kGate;
    const bool pieces = mm_whole<T>(a, TA, TB);
    const int64_t k_bytes = (int64_t)a.k * (int)sizeof(T);
    if constexpr (!TA && !TB)
        if (a.n <= kThinRows) {
            if constexpr (sizeof(T) == 1) {
                return a.out_f32 ? mm_thin<T, false, true, true>(a, s) : mm_thin<T, false, true, false>(a, s);
            } else {
                if (gate) return pieces ? mm_thin<T, true, true, false>(a, s) : mm_thin<T, true, false, false>(a, s);
                return pieces ? mm_thin<T, false, true, false>(a, s) : mm_thin<T, false, false, false>(a, s);
            }
        }
    const MmType type = sizeof(T) == 4 ? kF32 : sizeof(T) == 2 ? kBf16 : a.out_f32 ? kQ8Exact : kQ8;
    const Plan p = mm_plan(gate ? (int64_t)2 * a.m : a.m, a.n, k_bytes, type, pieces);
    if (p.time == kNoPlan) return fail(SP_ERR_UNSUPPORTED, "more results than a launch has threads for");
    a.steps = (int)((k_bytes + kStepBytes - 1) / kStepBytes);
    a.per_split = p.per_split, a.splits = p.splits, a.tiles_m = p.tiles_m, a.tiles_n = p.tiles_n;
    Mm last = a;
    const bool join = p.splits > 1;
    if (join) {
        a.last = kPartial, a.part = last.part = part;
        if (gate) a.m *= 2;
    }
    const bool alone = (int64_t)p.tiles_m * p.tiles_n * p.splits <= kCUs;
    auto go = [&](auto vec, auto exact) -> int {
        constexpr bool V = decltype(vec)::value, X = decltype(exact)::value;
        auto with = [&](auto last) -> int {
            constexpr Last L = (Last)decltype(last)::value;
            switch (p.shape) {
                case kLarge:
                    if constexpr (V && !X) return mm_launch<T, Large, TA, TB, V, X, L>(a, s);
                    break;
                case kMiddle:
                    if constexpr (V && !X && sizeof(T) < 4)
                        if (alone) return mm_launch<T, MiddleDeep, TA, TB, V, X, L>(a, s);
                    return mm_launch<T, Middle, TA, TB, V, X, L>(a, s);
                case kNarrow: return mm_launch<T, Narrow, TA, TB, V, X, L>(a, s);
                case kFew:
                    if constexpr (TA || TB) return mm_launch<T, Few, TA, TB, V, X, L>(a, s);
                    break;
            }
            return fail(SP_ERR_UNSUPPORTED, "no kernel for this product");
        };
        if constexpr (sizeof(T) > 1 && !TA && !TB)
            if (a.last == kGate) return with(std::integral_constant<int, kGate>{});
        if constexpr (sizeof(T) > 1 && TA && !TB)
            if (a.last == kGateBack) return with(std::integral_constant<int, kGateBack>{});
        return with(std::integral_constant<int, kStore>{});
    };
    if constexpr (sizeof(T) == 1) {
        SP_TRY(a.out_f32 ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{}));
    } else {
        SP_TRY(pieces ? go(std::true_type{}, std::false_type{}) : go(std::false_type{}, std::false_type{}));
    }
    if (join) {
        auto add = [&](auto groups) -> int {
            constexpr int G = decltype(groups)::value;
            const int64_t blocks = ((int64_t)((last.m + 7) / 8) * last.n + 256 / G - 1) / (256 / G);
            if (blocks > kMostThreads / 256) return fail(SP_ERR_UNSUPPORTED, "more results than a launch has threads for");
            hipLaunchKernelGGL((mm_join_kernel<T, G>), dim3((unsigned)blocks), dim3(256), 0, s, last);
            SP_HIP(hipGetLastError());
            return SP_OK;
        };
        SP_TRY(p.splits >= 8 ? add(std::integral_constant<int, 8>{}) : add(std::integral_constant<int, 1>{}));
    }
    return SP_OK;
}

inline int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }

// Of three products rows x n over a contraction: one launch's workgroups, or none if three launches are as fast.
struct Size {
    int64_t rows, n, k_bytes;
};
struct PlanThree {
    bool together;
    Plan p[3];
};
PlanThree mm_plan_three(const Size (&of)[3], MmType type, bool pieces);
inline int64_t mm_work_three(const Size (&of)[3], MmType type, bool pieces) {
    const PlanThree t = mm_plan_three(of, type, pieces);
    int64_t bytes = 0;
    for (int i = 0; i < 3; ++i)
        if (t.together && t.p[i].splits > 1) bytes += up256((int64_t)t.p[i].splits * of[i].rows * of[i].n * 4);
    return bytes;
}

// The first of a turned and a direct operand, the others of turned ones; every one kStore.  part: mm_work_three() bytes, and mm_work() of each.
template <typename T>
int mm_three(const Mm (&of)[3], char* part, hipStream_t s) {
    const MmType type = sizeof(T) == 4 ? kF32 : kBf16;
    Size size[3];
    bool whole[3];
    for (int i = 0; i < 3; ++i) {
        size[i] = Size{of[i].m, of[i].n, (int64_t)of[i].k * (int)sizeof(T)};
        whole[i] = mm_whole<T>(of[i], true, i > 0);
    }
    const PlanThree plan = mm_plan_three(size, type, whole[0] && whole[1] && whole[2]);
    if (!plan.together) {
        SP_TRY((mm<T, true, false>(of[0], reinterpret_cast<float*>(part), s)));
        SP_TRY((mm<T, true, true>(of[1], reinterpret_cast<float*>(part), s)));
        return mm<T, true, true>(of[2], reinterpret_cast<float*>(part), s);
    }
    Three t{}, join{};
    uint32_t blocks = 0, joins = 0;
    for (int i = 0; i < 3; ++i) {
        const Plan& p = plan.p[i];
        Mm& a = t.p[i];
        a = of[i];
        a.steps = (int)((size[i].k_bytes + kStepBytes - 1) / kStepBytes);
        a.per_split = p.per_split, a.splits = p.splits, a.tiles_m = p.tiles_m, a.tiles_n = p.tiles_n;
        join.p[i] = a;
        if (p.splits > 1) {
            a.last = kPartial, a.part = join.p[i].part = reinterpret_cast<float*>(part);
            part += up256((int64_t)p.splits * a.n * a.m * 4);
            joins += (uint32_t)(((int64_t)((a.m + 7) / 8) * a.n + 31) / 32);
        }
        blocks += (uint32_t)p.tiles_m * p.tiles_n * p.splits;
        t.end[i] = blocks, join.end[i] = joins;
    }
    auto go = [&](auto shape, auto vec0, auto vec) {
        using Sh = decltype(shape);
        hipLaunchKernelGGL((mm_three_kernel<T, Sh, decltype(vec0)::value, decltype(vec)::value>), dim3(blocks), dim3(Sh::kThreads), 0, s, t);
    };
    auto with = [&](auto shape) {
        const bool vec = whole[1] && whole[2];
        if (whole[0]) vec ? go(shape, std::true_type{}, std::true_type{}) : go(shape, std::true_type{}, std::false_type{});
        else vec ? go(shape, std::false_type{}, std::true_type{}) : go(shape, std::false_type{}, std::false_type{});
    };
    const bool deep = sizeof(T) < 4 && blocks <= kCUs && whole[0] && whole[1] && whole[2];
    if (plan.p[0].shape == kMiddle) {
        if constexpr (sizeof(T) < 4) deep ? go(MiddleDeep{}, std::true_type{}, std::true_type{}) : with(Middle{});
        else with(Middle{});
    } else {
        with(Narrow{});
    }
    SP_HIP(hipGetLastError());
    if (joins) {
        hipLaunchKernelGGL(mm_join_three_kernel<T>, dim3(joins), dim3(256), 0, s, join);
        SP_HIP(hipGetLastError());
    }
    return SP_OK;
}

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
