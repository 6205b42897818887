// Rotary positions: every pair of elements of a head is turned by an angle that grows with the row's position on one of its axes.
//
// Memory bound: x is read and y is written once.  The angles belong to a row and a pair, not to a head, so a workgroup takes a few rows,
// computes their cosines and sines once into LDS and then goes over all heads' elements.  position * frequency is taken in fp64 and in
// turns, its whole part dropped: a far position (2^31) is as exact as a near one, where a product in fp32 is off by a radian at 10^7.
// Pairs of neighbouring elements, and halves that are whole 16-byte pieces, move in 16-byte pieces; other halves pair by pair, with
// neighbouring lanes at neighbouring elements.  A thread reads both elements of a pair before it writes either, so y may be x.  373601 rows of 16 heads
// of 32 in bf16, 765 MB: 142 us (5.4 TB/s).  Frequencies come with the launch: from powers of two of their index in the kernel they took 150.
#include <algorithm>
#include <cmath>

#include "sp_elem.h"

namespace sp {
namespace {

constexpr int kMaxPairs = 128;
constexpr int kTable = 1024;  // cosines and sines of a workgroup: rows * pairs, unless one row has more
constexpr int kThreads = 256;

struct Rope {
    int64_t n, ldx, ldy, ld_pos;
    const int32_t* pos;
    int heads, dim, axes, pairs, rows;  // rows of a workgroup
    int first[4], end[4];               // pairs of each axis
    bool back;
    double freq[kMaxPairs];             // turns a position
};

// What a thread moves at a time: V elements of a head from `at` on and, if they are the first of pairs, their partners `second` elements
// behind (0: they stay as they are, or hold both of a pair); `pair`: their first pair.
struct Item {
    int at, second, pair;
};

__device__ __forceinline__ int axis_of(const Rope& a, int pair) {
    int axis = 0;
#pragma unroll
    for (int k = 1; k < 4; ++k) axis += k < a.axes && pair >= a.end[k - 1];
    return axis;
}

// Item q of a head: V pairs of an axis while there are any, then V elements that stay; neighbours in pieces: V elements, whatever they are.
template <int V, bool SPLIT>
__device__ __forceinline__ Item item_of(const Rope& a, int q) {
    if constexpr (!SPLIT && V > 1) return Item{q * V, 0, q * V / 2};
    const int pair = q * V;
    if (pair >= a.pairs) return Item{pair + a.pairs, 0, 0};
    if constexpr (!SPLIT) return Item{2 * pair, 1, pair};
    const int axis = axis_of(a, pair);
    return Item{pair + a.first[axis], a.end[axis] - a.first[axis], pair};
}

template <typename T, int V, bool SPLIT>
__global__ __launch_bounds__(kThreads) void rope_kernel(Rope a, const T* x, T* y) {
    __shared__ float2 table[kTable];
    const int64_t row0 = (int64_t)blockIdx.x * a.rows;
    const int rows = a.n - row0 < a.rows ? (int)(a.n - row0) : a.rows;
    for (int i = threadIdx.x; i < rows * a.pairs; i += kThreads) {
        const int r = i / a.pairs, pair = i - r * a.pairs;
        const double turns = (double)a.pos[(row0 + r) * a.ld_pos + axis_of(a, pair)] * a.freq[pair];
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        table[i] = float2{c, a.back ? -s : s};
    }
    __syncthreads();
    const int each = !SPLIT && V > 1 ? a.dim / V : (a.dim - a.pairs) / V;  // items of a head
    // item -> (row, head, item of the head), carried on from one to the next without dividing again
    const int step_h = kThreads / each, step_q = kThreads - step_h * each, step_r = step_h / a.heads;
    int h = threadIdx.x / each, q = threadIdx.x - h * each;
    int r = h / a.heads;
    h -= r * a.heads;
    while (r < rows) {
        const Item it = item_of<V, SPLIT>(a, q);
        const T* from = x + (row0 + r) * a.ldx + (int64_t)h * a.dim + it.at;
        T* to = y + (row0 + r) * a.ldy + (int64_t)h * a.dim + it.at;
        const float2* t = table + r * a.pairs + it.pair;
        if constexpr (V > 1) {
            Piece<T, V> p = load_piece<T, V>(from);
            if constexpr (SPLIT) {
                if (it.second) {
                    Piece<T, V> p2 = load_piece<T, V>(from + it.second);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float u = elem(p.e[i]), v = elem(p2.e[i]);
                        const float2 cs = t[i];
                        p.e[i] = to_elem<T>(u * cs.x - v * cs.y);
                        p2.e[i] = to_elem<T>(u * cs.y + v * cs.x);
                    }
                    store_piece<T, V>(to + it.second, p2);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; i += 2)
                    if (it.pair + i / 2 < a.pairs) {
                        const float u = elem(p.e[i]), v = elem(p.e[i + 1]);
                        const float2 cs = t[i / 2];
                        p.e[i] = to_elem<T>(u * cs.x - v * cs.y);
                        p.e[i + 1] = to_elem<T>(u * cs.y + v * cs.x);
                    }
            }
            store_piece<T, V>(to, p);
        } else {
            if (it.second) {
                const float u = elem(from[0]), v = elem(from[it.second]);
                const float2 cs = *t;
                to[0] = to_elem<T>(u * cs.x - v * cs.y);
                to[it.second] = to_elem<T>(u * cs.y + v * cs.x);
            } else {
                to[0] = from[0];
            }
        }
        q += step_q;
        h += step_h - step_r * a.heads;
        r += step_r;
        if (q >= each) q -= each, ++h;
        if (h >= a.heads) h -= a.heads, ++r;
    }
}

template <typename T, int V, bool SPLIT>
int rope_launch(Rope& a, const void* x, void* y, hipStream_t s) {
    // A launch of 2^32 threads or more is cut short without an error.
    const int64_t n = a.n, most = (int64_t)a.rows << 22;
    for (int64_t row = 0; row < n; row += most, a.pos += most * a.ld_pos) {
        a.n = std::min(most, n - row);
        hipLaunchKernelGGL((rope_kernel<T, V, SPLIT>), dim3((unsigned)((a.n + a.rows - 1) / a.rows)), dim3(kThreads), 0, s, a,
                           static_cast<const T*>(x) + row * a.ldx, static_cast<T*>(y) + row * a.ldy);
        SP_HIP(hipGetLastError());
    }
    return SP_OK;
}

template <typename T>
int rope_typed(Rope& a, bool split, const void* x, void* y, hipStream_t s) {
    constexpr int kN = 16 / (int)sizeof(T);
    bool pieces = aligned16(x) && aligned16(y) && a.dim % kN == 0 && (a.n == 1 || (a.ldx % kN == 0 && a.ldy % kN == 0));
    if (split)
        for (int k = 0; k < a.axes; ++k) pieces &= (a.end[k] - a.first[k]) % kN == 0;
    if (split) return pieces ? rope_launch<T, kN, true>(a, x, y, s) : rope_launch<T, 1, true>(a, x, y, s);
    return pieces ? rope_launch<T, kN, false>(a, x, y, s) : rope_launch<T, 1, false>(a, x, y, s);
}

int rope(const sp_rope* r, bool back, const void* d_x, int64_t ldx, void* d_y, int64_t ldy, hipStream_t s) {
    if (!r) return fail(SP_ERR_INVALID_ARG, "the description is NULL");
    if (r->dt != SP_F32 && r->dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (r->n < 0 || r->n > (int64_t)1 << 40 || r->heads < 1 || r->heads > 65536 || r->dim < 1) return fail(SP_ERR_INVALID_ARG, "bad row, head or element count");
    if (r->axes < 1 || r->axes > 4) return fail(SP_ERR_INVALID_ARG, "1 to 4 axes");
    if (!(r->base > 0.0) || !std::isfinite(r->base) || !std::isfinite(r->scale)) return fail(SP_ERR_INVALID_ARG, "base and scale must be finite, base positive");
    Rope a{};
    int64_t used = 0;
    for (int k = 0; k < r->axes; ++k) {
        if (r->part[k] < 0 || r->part[k] % 2) return fail(SP_ERR_INVALID_ARG, "an axis turns an even number of elements");
        used += r->part[k];
    }
    if (used > r->dim) return fail(SP_ERR_INVALID_ARG, "the axes turn more elements than a head has");
    if (r->dim > 2 * kMaxPairs) return fail(SP_ERR_UNSUPPORTED, "heads of more than 256 elements");
    const int64_t wide = (int64_t)r->heads * r->dim;
    if (ldx < wide || ldy < wide) return fail(SP_ERR_INVALID_ARG, "rows overlap");
    if (r->ld_pos < r->axes) return fail(SP_ERR_INVALID_ARG, "positions overlap");
    if (r->n == 0) return SP_OK;
    if (!d_x || !d_y || !r->d_pos) return fail(SP_ERR_INVALID_ARG, "a feature or position pointer is NULL");
    if (d_x == d_y && ldx != ldy && r->n > 1) return fail(SP_ERR_INVALID_ARG, "in place, rows are equally far apart");
    a.n = r->n, a.ldx = ldx, a.ldy = ldy, a.ld_pos = r->ld_pos, a.pos = r->d_pos;
    a.heads = r->heads, a.dim = r->dim, a.axes = r->axes, a.back = back;
    for (int k = 0; k < r->axes; ++k) {
        const int half = r->part[k] / 2;
        a.first[k] = a.pairs;
        // base^(-i / half) from powers for each bit of i: seven calls of pow instead of one a pair, at most seven roundings more
        double bit[8], *f = a.freq + a.pairs;
        for (int b = 0; b < 8 && (1 << b) < half; ++b) bit[b] = std::pow(r->base, -(double)(1 << b) / half);
        for (int i = 0; i < half; ++i) f[i] = i ? f[i & (i - 1)] * bit[__builtin_ctz(i)] : r->scale / 6.283185307179586476925;
        a.pairs += half;
        a.end[k] = a.pairs;
    }
    // Rows of a workgroup: about eight 16-byte pieces a thread, as far as the table has room, but no fewer than two workgroups a CU.
    const int64_t bytes = wide * (r->dt == SP_F32 ? 4 : 2);
    int64_t rows = std::max<int64_t>(1, (int64_t)kThreads * 16 * 8 / bytes);
    rows = std::min<int64_t>(rows, kTable / std::max(a.pairs, 1));
    a.rows = (int)std::max<int64_t>(1, std::min<int64_t>(rows, r->n / 512));
    return r->dt == SP_F32 ? rope_typed<float>(a, r->split != 0, d_x, d_y, s) : rope_typed<bf16_t>(a, r->split != 0, d_x, d_y, s);
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" {

int sp_rope_fwd(const sp_rope* a, const void* d_x, int64_t ldx, void* d_y, int64_t ldy, void* stream) {
    return rope(a, false, d_x, ldx, d_y, ldy, (hipStream_t)stream);
}

int sp_rope_bwd(const sp_rope* a, const void* d_dy, int64_t lddy, void* d_dx, int64_t lddx, void* stream) {
    return rope(a, true, d_dy, lddy, d_dx, lddx, (hipStream_t)stream);
}

}  // extern "C"
