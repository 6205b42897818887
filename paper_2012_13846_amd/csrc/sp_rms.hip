// Root-mean-square norm of the rows of a feature matrix with the residual's addition, its output as features or in 8 bits, and its
// gradients.
//
// Memory bound: the forward pass reads x and the residual and writes their sum and y, the backward pass reads the sum, dy and the sum's
// own gradient and writes dx, each once.  A row stays in the registers of the LANES threads that share it, 16 bytes (V elements) each and P times;
// the next row is asked for before this one is reduced.  Pieces that are not aligned (odd widths, views) are loaded and stored as wide by
// unaligned instructions, but for the piece that holds a row's end.  What is normalised is the sum as it is stored, so that the backward
// pass finds the same.  In 8 bits the 16 (fp32: 32) neighbouring lanes that hold 128 elements share their largest size.  The weight's gradient is
// summed in the lanes that own the columns, then over a workgroup's row groups through LDS, and the workgroups' sums are added in fp64 in X16384 x 4096 in bf16: 93 us forward (5.7 TB/s), 115 + 5 back (4.7).  Rows to 8 bits: 8192 x 2048 10.5 us, transposed 11.5.
#include <algorithm>
#include <type_traits>

#include "sp_q8.h"

namespace sp {
namespace {

template <int LANES>
constexpr int kBlock = LANES > 256 ? LANES : 256;

// V elements from `p`, of which `left` (1 or more) exist; zeros behind.
template <typename T, int V, bool ALIGNED>
__device__ __forceinline__ Piece<T, V> load_some(const T* p, int left) {
    Piece<T, V> r;
    if constexpr (ALIGNED) return load_piece<T, V>(p);
    if (left >= V) __builtin_memcpy(&r, p, sizeof r);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) r.e[i] = i < left ? p[i] : T(0);
    return r;
}
template <typename T, int V, bool ALIGNED>
__device__ __forceinline__ void store_some(T* p, const Piece<T, V>& r, int left) {
    if constexpr (ALIGNED) return store_piece<T, V>(p, r);
    if (left >= V) __builtin_memcpy(p, &r, sizeof r);
    else
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) p[i] = r.e[i];
}

template <typename T>
struct RmsFwd {
    const T *x, *res;  // res: NULL or the residual
    int64_t n;
    int c;
    const float* gamma;
    float eps;
    T *h, *y;          // h: with a residual, their sum; y: NULL if in 8 bits
    float* rstd;       // NULL if not asked for
    uint8_t *q, *qs;   // codes [n][blocks * 128], scales [n][blocks rounded up to 4]
};

// 1 / sqrt(mean + eps) of a row from its sum of squares.  Where that overflows, `again` sums the squares of the elements times 2^kDown (65536 squares
// of 2^(128 - 74) stay below 2^124, and the mean of a sum that overflowed is above 2^(112 - 148)).  Squares below 2^-126 lose bits, 65536 of them at most
// 2^-134: nothing to a sum or an eps of 2^-100, else `again` sums the squares of the elements times 2^kUp, which lie between 2^-98 and 2^100.
constexpr int kDown = -74, kUp = 100;
constexpr float kFew = 0x1p-100f;
struct Root {
    float r, rstd;  // y = row * r * gamma (up: row * 2^kUp * r * gamma, since rstd is beyond fp32 for rows below 2^-128)
    bool up;
};
template <typename Again>
__device__ __forceinline__ Root rstd_of(float squares, float inv, float eps, Again again) {
    const bool up = squares < kFew && eps < kFew;
    if (up || squares > 3.4028234e38f) {
        const int k = up ? kUp : kDown;
        const float r = 1.f / sqrtf(again(k) * inv + ldexpf(eps, 2 * k)), rstd = ldexpf(r, k);  // infinite squares: 0
        return Root{up ? r : rstd, rstd, up};
    }
    const float r = 1.f / sqrtf(squares * inv + eps);
    return Root{r, r, false};
}

// A lane's V elements of a row in 8 bits: with the lanes of the same 128 elements, from column `col` on.
template <int V>
__device__ __forceinline__ void put_q8(const float (&v)[V], int col, int wide, uint8_t* q, uint8_t* qs) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) top = q8_larger(top, q8_size(v[i]));
    const uint32_t code = q8_scale(q8_top<kQ8Block / V>(top));
    if (col >= wide) return;
    uint32_t words[V / 4];
#pragma unroll
    for (int i = 0; i < V; i += 4) words[i / 4] = q8_codes(v[i], v[i + 1], v[i + 2], v[i + 3], code);
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q + col) = uint2{words[0], words[1]};
    else *reinterpret_cast<uint32_t*>(q + col) = words[0];
    if (col % kQ8Block == 0) {
        const int block = col / kQ8Block;
        qs[block] = (uint8_t)code;
        if (col + kQ8Block >= wide)
            for (int b = block + 1; b % 4; ++b) qs[b] = 127;  // the places behind the last block
    }
}

template <typename T, int V, int LANES, int P, bool ALIGNED, bool Q8>
__global__ __launch_bounds__(kBlock<LANES>) void rms_fwd_kernel(RmsFwd<T> a) {
    constexpr int kGroups = kBlock<LANES> / LANES;
    __shared__ float room[kReduceRoom<LANES>];
    int turn = 0;
    const int l = threadIdx.x % LANES, c = a.c;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
    if (row >= a.n) return;
    const int wide = (c + kQ8Block - 1) / kQ8Block * kQ8Block, scales = (wide / kQ8Block + 3) / 4 * 4;
    float ga[P][V];
    Piece<T, V> nx[P], nr[P];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * LANES + l) * V;
            if (col < c) {
                nx[p] = load_some<T, V, ALIGNED>(a.x + r * c + col, c - col);
                if (a.res) nr[p] = load_some<T, V, ALIGNED>(a.res + r * c + col, c - col);
            }
        }
    };
#pragma unroll
    for (int p = 0; p < P; ++p) {
        nx[p] = nr[p] = Piece<T, V>{};
#pragma unroll
        for (int i = 0; i < V; ++i) ga[p][i] = (p * LANES + l) * V + i < c ? a.gamma[(p * LANES + l) * V + i] : 0.f;
    }
    fetch(row);
    const float inv = 1.f / (float)c;
    for (; row < a.n; row += step) {
        float v[P][V], s[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            Piece<T, V> sum;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sum.e[i] = a.res ? to_elem<T>(elem(nx[p].e[i]) + elem(nr[p].e[i])) : nx[p].e[i];
                v[p][i] = elem(sum.e[i]);
                s[0] += v[p][i] * v[p][i];
            }
            const int col = (p * LANES + l) * V;
            if (a.res && col < c) store_some<T, V, ALIGNED>(a.h + row * c + col, sum, c - col);
        }
        if (row + step < a.n) fetch(row + step);
        reduce_lanes<LANES, Add>(s, room, &turn);
        const Root root = rstd_of(s[0], inv, a.eps, [&](int k) {
            float t[1] = {0.f};
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float f = ldexpf(v[p][i], k);
                    t[0] += f * f;
                    if (k > 0) v[p][i] = f;
                }
            reduce_lanes<LANES, Add>(t, room, &turn);
            return t[0];
        });
        const float r = root.r;
        if (l == 0 && a.rstd) a.rstd[row] = root.rstd;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * LANES + l) * V;
            if constexpr (Q8) {
#pragma unroll
                for (int i = 0; i < V; ++i) v[p][i] = col + i < c ? v[p][i] * r * ga[p][i] : 0.f;
                put_q8<V>(v[p], col, wide, a.q + row * wide, a.qs + row * scales);
            } else {
                Piece<T, V> o;
#pragma unroll
                for (int i = 0; i < V; ++i) o.e[i] = to_elem<T>(v[p][i] * r * ga[p][i]);
                if (col < c) store_some<T, V, ALIGNED>(a.y + row * c + col, o, c - col);
            }
        }
    }
}

// Rows too long for registers: a workgroup a row, read again (from cache) for the output.
constexpr int kWide = 1024;
template <typename T, int V, bool ALIGNED, bool Q8>
__global__ __launch_bounds__(kWide) void rms_fwd_wide_kernel(RmsFwd<T> a) {
    __shared__ float room[kReduceRoom<kWide>];
    int turn = 0;
    const int c = a.c, wide = (c + kQ8Block - 1) / kQ8Block * kQ8Block, scales = (wide / kQ8Block + 3) / 4 * 4;
    const float inv = 1.f / (float)c;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* from = a.res ? a.h + row * c : a.x + row * c;
        float s[1] = {0.f};
        for (int col = threadIdx.x * V; col < c; col += kWide * V) {
            Piece<T, V> v = load_some<T, V, ALIGNED>(a.x + row * c + col, c - col);
            if (a.res) {
                const Piece<T, V> o = load_some<T, V, ALIGNED>(a.res + row * c + col, c - col);
#pragma unroll
                for (int i = 0; i < V; ++i) v.e[i] = to_elem<T>(elem(v.e[i]) + elem(o.e[i]));
                store_some<T, V, ALIGNED>(a.h + row * c + col, v, c - col);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += elem(v.e[i]) * elem(v.e[i]);
        }
        reduce_lanes<kWide, Add>(s, room, &turn);
        const Root root = rstd_of(s[0], inv, a.eps, [&](int k) {
            float t[1] = {0.f};
            for (int j = threadIdx.x * V; j < c; j += kWide * V) {
                const Piece<T, V> v = load_some<T, V, ALIGNED>(from + j, c - j);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float f = ldexpf(elem(v.e[i]), k);
                    t[0] += f * f;
                }
            }
            reduce_lanes<kWide, Add>(t, room, &turn);
            return t[0];
        });
        const float r = root.r, up = root.up ? ldexpf(1.f, kUp) : 1.f;
        if (threadIdx.x == 0 && a.rstd) a.rstd[row] = root.rstd;
        // (the thread itself has written the piece of the sum that it reads)
        for (int col = threadIdx.x * V; col < (Q8 ? wide : c); col += kWide * V) {
            Piece<T, V> v{};
            if (col < c) v = load_some<T, V, ALIGNED>(from + col, c - col);
            if constexpr (Q8) {
                float f[V];
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = col + i < c ? elem(v.e[i]) * up * r * a.gamma[col + i] : 0.f;
                put_q8<V>(f, col, wide, a.q + row * wide, a.qs + row * scales);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) v.e[i] = col + i < c ? to_elem<T>(elem(v.e[i]) * up * r * a.gamma[col + i]) : T(0);
                store_some<T, V, ALIGNED>(a.y + row * c + col, v, c - col);
            }
        }
    }
}

template <typename T>
struct RmsBwd {
    const T *h, *dy, *dh;  // dh: NULL or the sum's own gradient
    int64_t n;
    int c;
    const float *gamma, *rstd;
    T* dx;
    float* partial;        // [workgroups][c], or NULL: dgamma comes from the rows themselves
};

template <typename T, int V, int LANES, int P, bool ALIGNED, bool PARTIAL>
__device__ __forceinline__ void rms_bwd_rows(const RmsBwd<T>& a, int blocks) {
    constexpr int kGroups = kBlock<LANES> / LANES;
    __shared__ float room[kReduceRoom<LANES>];
    __shared__ float sums[PARTIAL && kGroups > 1 ? kBlock<LANES> * V * P : 1];
    int turn = 0;
    const int l = threadIdx.x % LANES, c = a.c;
    const int64_t step = (int64_t)blocks * kGroups;
    int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
    float ga[P][V], dg[P][V];
    Piece<T, V> nh[P], nd[P], ns[P];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * LANES + l) * V;
            if (col < c) {
                nh[p] = load_some<T, V, ALIGNED>(a.h + r * c + col, c - col);
                nd[p] = load_some<T, V, ALIGNED>(a.dy + r * c + col, c - col);
                if (a.dh) ns[p] = load_some<T, V, ALIGNED>(a.dh + r * c + col, c - col);
            }
        }
    };
#pragma unroll
    for (int p = 0; p < P; ++p) {
        nh[p] = nd[p] = ns[p] = Piece<T, V>{};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            ga[p][i] = (p * LANES + l) * V + i < c ? a.gamma[(p * LANES + l) * V + i] : 0.f;
            dg[p][i] = 0.f;
        }
    }
    if (row < a.n) fetch(row);
    const float inv = 1.f / (float)c;
    for (; row < a.n; row += step) {
        const float r = a.rstd[row];
        float hat[P][V], g[P][V], own[P][V], s[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = elem(nd[p].e[i]);
                hat[p][i] = elem(nh[p].e[i]) * r;
                own[p][i] = elem(ns[p].e[i]);
                g[p][i] = d * ga[p][i];
                s[0] += g[p][i] * hat[p][i];
                dg[p][i] += d * hat[p][i];
            }
        if (row + step < a.n) fetch(row + step);
        reduce_lanes<LANES, Add>(s, room, &turn);
        const float m = s[0] * inv;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * LANES + l) * V;
            Piece<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) o.e[i] = to_elem<T>(own[p][i] + r * (g[p][i] - hat[p][i] * m));
            if (col < c) store_some<T, V, ALIGNED>(a.dx + row * c + col, o, c - col);
        }
    }
    if constexpr (!PARTIAL) return;
    float* out = a.partial + (size_t)blockIdx.x * c;
    if constexpr (kGroups > 1) {
        constexpr int kCols = LANES * V * P;  // [group][column], the groups added in order
        float* mine = sums + (threadIdx.x / LANES) * kCols;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) mine[(p * LANES + l) * V + i] = dg[p][i];
        __syncthreads();
        for (int t = threadIdx.x; t < kCols; t += kBlock<LANES>) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kGroups; ++k) s += sums[k * kCols + t];
            if (t < c) out[t] = s;
        }
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if ((p * LANES + l) * V + i < c) out[(p * LANES + l) * V + i] = dg[p][i];
    }
}

template <typename T, int V, int LANES, int P, bool ALIGNED>
__global__ __launch_bounds__(kBlock<LANES>) void rms_bwd_kernel(RmsBwd<T> a) {
    rms_bwd_rows<T, V, LANES, P, ALIGNED, true>(a, gridDim.x);
}

// dgamma of 4 V columns, straight from the rows: 64 rows at a time, 4 of a thread's asked for at once, its sums in fp32, those of the threads in fp64.
constexpr int kShort = 256;
template <typename T, int V, bool ALIGNED>
__device__ __forceinline__ void rms_bwd_columns(const RmsBwd<T>& a, int slab, float* dgamma) {
    constexpr int kSide = 4, kGroups = kShort / kSide, kAtOnce = 4;
    __shared__ float sums[kGroups][kSide * V + 1];
    const int group = threadIdx.x / kSide, at = threadIdx.x % kSide * V, col = slab * kSide * V + at, c = a.c;
    float dg[V] = {};
    if (col < c)
        for (int64_t row = group; row < a.n; row += kGroups * kAtOnce) {
            Piece<T, V> h[kAtOnce], d[kAtOnce];
            float r[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t from = min(row + kGroups * k, a.n - 1);
                h[k] = load_some<T, V, ALIGNED>(a.h + from * c + col, c - col);
                d[k] = load_some<T, V, ALIGNED>(a.dy + from * c + col, c - col);
                r[k] = a.rstd[from];
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (row + kGroups * k < a.n)
#pragma unroll
                    for (int i = 0; i < V; ++i) dg[i] += elem(d[k].e[i]) * (elem(h[k].e[i]) * r[k]);
        }
#pragma unroll
    for (int i = 0; i < V; ++i) sums[group][at + i] = dg[i];
    __syncthreads();
    const int t = threadIdx.x;
    if (t < kSide * V && slab * kSide * V + t < c) {
        double s = 0.0;
#pragma unroll 16
        for (int g = 0; g < kGroups; ++g) s += (double)sums[g][t];
        dgamma[slab * kSide * V + t] = (float)s;
    }
}
// A small matrix: the first `rows` workgroups take rows, the others columns, in one launch and without work memory.  (Two launches and a
// workgroup's parts: 1428 rows of 128 in bf16 24.5 us a forward and backward pass, most of it the host's.)
template <typename T, int V, int LANES, int P, bool ALIGNED>
__global__ __launch_bounds__(kShort) void rms_bwd_short_kernel(RmsBwd<T> a, int rows, float* dgamma) {
    if ((int)blockIdx.x < rows) rms_bwd_rows<T, V, LANES, P, ALIGNED, false>(a, rows);
    else rms_bwd_columns<T, V, ALIGNED>(a, blockIdx.x - rows, dgamma);
}
template <typename T, int V, bool ALIGNED>
__global__ __launch_bounds__(kShort) void rms_bwd_columns_kernel(RmsBwd<T> a, float* dgamma) {
    rms_bwd_columns<T, V, ALIGNED>(a, blockIdx.x, dgamma);
}

template <typename T>
__global__ __launch_bounds__(kWide) void rms_bwd_wide_kernel(RmsBwd<T> a) {
    __shared__ float room[kReduceRoom<kWide>];
    int turn = 0;
    const int c = a.c;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *h = a.h + row * c, *dy = a.dy + row * c;
        const float r = a.rstd[row];
        float s[1] = {0.f};
        for (int j = threadIdx.x; j < c; j += kWide) s[0] += elem(dy[j]) * a.gamma[j] * (elem(h[j]) * r);
        reduce_lanes<kWide, Add>(s, room, &turn);
        const float m = s[0] / (float)c;
        for (int j = threadIdx.x; j < c; j += kWide)
            a.dx[row * c + j] = to_elem<T>((a.dh ? elem(a.dh[row * c + j]) : 0.f) + r * (elem(dy[j]) * a.gamma[j] - elem(h[j]) * r * m));
    }
}

template <typename T>
__global__ __launch_bounds__(256) void rms_param_kernel(RmsBwd<T> a, int64_t slab) {
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= a.c) return;
    const int64_t r0 = blockIdx.y * slab, r1 = r0 + slab < a.n ? r0 + slab : a.n;
    float dg = 0.f;
    for (int64_t r = r0; r < r1; ++r) dg += elem(a.dy[r * a.c + col]) * (elem(a.h[r * a.c + col]) * a.rstd[r]);
    a.partial[(size_t)blockIdx.y * a.c + col] = dg;
}

// dgamma = the sums of `blocks` partial rows: a workgroup 16 columns, 64 rows at a time and 16 of a thread's asked for at once (one after another a
// load's way each was 9 us of 1024 rows of 77)
__global__ __launch_bounds__(1024) void rms_param_final_kernel(const float* __restrict__ partial, int blocks, int c, float* __restrict__ dgamma) {
    constexpr int kCols = 16, kGroups = 64, kAtOnce = 16;
    __shared__ double sums[kGroups][kCols + 1];
    const int at = blockIdx.x * kCols + threadIdx.x % kCols, group = threadIdx.x / kCols, col = min(at, c - 1);
    double s = 0.0;
    for (int b = group; b < blocks; b += kGroups * kAtOnce) {
        float v[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) v[i] = partial[(size_t)min(b + kGroups * i, blocks - 1) * c + col];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) s += b + kGroups * i < blocks ? (double)v[i] : 0.0;
    }
    sums[group][threadIdx.x % kCols] = s;
    __syncthreads();
    if (group == 0 && at < c) {
        double t = 0.0;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) t += sums[i][threadIdx.x];
        dgamma[at] = (float)t;
    }
}

// The lanes and pieces a lane that hold `pieces` pieces of a row, at least `least` lanes (those of 128 elements, in 8 bits); 0: none do.
struct Shape {
    int lanes, per;
};
Shape shape_of(int64_t pieces, int v, int least, bool backward) {
    for (const Shape s : {Shape{8, 1}, Shape{16, 1}, Shape{32, 1}, Shape{64, 1}, Shape{64, 2}, Shape{256, 1}, Shape{256, 2}})
        if (s.lanes >= least && pieces <= (int64_t)s.lanes * s.per) return s;
    if (v == 4) {
        for (const Shape s : {Shape{256, 4}, Shape{512, 4}})
            if (pieces <= (int64_t)s.lanes * s.per) return s;
    } else {
        if (pieces <= 1024) return Shape{512, 2};
        if (pieces <= 2048 && !backward) return Shape{1024, 2};  // a workgroup of 1024 has no registers for the backward pass of two pieces
    }
    return Shape{0, 0};
}
// f(std::integral_constant lanes, pieces a lane)
template <int V, bool BACK, typename F>
int with_shape(Shape s, F f) {
#define SP_SHAPE(L, P) \
    if (s.lanes == L && s.per == P) return f(std::integral_constant<int, L>{}, std::integral_constant<int, P>{})
    SP_SHAPE(8, 1);
    SP_SHAPE(16, 1);
    SP_SHAPE(32, 1);
    SP_SHAPE(64, 1);
    SP_SHAPE(64, 2);
    SP_SHAPE(256, 1);
    SP_SHAPE(256, 2);
    if constexpr (V == 4) {
        SP_SHAPE(256, 4);
        SP_SHAPE(512, 4);
    } else {
        SP_SHAPE(512, 2);
        if constexpr (!BACK) SP_SHAPE(1024, 2);
    }
#undef SP_SHAPE
    return fail(SP_ERR_UNSUPPORTED, "no kernel for this width");
}
int rows_of(int lanes) { return std::max(lanes, 256) / lanes; }  // of a workgroup at a time

int fwd_blocks(int64_t n, Shape s, int v) {
    return (int)std::min<int64_t>((n + rows_of(s.lanes) - 1) / rows_of(s.lanes), s.lanes > 256 ? 512 : s.per * v > 8 ? 1024 : 2048);
}
int bwd_blocks(int64_t n, Shape s, int v) {
    return (int)std::min<int64_t>((n + rows_of(s.lanes) - 1) / rows_of(s.lanes), s.lanes > 256 ? 256 : s.per * v > 8 ? 256 : 1024);
}
constexpr int kMostSlabs = 256;
int64_t slab_of(int64_t n) { return std::max<int64_t>(64, (n + kMostSlabs - 1) / kMostSlabs); }

// Reading h and dy again for dgamma costs less than a launch
bool short_rows(int64_t n, int c, Shape s) { return n > 0 && s.lanes && s.lanes <= kShort && n <= 4096 && n * c <= (1 << 18); }

template <typename T, bool ALIGNED, bool Q8>
int rms_fwd(const RmsFwd<T>& a, hipStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    const Shape shape = shape_of((a.c + V - 1) / V, V, Q8 ? kQ8Block / V : 1, false);
    if (!shape.lanes) {
        hipLaunchKernelGGL((rms_fwd_wide_kernel<T, V, ALIGNED, Q8>), dim3((unsigned)std::min<int64_t>(a.n, 512)), dim3(kWide), 0, s, a);
        SP_HIP(hipGetLastError());
        return SP_OK;
    }
    return with_shape<V, false>(shape, [&](auto lanes, auto per) -> int {
        constexpr int L = decltype(lanes)::value, P = decltype(per)::value;
        if constexpr (!Q8 || L >= kQ8Block / V) {
            hipLaunchKernelGGL((rms_fwd_kernel<T, V, L, P, ALIGNED, Q8>), dim3(fwd_blocks(a.n, shape, V)), dim3(kBlock<L>), 0, s, a);
            SP_HIP(hipGetLastError());
            return SP_OK;
        }
        return fail(SP_ERR_UNSUPPORTED, "no kernel for this width");
    });
}

template <typename T, bool ALIGNED>
int rms_bwd(RmsBwd<T> a, float* dgamma, hipStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    const Shape shape = shape_of((a.c + V - 1) / V, V, 1, true);
    int blocks;
    if (short_rows(a.n, a.c, shape)) {
        const int rows = bwd_blocks(a.n, shape, V), columns = (a.c + 4 * V - 1) / (4 * V);
        const bool same = (const void*)a.dy == (const void*)a.dx;  // dgamma first
        if (same) hipLaunchKernelGGL((rms_bwd_columns_kernel<T, V, ALIGNED>), dim3(columns), dim3(kShort), 0, s, a, dgamma);
        SP_TRY((with_shape<V, true>(shape, [&](auto lanes, auto per) -> int {
            constexpr int L = decltype(lanes)::value, P = decltype(per)::value;
            if constexpr (L <= kShort) {
                hipLaunchKernelGGL((rms_bwd_short_kernel<T, V, L, P, ALIGNED>), dim3(rows + (same ? 0 : columns)), dim3(kShort), 0, s, a, rows, dgamma);
                return SP_OK;
            }
            return fail(SP_ERR_UNSUPPORTED, "no kernel for this width");
        })));
        SP_HIP(hipGetLastError());
        return SP_OK;
    }
    if (a.n == 0) {
        blocks = 0;
    } else if (!shape.lanes) {
        const int64_t slab = slab_of(a.n);
        blocks = (int)((a.n + slab - 1) / slab);
        // before dx, which may be dy's memory
        hipLaunchKernelGGL(rms_param_kernel<T>, dim3((a.c + 255) / 256, blocks), dim3(256), 0, s, a, slab);
        hipLaunchKernelGGL(rms_bwd_wide_kernel<T>, dim3((unsigned)std::min<int64_t>(a.n, 512)), dim3(kWide), 0, s, a);
    } else {
        blocks = bwd_blocks(a.n, shape, V);
        SP_TRY((with_shape<V, true>(shape, [&](auto lanes, auto per) -> int {
            constexpr int L = decltype(lanes)::value, P = decltype(per)::value;
            hipLaunchKernelGGL((rms_bwd_kernel<T, V, L, P, ALIGNED>), dim3(blocks), dim3(kBlock<L>), 0, s, a);
            return SP_OK;
        })));
    }
    hipLaunchKernelGGL(rms_param_final_kernel, dim3((a.c + 15) / 16), dim3(1024), 0, s, a.partial, blocks, a.c, dgamma);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

int check(int64_t n, int c, sp_dtype dt) {
    if (n < 0 || n > (int64_t)1 << 40 || c < 1 || c > 65536) return fail(SP_ERR_INVALID_ARG, "bad row or channel count");
    if (dt != SP_F32 && dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    return SP_OK;
}

template <typename T>
int rms_fwd_typed(const RmsFwd<T>& a, hipStream_t s) {
    bool aligned = a.c % (16 / (int)sizeof(T)) == 0;
    for (const void* p : {(const void*)a.x, (const void*)a.res, (const void*)a.h, (const void*)a.y}) aligned &= aligned16(p);
    if (a.q) return aligned ? rms_fwd<T, true, true>(a, s) : rms_fwd<T, false, true>(a, s);
    return aligned ? rms_fwd<T, true, false>(a, s) : rms_fwd<T, false, false>(a, s);
}

int rms_fwd_any(const void* d_x, const void* d_res, int64_t n, int32_t c, const float* d_gamma, float eps, void* d_h, void* d_y, float* d_rstd,
                uint8_t* d_q, uint8_t* d_qs, sp_dtype dt, hipStream_t s) {
    if (!(eps >= 0.f)) return fail(SP_ERR_INVALID_ARG, "eps must not be negative");
    if (d_res && !d_h) return fail(SP_ERR_INVALID_ARG, "the sum with the residual needs a place");
    if (!d_res && d_h) return fail(SP_ERR_INVALID_ARG, "without a residual there is no sum to store");
    if (d_y && (d_y == d_h)) return fail(SP_ERR_INVALID_ARG, "y and the sum need a place each");
    if (n == 0) return SP_OK;
    if (dt == SP_F32)
        return rms_fwd_typed(RmsFwd<float>{(const float*)d_x, (const float*)d_res, n, c, d_gamma, eps, (float*)d_h, (float*)d_y, d_rstd, d_q, d_qs}, s);
    return rms_fwd_typed(RmsFwd<bf16_t>{(const bf16_t*)d_x, (const bf16_t*)d_res, n, c, d_gamma, eps, (bf16_t*)d_h, (bf16_t*)d_y, d_rstd, d_q, d_qs}, s);
}

template <typename T>
int rms_bwd_typed(const RmsBwd<T>& a, float* dgamma, hipStream_t s) {
    bool aligned = a.c % (16 / (int)sizeof(T)) == 0;
    for (const void* p : {(const void*)a.h, (const void*)a.dy, (const void*)a.dh, (const void*)a.dx}) aligned &= aligned16(p);
    return aligned ? rms_bwd<T, true>(a, dgamma, s) : rms_bwd<T, false>(a, dgamma, s);
}

// Rows in 8 bits as they are, and the rows of the transposed matrix, each 128 of its elements from 128 rows of x.
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void q8_rows_kernel(const T* __restrict__ x, int64_t ldx, int64_t n, int c, uint8_t* q, uint8_t* qs) {
    constexpr int V = 16 / (int)sizeof(T), kLanes = kQ8Block / V;
    const int wide = (c + kQ8Block - 1) / kQ8Block * kQ8Block, scales = (wide / kQ8Block + 3) / 4 * 4;
    // a workgroup: 256 / kLanes blocks of 128 elements, one row's or several rows'
    const int64_t blocks_row = wide / kQ8Block, all = n * blocks_row;
    for (int64_t b = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes; b < all; b += (int64_t)gridDim.x * (256 / kLanes)) {
        const int64_t row = all < ((int64_t)1 << 32) ? (int64_t)((uint32_t)b / (uint32_t)blocks_row) : b / blocks_row;
        const int col = (int)(b - row * blocks_row) * kQ8Block + (threadIdx.x % kLanes) * V;
        Piece<T, V> v{};
        if (col < c) v = load_some<T, V, ALIGNED>(x + row * ldx + col, c - col);
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = elem(v.e[i]);
        put_q8<V>(f, col, wide, q + row * wide, qs + row * scales);
    }
}

// A workgroup: 128 rows and 64 columns of x, through LDS as they are stored, so that of bf16 eight workgroups share a CU (8192 x 2048: 11.5 us, 4.4 TB/s;
// four of them, with 32 bits an element: 14.5).
constexpr int kTurnCols = 64;
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void q8_turned_kernel(const T* __restrict__ x, int64_t ldx, int64_t n, int c, int64_t first, uint8_t* q, uint8_t* qs) {
    constexpr int V = 16 / (int)sizeof(T), kPieces = kTurnCols / V, kEach = kQ8Block * kPieces / 256;
    constexpr int kPad = 4 / (int)sizeof(T);  // a column is an odd number of banks behind the last
    __shared__ __attribute__((aligned(4))) T tile[kTurnCols][kQ8Block + kPad];
    const int64_t blocks = (n + kQ8Block - 1) / kQ8Block, wide = blocks * kQ8Block, scales = (blocks + 3) / 4 * 4;
    const int64_t block = first + blockIdx.x, row0 = block * kQ8Block;
    const int col0 = blockIdx.y * kTurnCols;
    Piece<T, V> in[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = k * 256 + threadIdx.x, r = i / kPieces, j = (i % kPieces) * V;
        in[k] = Piece<T, V>{};
        if (row0 + r < n && col0 + j < c) in[k] = load_some<T, V, ALIGNED>(x + (row0 + r) * ldx + col0 + j, c - col0 - j);
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = k * 256 + threadIdx.x, r = i / kPieces, j = (i % kPieces) * V;
#pragma unroll
        for (int e = 0; e < V; ++e) tile[j + e][r] = in[k].e[e];
    }
    __syncthreads();
    // four lanes a column, 32 rows each; of fp32, lanes 2 and 3 begin at the second 16, since they share banks with lanes 0 and 1
    const int j = threadIdx.x / 4, part = threadIdx.x % 4, swap = sizeof(T) == 4 ? part >> 1 : 0;
    float v[32], top = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v[i] = elem(tile[j][part * 32 + (i ^ (swap << 4))]);
        top = q8_larger(top, q8_size(v[i]));
    }
    const uint32_t code = q8_scale(q8_top<4>(top));
    if (col0 + j >= c) return;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = q8_codes(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], code);
    uint4* to = reinterpret_cast<uint4*>(q + (int64_t)(col0 + j) * wide + row0 + part * 32);
    to[swap] = uint4{w[0], w[1], w[2], w[3]};
    to[swap ^ 1] = uint4{w[4], w[5], w[6], w[7]};
    if (part == 0) {
        uint8_t* s = qs + (int64_t)(col0 + j) * scales;
        s[block] = (uint8_t)code;
        if (block + 1 == blocks)
            for (int64_t b = blocks; b < scales; ++b) s[b] = 127;
    }
}

template <typename T>
int q8_rows(const T* x, int64_t ldx, int64_t n, int c, bool transposed, uint8_t* q, uint8_t* qs, hipStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool aligned = aligned16(x) && c % V == 0 && (ldx % V == 0 || n == 1);
    if (transposed) {
        // A launch of 2^32 threads or more is cut short without an error.
        constexpr int64_t kMost = 1 << 22;
        for (int64_t first = 0, blocks = q8_blocks(n); first < blocks; first += kMost) {
            const dim3 grid((unsigned)std::min(kMost, blocks - first), (unsigned)((c + kTurnCols - 1) / kTurnCols));
            if (aligned) hipLaunchKernelGGL((q8_turned_kernel<T, true>), grid, dim3(256), 0, s, x, ldx, n, c, first, q, qs);
            else hipLaunchKernelGGL((q8_turned_kernel<T, false>), grid, dim3(256), 0, s, x, ldx, n, c, first, q, qs);
        }
    } else {
        const int64_t each = 256 / (kQ8Block / V), want = (n * q8_blocks(c) + each - 1) / each;
        const dim3 grid((unsigned)std::min<int64_t>(want, 8192));
        if (aligned) hipLaunchKernelGGL((q8_rows_kernel<T, true>), grid, dim3(256), 0, s, x, ldx, n, c, q, qs);
        else hipLaunchKernelGGL((q8_rows_kernel<T, false>), grid, dim3(256), 0, s, x, ldx, n, c, q, qs);
    }
    SP_HIP(hipGetLastError());
    return SP_OK;
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" {

int sp_rms_norm_fwd(const void* d_x, const void* d_res, int64_t n, int32_t c, const float* d_gamma, float eps, void* d_h, void* d_y,
                    float* d_rstd, sp_dtype dt, void* stream) {
    SP_TRY(check(n, c, dt));
    if (!d_gamma || (n > 0 && (!d_x || !d_y || !d_rstd))) return fail(SP_ERR_INVALID_ARG, "a feature/parameter/statistics pointer is NULL");
    return rms_fwd_any(d_x, d_res, n, c, d_gamma, eps, d_h, d_y, d_rstd, nullptr, nullptr, dt, (hipStream_t)stream);
}

int sp_rms_norm_q8(const void* d_x, const void* d_res, int64_t n, int32_t c, const float* d_gamma, float eps, void* d_h, uint8_t* d_q,
                   uint8_t* d_scales, sp_dtype dt, void* stream) {
    SP_TRY(check(n, c, dt));
    if (!d_gamma || (n > 0 && (!d_x || !d_q || !d_scales))) return fail(SP_ERR_INVALID_ARG, "a feature/parameter/code pointer is NULL");
    if (!aligned16(d_q)) return fail(SP_ERR_INVALID_ARG, "codes must be 16-byte aligned");
    return rms_fwd_any(d_x, d_res, n, c, d_gamma, eps, d_h, nullptr, nullptr, d_q, d_scales, dt, (hipStream_t)stream);
}

int64_t sp_rms_norm_bwd_work(int64_t n, int32_t c, sp_dtype dt) {
    if (check(n, c, dt) != SP_OK) return -1;
    const int v = dt == SP_F32 ? 4 : 8;
    const Shape shape = shape_of((c + v - 1) / v, v, 1, true);
    if (n == 0 || short_rows(n, c, shape)) return 256;
    return std::max<int64_t>(512, (int64_t)(shape.lanes ? bwd_blocks(n, shape, v) : kMostSlabs) * c * 4);
}

int sp_rms_norm_bwd(const void* d_h, const void* d_dy, const void* d_dh, int64_t n, int32_t c, const float* d_gamma, const float* d_rstd,
                    void* d_dx, float* d_dgamma, void* d_work, sp_dtype dt, void* stream) {
    SP_TRY(check(n, c, dt));
    if (!d_gamma || !d_dgamma || (n > 0 && (!d_h || !d_dy || !d_dx || !d_rstd || !d_work)))
        return fail(SP_ERR_INVALID_ARG, "a feature/parameter/gradient/work pointer is NULL");
    float* work = static_cast<float*>(d_work);
    if (dt == SP_F32)
        return rms_bwd_typed(RmsBwd<float>{(const float*)d_h, (const float*)d_dy, (const float*)d_dh, n, c, d_gamma, d_rstd, (float*)d_dx, work},
                             d_dgamma, (hipStream_t)stream);
    return rms_bwd_typed(RmsBwd<bf16_t>{(const bf16_t*)d_h, (const bf16_t*)d_dy, (const bf16_t*)d_dh, n, c, d_gamma, d_rstd, (bf16_t*)d_dx, work},
                         d_dgamma, (hipStream_t)stream);
}

int64_t sp_q8_codes_bytes(int64_t n, int64_t c) {
    int64_t bytes;
    if (n < 0 || c < 1 || n > (int64_t)1 << 40 || c > (int64_t)1 << 40 || __builtin_mul_overflow(n, q8_blocks(c) * kQ8Block, &bytes)) return -1;
    return bytes;
}
int64_t sp_q8_scales_bytes(int64_t n, int64_t c) {
    int64_t bytes;
    if (n < 0 || c < 1 || n > (int64_t)1 << 40 || c > (int64_t)1 << 40 || __builtin_mul_overflow(n, q8_scales(c), &bytes)) return -1;
    return bytes;
}

int sp_q8_rows(const void* d_x, int64_t ldx, int64_t n, int32_t c, int32_t transposed, uint8_t* d_q, uint8_t* d_scales, sp_dtype dt, void* stream) {
    if (n < 0 || n > (int64_t)1 << 40 || c < 1 || c > 1 << 22) return fail(SP_ERR_INVALID_ARG, "bad row or channel count");
    if (dt != SP_F32 && dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (ldx < c) return fail(SP_ERR_INVALID_ARG, "rows overlap");
    if (n == 0) return SP_OK;  // (transposed, rows of no elements have no codes)
    if (!d_x || !d_q || !d_scales) return fail(SP_ERR_INVALID_ARG, "a feature or code pointer is NULL");
    if (!aligned16(d_q)) return fail(SP_ERR_INVALID_ARG, "codes must be 16-byte aligned");
    if (dt == SP_F32) return q8_rows((const float*)d_x, ldx, n, c, transposed != 0, d_q, d_scales, (hipStream_t)stream);
    return q8_rows((const bf16_t*)d_x, ldx, n, c, transposed != 0, d_q, d_scales, (hipStream_t)stream);
}

}  // extern "C"
