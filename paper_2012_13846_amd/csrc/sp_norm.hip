// Layer normalisation of the rows of a feature matrix, forward and backward with the gradients of weight and bias.
//
// Memory bound: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx, each once.  A row stays in
// the registers of the LANES threads that share it (8 lanes to a workgroup of 1024, by the row's length), so its statistics take no
// second read; the next row is asked for before this one is reduced.  The variance is that of d = x - m with m the row's fp32 mean,
// and m is corrected by the mean of d: as good where the mean is large against the spread.  The parameters' gradients are summed in
// the registers of the lanes that own the columns, over all rows of a workgroup (the grid is no larger than the chip's fill), then
// over its row groups through LDS, and the workgroups' partial sums are added in fp64 in a fixed order by a second kernel.
// Rows that no workgroup can hold (more than 16 elements a thread of 1024) are read again from cache for every statistic.
// Measured: 373601 x 256 bf16 forward 80 - 86 us (4.5 - 4.8 TB/s; a large copy 5.0 - 6.3), backward 114 - 117 + 5 (4.9 - 5.0); 16384 x 4096
// 54 - 56 (4.8) and 86 - 88 + 5 (4.6).
#include <algorithm>

#include "sp_elem.h"

namespace sp {
namespace {

template <int LANES>
constexpr int kBlock = LANES > 256 ? LANES : 256;

// A row with an infinity or NaN has neither spread nor scale: NaN, which a maximum with zero would lose.  Its mean is its sum's.
__device__ __forceinline__ float rstd_of(float var, float eps) { return 1.f / sqrtf((var < 0.f ? 0.f : var) + eps); }
__device__ __forceinline__ float mean_of(float m0, float delta) { return delta == delta ? m0 + delta : m0; }

template <typename T, int V, int LANES, int P>
__global__ __launch_bounds__(kBlock<LANES>) void layer_norm_fwd_kernel(const T* __restrict__ x, int64_t n, int c,
                                                                       const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                       float eps, T* __restrict__ y, float* __restrict__ mean,
                                                                       float* __restrict__ rstd) {
    constexpr int kGroups = kBlock<LANES> / LANES;
    __shared__ float room[kReduceRoom<LANES>];
    int turn = 0;
    const int l = threadIdx.x % LANES;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
    if (row >= n) return;
    float ga[P][V], be[P][V];
    Piece<T, V> next[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int col = (p * LANES + l) * V;
        next[p] = Piece<T, V>{};
        if (col < c) next[p] = load_piece<T, V>(x + row * c + col);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            ga[p][i] = col < c ? gamma[col + i] : 0.f;
            be[p][i] = col < c ? beta[col + i] : 0.f;
        }
    }
    const float inv = 1.f / (float)c;
    for (; row < n; row += step) {
        float v[P][V], s[1] = {0.f}, q[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += v[p][i] = elem(next[p].e[i]);
        if (row + step < n)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int col = (p * LANES + l) * V;
                if (col < c) next[p] = load_piece<T, V>(x + (row + step) * c + col);
            }
        reduce_lanes<LANES, Add>(s, room, &turn);
        const float m0 = s[0] * inv;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = (p * LANES + l) * V < c ? v[p][i] - m0 : 0.f;
                v[p][i] = d;
                q[0] += d;
                q[1] += d * d;
            }
        reduce_lanes<LANES, Add>(q, room, &turn);
        const float delta = q[0] * inv;
        const float r = rstd_of(q[1] * inv - delta * delta, eps);
        if (l == 0) {
            mean[row] = mean_of(m0, delta);
            rstd[row] = r;
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * LANES + l) * V;
            Piece<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) o.e[i] = to_elem<T>((v[p][i] - delta) * r * ga[p][i] + be[p][i]);
            if (col < c) store_piece<T, V>(y + row * c + col, o);
        }
    }
}

// partial[workgroup][0][c] = sum over its rows of dy * xhat, [1][c] = of dy
template <typename T, int V, int LANES, int P>
__global__ __launch_bounds__(kBlock<LANES>) void layer_norm_bwd_kernel(const T* __restrict__ x, const T* dy, int64_t n, int c,
                                                                       const float* __restrict__ gamma, const float* __restrict__ mean,
                                                                       const float* __restrict__ rstd, T* dx, float* __restrict__ partial) {
    constexpr int kGroups = kBlock<LANES> / LANES;
    __shared__ float room[kReduceRoom<LANES>];
    __shared__ float sums[kGroups > 1 ? 2 * kBlock<LANES> * V * P : 1];
    int turn = 0;
    const int l = threadIdx.x % LANES;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
    float ga[P][V], dg[P][V], db[P][V];
    Piece<T, V> nx[P], nd[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int col = (p * LANES + l) * V;
        nx[p] = nd[p] = Piece<T, V>{};
        if (row < n && col < c) {
            nx[p] = load_piece<T, V>(x + row * c + col);
            nd[p] = load_piece<T, V>(dy + row * c + col);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            ga[p][i] = col < c ? gamma[col + i] : 0.f;
            dg[p][i] = db[p][i] = 0.f;
        }
    }
    const float inv = 1.f / (float)c;
    for (; row < n; row += step) {
        const float m = mean[row], r = rstd[row];
        float xh[P][V], g[P][V], s[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool in = (p * LANES + l) * V < c;
                const float d = elem(nd[p].e[i]);
                xh[p][i] = in ? (elem(nx[p].e[i]) - m) * r : 0.f;
                g[p][i] = d * ga[p][i];
                s[0] += g[p][i];
                s[1] += g[p][i] * xh[p][i];
                dg[p][i] += d * xh[p][i];
                db[p][i] += d;
            }
        if (row + step < n)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int col = (p * LANES + l) * V;
                if (col < c) {
                    nx[p] = load_piece<T, V>(x + (row + step) * c + col);
                    nd[p] = load_piece<T, V>(dy + (row + step) * c + col);
                }
            }
        reduce_lanes<LANES, Add>(s, room, &turn);
        const float a = s[0] * inv, b = s[1] * inv;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * LANES + l) * V;
            Piece<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) o.e[i] = to_elem<T>(r * (g[p][i] - a - xh[p][i] * b));
            if (col < c) store_piece<T, V>(dx + row * c + col, o);
        }
    }
    float* out = partial + (size_t)blockIdx.x * 2 * c;
    if constexpr (kGroups > 1) {
        // [group][value][column], the groups added in order
        constexpr int kCols = LANES * V * P;
        float* mine = sums + (threadIdx.x / LANES) * 2 * kCols;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                mine[(p * LANES + l) * V + i] = dg[p][i];
                mine[kCols + (p * LANES + l) * V + i] = db[p][i];
            }
        __syncthreads();
        for (int t = threadIdx.x; t < 2 * kCols; t += kBlock<LANES>) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kGroups; ++k) s += sums[k * 2 * kCols + t];
            const int q = t / kCols, col = t % kCols;
            if (col < c) out[q * c + col] = s;
        }
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * LANES + l) * V;
            if (col < c)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    out[col + i] = dg[p][i];
                    out[c + col + i] = db[p][i];
                }
        }
    }
}

// Rows too long for registers: a workgroup a row, every statistic a pass over it (the passes after the first hit the caches).
constexpr int kWide = 1024;
template <typename T>
__global__ __launch_bounds__(kWide) void layer_norm_fwd_wide_kernel(const T* __restrict__ x, int64_t n, int c,
                                                                    const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                    float eps, T* __restrict__ y, float* __restrict__ mean,
                                                                    float* __restrict__ rstd) {
    __shared__ float room[kReduceRoom<kWide>];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* xr = x + row * c;
        float s[1] = {0.f}, q[2] = {0.f, 0.f};
        for (int j = threadIdx.x; j < c; j += kWide) s[0] += elem(xr[j]);
        reduce_lanes<kWide, Add>(s, room, &turn);
        const float m0 = s[0] / (float)c;
        for (int j = threadIdx.x; j < c; j += kWide) {
            const float d = elem(xr[j]) - m0;
            q[0] += d;
            q[1] += d * d;
        }
        reduce_lanes<kWide, Add>(q, room, &turn);
        const float delta = q[0] / (float)c;
        const float r = rstd_of(q[1] / (float)c - delta * delta, eps);
        if (threadIdx.x == 0) {
            mean[row] = mean_of(m0, delta);
            rstd[row] = r;
        }
        for (int j = threadIdx.x; j < c; j += kWide) y[row * c + j] = to_elem<T>((elem(xr[j]) - m0 - delta) * r * gamma[j] + beta[j]);
    }
}

template <typename T>
__global__ __launch_bounds__(kWide) void layer_norm_bwd_wide_kernel(const T* __restrict__ x, const T* dy, int64_t n, int c,
                                                                    const float* __restrict__ gamma, const float* __restrict__ mean,
                                                                    const float* __restrict__ rstd, T* dx) {
    __shared__ float room[kReduceRoom<kWide>];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T *xr = x + row * c, *dr = dy + row * c;
        const float m = mean[row], r = rstd[row];
        float s[2] = {0.f, 0.f};
        for (int j = threadIdx.x; j < c; j += kWide) {
            const float g = elem(dr[j]) * gamma[j];
            s[0] += g;
            s[1] += g * ((elem(xr[j]) - m) * r);
        }
        reduce_lanes<kWide, Add>(s, room, &turn);
        const float a = s[0] / (float)c, b = s[1] / (float)c;
        for (int j = threadIdx.x; j < c; j += kWide)
            dx[row * c + j] = to_elem<T>(r * (elem(dr[j]) * gamma[j] - a - (elem(xr[j]) - m) * r * b));
    }
}

constexpr int kSlab = 64;  // rows of one partial sum
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_param_kernel(const T* __restrict__ x, const T* __restrict__ dy, int64_t n, int c,
                                                               const float* __restrict__ mean, const float* __restrict__ rstd,
                                                               int64_t slab, float* __restrict__ partial) {
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= c) return;
    const int64_t r0 = blockIdx.y * slab, r1 = r0 + slab < n ? r0 + slab : n;
    float dg = 0.f, db = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        const float d = elem(dy[r * c + col]);
        dg += d * ((elem(x[r * c + col]) - mean[r]) * rstd[r]);
        db += d;
    }
    partial[(size_t)blockIdx.y * 2 * c + col] = dg;
    partial[((size_t)blockIdx.y * 2 + 1) * c + col] = db;
}

// dgamma / dbeta = the sums of `blocks` partial rows of 2 c values: 32 columns and 32 rows at a time
__global__ __launch_bounds__(1024) void layer_norm_param_final_kernel(const float* __restrict__ partial, int blocks, int c,
                                                                      float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ double sums[32][33];
    const int at = blockIdx.x * 32 + (threadIdx.x & 31), group = threadIdx.x >> 5;
    double s = 0.0;
    if (at < 2 * c) {
        int b = group;
        for (; b + 96 < blocks; b += 128) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = partial[(size_t)(b + 32 * i) * 2 * c + at];
#pragma unroll
            for (int i = 0; i < 4; ++i) s += (double)v[i];
        }
        for (; b < blocks; b += 32) s += (double)partial[(size_t)b * 2 * c + at];
    }
    sums[group][threadIdx.x & 31] = s;
    __syncthreads();
    if (group == 0 && at < 2 * c) {
        double t = 0.0;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sums[i][threadIdx.x];
        if (at < c) dgamma[at] = (float)t;
        else dbeta[at - c] = (float)t;
    }
}

struct NormArgs {
    const void *x, *dy;
    int64_t n;
    int c;
    const float *gamma, *beta;
    float eps;
    void* out;  // y or dx
    float *mean, *rstd, *dgamma, *dbeta;
    hipStream_t s;
};

int param_final(const NormArgs& a, const float* partial, int blocks) {
    hipLaunchKernelGGL(layer_norm_param_final_kernel, dim3((2 * a.c + 31) / 32), dim3(1024), 0, a.s, partial, blocks, a.c, a.dgamma, a.dbeta);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T, int V, int LANES, int P>
int norm_rows(const NormArgs& a) {
    constexpr int kGroups = kBlock<LANES> / LANES;
    const int64_t want = (a.n + kGroups - 1) / kGroups;
    if (!a.dy) {
        // Enough workgroups to fill the chip, and no more: each loads the parameters.  us for forward and backward in bf16, 1024 / 2048 /
        // 4096 workgroups here: 16384 x 4096 148 / 155 / 198, 373601 x 256 222 / 206 / 207; 512 / 1024 / 2048: 8000 x 8192 153 / 172 / 208.
        const unsigned blocks = (unsigned)std::min<int64_t>(want, LANES > 256 ? 512 : P * V > 8 ? 1024 : 2048);
        hipLaunchKernelGGL((layer_norm_fwd_kernel<T, V, LANES, P>), dim3(blocks), dim3(kBlock<LANES>), 0, a.s, static_cast<const T*>(a.x), a.n,
                           a.c, a.gamma, a.beta, a.eps, static_cast<T*>(a.out), a.mean, a.rstd);
        SP_HIP(hipGetLastError());
        return SP_OK;
    }
    const int blocks = (int)std::min<int64_t>(want, LANES > 256 ? 256 : P * V > 8 ? 512 : 1024);
    Buf partial = dev_alloc((size_t)blocks * 2 * a.c * 4, a.s);
    if (!partial) return SP_ERR_ALLOC;
    hipLaunchKernelGGL((layer_norm_bwd_kernel<T, V, LANES, P>), dim3(blocks), dim3(kBlock<LANES>), 0, a.s, static_cast<const T*>(a.x),
                       static_cast<const T*>(a.dy), a.n, a.c, a.gamma, a.mean, a.rstd, static_cast<T*>(a.out), ptr<float>(partial));
    return param_final(a, ptr<float>(partial), blocks);
}

template <typename T>
int norm_wide(const NormArgs& a) {
    const unsigned rows = (unsigned)std::min<int64_t>(a.n, 512);
    if (!a.dy) {
        hipLaunchKernelGGL(layer_norm_fwd_wide_kernel<T>, dim3(rows), dim3(kWide), 0, a.s, static_cast<const T*>(a.x), a.n, a.c, a.gamma,
                           a.beta, a.eps, static_cast<T*>(a.out), a.mean, a.rstd);
        SP_HIP(hipGetLastError());
        return SP_OK;
    }
    const int64_t slab = std::max<int64_t>(kSlab, (a.n + 255) / 256);
    const int blocks = (int)((a.n + slab - 1) / slab);
    Buf partial = dev_alloc((size_t)blocks * 2 * a.c * 4, a.s);
    if (!partial) return SP_ERR_ALLOC;
    // before dx, which may be dy's memory
    hipLaunchKernelGGL(layer_norm_param_kernel<T>, dim3((a.c + 255) / 256, blocks), dim3(256), 0, a.s, static_cast<const T*>(a.x),
                       static_cast<const T*>(a.dy), a.n, a.c, a.mean, a.rstd, slab, ptr<float>(partial));
    hipLaunchKernelGGL(layer_norm_bwd_wide_kernel<T>, dim3(rows), dim3(kWide), 0, a.s, static_cast<const T*>(a.x),
                       static_cast<const T*>(a.dy), a.n, a.c, a.gamma, a.mean, a.rstd, static_cast<T*>(a.out));
    return param_final(a, ptr<float>(partial), blocks);
}

// Rows of single elements (a width that is no whole number of 16-byte pieces): exactly as many steps of 16, 32 or 64 lanes as it takes,
// at most 8: 200000 x 77 in bf16 82 -> 48 us against 64 lanes with two steps, the second a fifth full.
template <typename T, int LANES>
int norm_steps(const NormArgs& a) {
    switch ((a.c + LANES - 1) / LANES) {
        case 1: return norm_rows<T, 1, LANES, 1>(a);
        case 2: return norm_rows<T, 1, LANES, 2>(a);
        case 3: return norm_rows<T, 1, LANES, 3>(a);
        case 4: return norm_rows<T, 1, LANES, 4>(a);
        case 5: return norm_rows<T, 1, LANES, 5>(a);
        case 6: return norm_rows<T, 1, LANES, 6>(a);
        case 7: return norm_rows<T, 1, LANES, 7>(a);
        default: return norm_rows<T, 1, LANES, 8>(a);
    }
}

// The fewest lanes that hold a row of `c` elements in pieces of V, at most 16 elements a lane.
template <typename T, int V>
int norm_sized(const NormArgs& a) {
    const int pieces = (a.c + V - 1) / V;
    if constexpr (V > 1) {
        if (pieces <= 8) return norm_rows<T, V, 8, 1>(a);
        if (pieces <= 16) return norm_rows<T, V, 16, 1>(a);
        if (pieces <= 32) return norm_rows<T, V, 32, 1>(a);
        if (pieces <= 64) return norm_rows<T, V, 64, 1>(a);
        if (pieces <= 128) return norm_rows<T, V, 64, 2>(a);
        if (pieces <= 256) return norm_rows<T, V, 256, 1>(a);
        if (pieces <= 512) return norm_rows<T, V, 256, 2>(a);
        if constexpr (V == 4) {
            if (pieces <= 1024) return norm_rows<T, V, 256, 4>(a);
            if (pieces <= 2048) return norm_rows<T, V, 512, 4>(a);
            if (pieces <= 4096) return norm_rows<T, V, 1024, 4>(a);
        } else {
            if (pieces <= 1024) return norm_rows<T, V, 512, 2>(a);
            if (pieces <= 2048) return norm_rows<T, V, 1024, 2>(a);
        }
    } else {
        if (pieces <= 128) return norm_steps<T, 16>(a);
        if (pieces <= 256) return norm_steps<T, 32>(a);
        if (pieces <= 512) return norm_steps<T, 64>(a);
        if (pieces <= 1024) return norm_rows<T, V, 256, 4>(a);
        if (pieces <= 2048) return norm_rows<T, V, 256, 8>(a);
        if (pieces <= 8192) return norm_rows<T, V, 1024, 8>(a);
    }
    return norm_wide<T>(a);
}

template <typename T>
int norm_typed(const NormArgs& a) {
    constexpr int kN = 16 / (int)sizeof(T);
    const bool pieces = a.c % kN == 0 && aligned16(a.x) && aligned16(a.out) && (!a.dy || aligned16(a.dy));
    return pieces ? norm_sized<T, kN>(a) : norm_sized<T, 1>(a);
}

int check(int64_t n, int c, sp_dtype dt) {
    if (n < 0 || n > (int64_t)1 << 40 || c < 1 || c > 65536) return fail(SP_ERR_INVALID_ARG, "bad row or channel count");
    if (dt != SP_F32 && dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    return SP_OK;
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" {

int sp_layer_norm_fwd(const void* d_x, int64_t n, int32_t c, const float* d_gamma, const float* d_beta, float eps, void* d_y,
                      float* d_mean, float* d_rstd, sp_dtype dt, void* stream) {
    SP_TRY(check(n, c, dt));
    if (!(eps >= 0.f)) return fail(SP_ERR_INVALID_ARG, "eps must not be negative");
    if (!d_gamma || !d_beta || (n > 0 && (!d_x || !d_y || !d_mean || !d_rstd)))
        return fail(SP_ERR_INVALID_ARG, "a feature/parameter/statistics pointer is NULL");
    if (n == 0) return SP_OK;
    const NormArgs a{d_x, nullptr, n, c, d_gamma, d_beta, eps, d_y, d_mean, d_rstd, nullptr, nullptr, (hipStream_t)stream};
    return dt == SP_F32 ? norm_typed<float>(a) : norm_typed<bf16_t>(a);
}

int sp_layer_norm_bwd(const void* d_x, const void* d_dy, int64_t n, int32_t c, const float* d_gamma, const float* d_mean,
                      const float* d_rstd, void* d_dx, float* d_dgamma, float* d_dbeta, sp_dtype dt, void* stream) {
    SP_TRY(check(n, c, dt));
    if (!d_gamma || !d_dgamma || !d_dbeta || (n > 0 && (!d_x || !d_dy || !d_dx || !d_mean || !d_rstd)))
        return fail(SP_ERR_INVALID_ARG, "a feature/parameter/gradient pointer is NULL");
    const NormArgs a{d_x, d_dy, n, c, d_gamma, nullptr, 0.f, d_dx, const_cast<float*>(d_mean), const_cast<float*>(d_rstd), d_dgamma, d_dbeta,
                     (hipStream_t)stream};
    if (n == 0) return param_final(a, nullptr, 0);  // sums of nothing
    return dt == SP_F32 ? norm_typed<float>(a) : norm_typed<bf16_t>(a);
}

}  // extern "C"
