// The loss against a teacher's top logits and its gradient, in one pass over the student's logits.
//
// Memory bound: n * m logits read, as many gradients written; the teacher's k entries a row are little beside them.  A row stays as it
// was read, in the registers of the LANES threads that share it (8 lanes to a workgroup of 256, at most 8 pieces of 16 bytes or
// elements a thread), between the maximum, the sum of exponentials and the gradient, so it is read once; longer rows are read a
// second time.  exp((z - max) / T) is exp2((z - max) * c2) with c2 = log2(e) / T: the difference first, so that rows of the type's
// lowest value (masked classes) stay what they are.
// The teacher's columns are written after the row by the lane that holds the column's first entry; two entries of one column are
// added by that lane, in the order of the entries, so there are no atomics.
#include <algorithm>

#include "sp_elem.h"

namespace sp {
namespace {

constexpr int kMaxTop = 256;
constexpr float kLog2e = 1.4426950408889634f;

template <int LANES>
constexpr int kBlock = LANES > 256 ? LANES : 256;

struct DistillArgs {
    const void* z;
    int64_t n;
    int m;
    const float* top;
    const int32_t* index;
    int k;
    float temperature;
    const float* weight;
    float* loss;
    void* dz;
    hipStream_t s;
};

// A row's entries in LDS (a: softmax; col: column or -1, up to a multiple of 4), made by the first kLead of the row's lanes, all of
// them in one wavefront, while the others read the row.
struct Entries {
    float *a, *log_a, *zj;
    int32_t* col;
    int k;
    static constexpr int kWords = 4;
    __device__ __forceinline__ Entries(float* p, int k_) : k(k_) {
        const int pitch = (k + 3) & ~3;
        a = p;
        log_a = p + pitch;
        zj = p + 2 * pitch;
        col = reinterpret_cast<int32_t*>(p + 3 * pitch);
    }
};
template <int LANES>
constexpr int kLead = LANES < 64 ? LANES : 64;

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float log_of(float v) { return __builtin_amdgcn_logf(v) * 0.6931471805599453f; }

// a_j = softmax(top / T) over the row's entries; whether there are any (NaN is one).  By the leading lanes.
template <typename T, int L>
__device__ __forceinline__ bool teacher(const Entries& e, const T* z, int64_t row, int m, const float* top, const int32_t* index, float inv_t,
                                        int l) {
    float mx = -INFINITY, s = 0.f;
    for (int j = l; j < e.k; j += L) {
        const int col = index[row * e.k + j];
        const bool in = (unsigned)col < (unsigned)m;
        const float t = in ? top[row * e.k + j] : -INFINITY;
        e.col[j] = in ? col : -1;
        e.log_a[j] = t;
        e.zj[j] = in ? elem(z[col]) : 0.f;
        mx = fmaxf(mx, t);
    }
    if (l < (-e.k & 3)) {
        e.col[e.k + l] = -1;
        e.a[e.k + l] = 0.f;
    }
    mx = lanes_reduce<L, Max>(mx);
    for (int j = l; j < e.k; j += L) {
        const float top_j = e.log_a[j], t = (top_j - mx) * inv_t;
        const float a = top_j == -INFINITY ? 0.f : exp2_of(t * kLog2e);  // -infinity: no entry, too
        e.log_a[j] = t;
        e.a[j] = a;
        s += a;
    }
    s = lanes_reduce<L, Add>(s);
    const float log_s = log_of(s), inv = 1.f / s;
    for (int j = l; j < e.k; j += L) {
        e.a[j] *= inv;
        e.log_a[j] -= log_s;
    }
    return s != 0.f;  // the largest entry adds 1
}

// sum over j of a_j (log a_j - (z_j - max) / T), by the leading lanes
template <int L>
__device__ __forceinline__ float teacher_loss(const Entries& e, float mx, float inv_t, int l) {
    float part = 0.f;
    for (int j = l; j < e.k; j += L) {
        const float a = e.a[j];
        if (a != 0.f) part += a * (e.log_a[j] - (e.zj[j] - mx) * inv_t);
    }
    return lanes_reduce<L, Add>(part);
}

// dz at the teacher's columns: scale * (p - the shares of all entries of the column), by the leading lanes
template <typename T, int L>
__device__ __forceinline__ void teacher_columns(const Entries& e, T* dz, float c2, float mx, float inv_sum, float scale, int l) {
    for (int j = l; j < e.k; j += L) {
        const int col = e.col[j];
        if (col < 0) continue;
        float a = 0.f;
        int first = j;
        for (int i = 0; i < e.k; i += 4) {
            const int4 c = *reinterpret_cast<const int4*>(e.col + i);
            const float4 v = *reinterpret_cast<const float4*>(e.a + i);
            a += c.x == col ? v.x : 0.f;
            a += c.y == col ? v.y : 0.f;
            a += c.z == col ? v.z : 0.f;
            a += c.w == col ? v.w : 0.f;
            first = min(first, c.x == col ? i : c.y == col ? i + 1 : c.z == col ? i + 2 : c.w == col ? i + 3 : j);
        }
        if (first == j) dz[col] = to_elem<T>(scale * (exp2_of((e.zj[j] - mx) * c2) * inv_sum - a));
    }
}

// The lanes of a row meet: LDS and memory that one wrote is there for the others
template <int LANES>
__device__ __forceinline__ void meet() {
    if constexpr (LANES > 64) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// R pieces of V logits a lane.  160000 x 40 fp32 with five entries: 18 us, 3.2 TB/s; eight lanes a row: 16 take 24 us.
template <typename T, int V, int LANES, int R>
__global__ __launch_bounds__(kBlock<LANES>) void distill_kernel(const T* z, int64_t n, int m, const float* __restrict__ top,
                                                                const int32_t* __restrict__ index, int k, float temperature, float inv_t,
                                                                const float* __restrict__ weight, float each,
                                                                double* __restrict__ partial, T* dz) {
    constexpr int kGroups = kBlock<LANES> / LANES, L = kLead<LANES>;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    __shared__ float room[kReduceRoom<LANES>];
    __shared__ double losses[kGroups];
    __shared__ int any[kGroups];
    int turn = 0;
    const int g = threadIdx.x / LANES, l = threadIdx.x % LANES;
    const Entries e(lds + g * Entries::kWords * ((k + 3) & ~3), k);
    const float c2 = kLog2e * inv_t;
    double loss = 0.0;
    for (int64_t row = (int64_t)blockIdx.x * kGroups + g; row < n; row += (int64_t)gridDim.x * kGroups) {
        const T* zr = z + row * m;
        Piece<T, V> v[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int col = (r * LANES + l) * V;
            if (col < m) v[r] = load_piece<T, V>(zr + col);
        }
        bool some = true;
        if (l < L) {
            some = teacher<T, L>(e, zr, row, m, top, index, inv_t, l);
            if (LANES > 64 && l == 0) any[g] = some;
        }
        float mx[1] = {-INFINITY}, sum[1] = {0.f};
#pragma unroll
        for (int r = 0; r < R; ++r)
            if ((r * LANES + l) * V < m)
#pragma unroll
                for (int i = 0; i < V; ++i) mx[0] = fmaxf(mx[0], elem(v[r].e[i]));
        reduce_lanes<LANES, Max>(mx, room, &turn);
        if (LANES > 64) some = any[g];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if ((r * LANES + l) * V < m)
#pragma unroll
                for (int i = 0; i < V; ++i) sum[0] += exp2_of((elem(v[r].e[i]) - mx[0]) * c2);
        reduce_lanes<LANES, Add>(sum, room, &turn);
        const float w = weight ? weight[row] : each, inv_sum = 1.f / sum[0], scale = w * temperature;
        if (dz) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int col = (r * LANES + l) * V;
                Piece<T, V> o;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    o.e[i] = to_elem<T>(some ? scale * (exp2_of((elem(v[r].e[i]) - mx[0]) * c2) * inv_sum) : 0.f);
                if (col < m) store_piece<T, V>(dz + row * m + col, o);
            }
        }
        meet<LANES>();  // the row is written before its columns of the teacher are written again
        if (l < L) {
            const float part = teacher_loss<L>(e, mx[0], inv_t, l);
            if (l == 0 && some) loss += (double)w * (double)temperature * (double)temperature * ((double)part + (double)log_of(sum[0]));
            if (dz && some) teacher_columns<T, L>(e, dz + row * m, c2, mx[0], inv_sum, scale, l);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the leading lanes alone use the entries
    }
    if (l == 0) losses[g] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < kGroups; ++i) s += losses[i];
        partial[blockIdx.x] = s;
    }
}

// Longer rows (16 pieces a thread leave a SIMD two wavefronts: 32768 bf16 logits in registers 270 us, here 194): read twice, the second time from the chip's last cache, with a
// running maximum and sum the first time.  The gradient's stores do not stay in that cache, which leaves it to the rows: 550 -> 502 us
// on 4096 x 131072 in bf16 (4.3 TB/s of logits and gradient).  512 threads: 256 take 557 us, 1024 516.
constexpr int kWide = 512;
template <typename T, int V>
__global__ __launch_bounds__(kWide, 4) void distill_wide_kernel(const T* z, int64_t n, int m, const float* __restrict__ top,
                                                                const int32_t* __restrict__ index, int k, float temperature, float inv_t,
                                                                const float* __restrict__ weight, float each,
                                                                double* __restrict__ partial, T* dz) {
    constexpr int kAhead = sizeof(T) * V == 16 && V == 8 ? 4 : 8;  // pieces asked for at a time: 8 of bf16 spill
    extern __shared__ __attribute__((aligned(16))) float lds[];
    __shared__ float room[2][2 * kWide / 64];
    __shared__ int any;
    const int l = threadIdx.x;
    const Entries e(lds, k);
    const float c2 = kLog2e * inv_t;
    double loss = 0.0;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x, turn ^= 1) {
        const T* zr = z + row * m;
        bool some = true;
        if (l < 64) {
            some = teacher<T, 64>(e, zr, row, m, top, index, inv_t, l);
            if (l == 0) any = some;
        }
        float mx = -INFINITY, sum = 0.f;
        for (int64_t c0 = (int64_t)l * V; c0 < m; c0 += (int64_t)kWide * V * kAhead) {
            Piece<T, V> v[kAhead];
#pragma unroll
            for (int r = 0; r < kAhead; ++r) {
                const int64_t col = c0 + (int64_t)r * kWide * V;
                if (col < m) v[r] = load_piece<T, V>(zr + col);
            }
            float t = mx;
#pragma unroll
            for (int r = 0; r < kAhead; ++r)
                if (c0 + (int64_t)r * kWide * V < m)
#pragma unroll
                    for (int i = 0; i < V; ++i) t = fmaxf(t, elem(v[r].e[i]));
            const float base = t == -INFINITY ? 0.f : t;
            sum *= exp2_of((mx - base) * c2);
            mx = t;
#pragma unroll
            for (int r = 0; r < kAhead; ++r)
                if (c0 + (int64_t)r * kWide * V < m)
#pragma unroll
                    for (int i = 0; i < V; ++i) sum += exp2_of((elem(v[r].e[i]) - base) * c2);
        }
        // the lanes' maxima and sums joined
        {
            const float top_w = lanes_reduce<64, Max>(mx), base = top_w == -INFINITY ? 0.f : top_w;
            const float sum_w = lanes_reduce<64, Add>(sum * exp2_of((mx - base) * c2));
            if ((l & 63) == 0) {
                room[turn][l >> 6] = top_w;
                room[turn][kWide / 64 + (l >> 6)] = sum_w;
            }
            __syncthreads();
            float all = -INFINITY, s = 0.f;
#pragma unroll
            for (int i = 0; i < kWide / 64; ++i) all = fmaxf(all, room[turn][i]);
            const float from = all == -INFINITY ? 0.f : all;
#pragma unroll
            for (int i = 0; i < kWide / 64; ++i) s += room[turn][kWide / 64 + i] * exp2_of((room[turn][i] - from) * c2);
            mx = all;
            sum = all == -INFINITY ? NAN : s;  // nothing but -infinity: there is no softmax
        }
        some = any;
        const float w = weight ? weight[row] : each, inv_sum = 1.f / sum, scale = w * temperature, p_scale = scale * inv_sum;
        if (dz) {
            for (int64_t c0 = (int64_t)l * V; c0 < m; c0 += (int64_t)kWide * V * kAhead) {
                Piece<T, V> v[kAhead];
#pragma unroll
                for (int r = 0; r < kAhead; ++r) {
                    const int64_t col = c0 + (int64_t)r * kWide * V;
                    if (col < m) v[r] = load_piece<T, V>(zr + col);
                }
#pragma unroll
                for (int r = 0; r < kAhead; ++r) {
                    const int64_t col = c0 + (int64_t)r * kWide * V;
#pragma unroll
                    for (int i = 0; i < V; ++i) v[r].e[i] = to_elem<T>(some ? p_scale * exp2_of((elem(v[r].e[i]) - mx) * c2) : 0.f);
                    if (col < m) store_piece_past<T, V>(dz + row * m + col, v[r]);
                }
            }
        }
        __syncthreads();
        if (l < 64) {
            const float part = teacher_loss<64>(e, mx, inv_t, l);
            if (l == 0 && some) loss += (double)w * (double)temperature * (double)temperature * ((double)part + (double)log_of(sum));
            if (dz && some) teacher_columns<T, 64>(e, dz + row * m, c2, mx, inv_sum, scale, l);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (l == 0) partial[blockIdx.x] = loss;
}

__global__ __launch_bounds__(256) void distill_loss_kernel(const double* __restrict__ partial, int blocks, float* __restrict__ loss) {
    __shared__ double sums[256];
    double s = 0.0;
    for (int b = threadIdx.x; b < blocks; b += 256) s += partial[b];
    sums[threadIdx.x] = s;
    for (int half = 128; half > 0; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < half) sums[threadIdx.x] += sums[threadIdx.x + half];
    }
    if (threadIdx.x == 0) *loss = (float)sums[0];
}

int finish(const DistillArgs& a, const double* partial, int blocks) {
    hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(256), 0, a.s, partial, blocks, a.loss);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T, int V, int LANES, int R>
int launch(const DistillArgs& a) {
    constexpr int kGroups = kBlock<LANES> / LANES;
    const int blocks = (int)std::min<int64_t>((a.n + kGroups - 1) / kGroups, LANES > 256 ? 1024 : 4096);
    Buf partial = dev_alloc((size_t)blocks * 8, a.s);
    if (!partial) return SP_ERR_ALLOC;
    const float inv_t = 1.f / a.temperature, each = 1.f / (float)a.n;
    auto kernel = distill_kernel<T, V, LANES, R>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kBlock<LANES>), (size_t)kGroups * Entries::kWords * ((a.k + 3) & ~3) * 4, a.s, static_cast<const T*>(a.z), a.n, a.m,
                       a.top, a.index, a.k, a.temperature, inv_t, a.weight, each, ptr<double>(partial), static_cast<T*>(a.dz));
    return finish(a, ptr<double>(partial), blocks);
}

template <typename T, int V>
int launch_wide(const DistillArgs& a) {
    const int blocks = (int)std::min<int64_t>(a.n, 1024);
    Buf partial = dev_alloc((size_t)blocks * 8, a.s);
    if (!partial) return SP_ERR_ALLOC;
    const float inv_t = 1.f / a.temperature, each = 1.f / (float)a.n;
    auto kernel = distill_wide_kernel<T, V>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kWide), (size_t)Entries::kWords * ((a.k + 3) & ~3) * 4, a.s, static_cast<const T*>(a.z), a.n, a.m, a.top, a.index, a.k,
                       a.temperature, inv_t, a.weight, each, ptr<double>(partial), static_cast<T*>(a.dz));
    return finish(a, ptr<double>(partial), blocks);
}

// The fewest lanes that hold a row; with many entries no fewer than a wavefront, which go over the pairs of entries (more rows a
// workgroup would also need more LDS for them).
template <typename T, int V>
int sized(const DistillArgs& a) {
    const int pieces = (a.m + V - 1) / V;
    if (pieces <= 16 && a.k <= 32) return launch<T, V, 8, 2>(a);
    if (pieces <= 64 && a.k <= 64) return launch<T, V, 16, 4>(a);
    if (pieces <= 256) return launch<T, V, 64, 4>(a);
    if (pieces <= 1024) return launch<T, V, 256, 4>(a);
    if (pieces <= 2048) return launch<T, V, 256, 8>(a);
    return launch_wide<T, V>(a);
}

template <typename T>
int typed(const DistillArgs& a) {
    constexpr int kN = 16 / (int)sizeof(T);
    const bool pieces = a.m % kN == 0 && aligned16(a.z) && (!a.dz || aligned16(a.dz));
    return pieces ? sized<T, kN>(a) : sized<T, 1>(a);
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" int sp_distill(const void* d_logits, int64_t n, int32_t m, const float* d_top, const int32_t* d_index, int32_t k,
                          float temperature, const float* d_weight, float* d_loss, void* d_dlogits, sp_dtype dt, void* stream) {
    if (n < 0 || n > (int64_t)1 << 40 || m < 1 || k < 1 || k > kMaxTop) return fail(SP_ERR_INVALID_ARG, "bad row, class or entry count");
    if (dt != SP_F32 && dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    // 1 / T and log2(e) / T are fp32 numbers, too
    if (!(temperature >= 1e-37f) || !(temperature <= 3.0e38f)) return fail(SP_ERR_INVALID_ARG, "the temperature must be positive and finite (at least 1e-37)");
    if (!d_loss || (n > 0 && (!d_logits || !d_top || !d_index))) return fail(SP_ERR_INVALID_ARG, "a logit/teacher/loss pointer is NULL");
    const DistillArgs a{d_logits, n, m, d_top, d_index, k, temperature, d_weight, d_loss, d_dlogits, (hipStream_t)stream};
    if (n == 0) return finish(a, nullptr, 0);
    return dt == SP_F32 ? typed<float>(a) : typed<bf16_t>(a);
}
