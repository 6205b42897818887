// The loss against a teacher's top logits and its gradient, in one pass over the student's logits.
//
// Memory bound: n * m logits read, as many gradients written; the teacher's k entries a row are little beside them.  A row stays as it
// was read, in the registers of the LANES threads that share it (16 lanes to a workgroup of 1024, at most 16 pieces of 16 bytes a
// thread: 65536 fp32 or 131072 bf16 logits), between the maximum, the sum of exponentials and the gradient, so it is read once; longer
// rows, and rows that are no whole pieces beyond 16384 elements, are read once more for each.  exp((z - max) / T) is exp2((z - max) *
// c2) with c2 = log2(e) / T: the difference first, so that rows of the type's lowest value (masked classes) stay what they are.
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

// What the lanes of a row know of its teacher: entries in LDS (a: softmax, then the gradient's share; col: column or -1)
struct Entries {
    float *a, *log_a, *zj;
    int32_t* col;
    __device__ __forceinline__ Entries(float* p, int k) : a(p), log_a(p + k), zj(p + 2 * k), col(reinterpret_cast<int32_t*>(p + 3 * k)) {}
};

// a_j = softmax(top / T) over the row's entries, in LDS; whether there are any.  The row's lanes call it together.
template <typename T, int LANES>
__device__ __forceinline__ bool teacher(const Entries& e, const T* z, int64_t row, int m, const float* top, const int32_t* index, int k,
                                        float inv_t, int l, float* room, int* turn) {
    float mx[1] = {-INFINITY}, s[1] = {0.f};
    for (int j = l; j < k; j += LANES) {
        const int col = index[row * k + j];
        const bool in = col >= 0 && col < m;
        const float t = in ? top[row * k + j] : -INFINITY;
        e.col[j] = in ? col : -1;
        e.log_a[j] = t;
        e.zj[j] = in ? elem(z[col]) : 0.f;
        mx[0] = fmaxf(mx[0], t);
    }
    reduce_lanes<LANES, Max>(mx, room, turn);
    for (int j = l; j < k; j += LANES) {
        const float t = (e.log_a[j] - mx[0]) * inv_t;
        e.log_a[j] = t;
        e.a[j] = e.col[j] < 0 || t == -INFINITY ? 0.f : expf(t);
        s[0] += e.a[j];
    }
    reduce_lanes<LANES, Add>(s, room, turn);
    const float log_s = logf(s[0]);
    for (int j = l; j < k; j += LANES) {
        e.a[j] /= s[0];
        e.log_a[j] -= log_s;
    }
    return mx[0] != -INFINITY;
}

// sum over j of a_j (log a_j - (z_j - max) / T)
template <int LANES>
__device__ __forceinline__ float teacher_loss(const Entries& e, int k, float mx, float inv_t, int l, float* room, int* turn) {
    float part[1] = {0.f};
    for (int j = l; j < k; j += LANES) {
        const float a = e.a[j];
        if (a != 0.f) part[0] += a * (e.log_a[j] - (e.zj[j] - mx) * inv_t);
    }
    reduce_lanes<LANES, Add>(part, room, turn);
    return part[0];
}

// dz at the teacher's columns: scale * (p - the shares of all entries of the column)
template <typename T, int LANES>
__device__ __forceinline__ void teacher_columns(const Entries& e, T* dz, int k, float c2, float mx, float inv_sum, float scale, int l) {
    for (int j = l; j < k; j += LANES) {
        const int col = e.col[j];
        if (col < 0) continue;
        float a = 0.f;
        bool first = true;
        for (int i = 0; i < k; ++i)
            if (e.col[i] == col) {
                first &= i >= j;
                a += e.a[i];
            }
        if (first) dz[col] = to_elem<T>(scale * (__builtin_amdgcn_exp2f((e.zj[j] - mx) * c2) * inv_sum - a));
    }
}

// R pieces of V logits a lane
template <typename T, int V, int LANES, int R>
__global__ __launch_bounds__(kBlock<LANES>) void distill_kernel(const T* z, int64_t n, int m, const float* __restrict__ top,
                                                                const int32_t* __restrict__ index, int k, float inv_t, float tt,
                                                                const float* __restrict__ weight, float each,
                                                                double* __restrict__ partial, T* dz) {
    constexpr int kGroups = kBlock<LANES> / LANES;
    extern __shared__ float lds[];
    __shared__ float room[kReduceRoom<LANES>];
    __shared__ double losses[kGroups];
    int turn = 0;
    const int g = threadIdx.x / LANES, l = threadIdx.x % LANES;
    const Entries e(lds + g * 4 * k, k);
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
        const bool some = teacher<T, LANES>(e, zr, row, m, top, index, k, inv_t, l, room, &turn);
        float mx[1] = {-INFINITY}, sum[1] = {0.f};
#pragma unroll
        for (int r = 0; r < R; ++r)
            if ((r * LANES + l) * V < m)
#pragma unroll
                for (int i = 0; i < V; ++i) mx[0] = fmaxf(mx[0], elem(v[r].e[i]));
        reduce_lanes<LANES, Max>(mx, room, &turn);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if ((r * LANES + l) * V < m)
#pragma unroll
                for (int i = 0; i < V; ++i) sum[0] += __builtin_amdgcn_exp2f((elem(v[r].e[i]) - mx[0]) * c2);
        reduce_lanes<LANES, Add>(sum, room, &turn);
        const float w = weight ? weight[row] : each, inv_sum = 1.f / sum[0], scale = w * tt * inv_t;
        const float part = teacher_loss<LANES>(e, k, mx[0], inv_t, l, room, &turn);
        if (l == 0 && some) loss += (double)w * (double)tt * ((double)part + (double)logf(sum[0]));
        if (dz) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int col = (r * LANES + l) * V;
                Piece<T, V> o;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    o.e[i] = to_elem<T>(some ? scale * (__builtin_amdgcn_exp2f((elem(v[r].e[i]) - mx[0]) * c2) * inv_sum) : 0.f);
                if (col < m) store_piece<T, V>(dz + row * m + col, o);
            }
            if constexpr (LANES > 64) __syncthreads();  // the row is written before its columns of the teacher are written again
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (some) teacher_columns<T, LANES>(e, dz + row * m, k, c2, mx[0], inv_sum, scale, l);
        }
        if constexpr (LANES > 64) __syncthreads();  // the next row's entries overwrite these
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (l == 0) losses[g] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < kGroups; ++i) s += losses[i];
        partial[blockIdx.x] = s;
    }
}

// Rows that do not fit the registers of a workgroup
constexpr int kWide = 1024;
template <typename T, int V>
__global__ __launch_bounds__(kWide) void distill_wide_kernel(const T* z, int64_t n, int m, const float* __restrict__ top,
                                                             const int32_t* __restrict__ index, int k, float inv_t, float tt,
                                                             const float* __restrict__ weight, float each, double* __restrict__ partial,
                                                             T* dz) {
    extern __shared__ float lds[];
    __shared__ float room[kReduceRoom<kWide>];
    int turn = 0;
    const int l = threadIdx.x;
    const Entries e(lds, k);
    const float c2 = kLog2e * inv_t;
    double loss = 0.0;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* zr = z + row * m;
        const bool some = teacher<T, kWide>(e, zr, row, m, top, index, k, inv_t, l, room, &turn);
        float mx[1] = {-INFINITY}, sum[1] = {0.f};
        for (int64_t col = l * V; col < m; col += kWide * V) {
            const Piece<T, V> v = load_piece<T, V>(zr + col);
#pragma unroll
            for (int i = 0; i < V; ++i) mx[0] = fmaxf(mx[0], elem(v.e[i]));
        }
        reduce_lanes<kWide, Max>(mx, room, &turn);
        for (int64_t col = l * V; col < m; col += kWide * V) {
            const Piece<T, V> v = load_piece<T, V>(zr + col);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0] += __builtin_amdgcn_exp2f((elem(v.e[i]) - mx[0]) * c2);
        }
        reduce_lanes<kWide, Add>(sum, room, &turn);
        const float w = weight ? weight[row] : each, inv_sum = 1.f / sum[0], scale = w * tt * inv_t;
        const float part = teacher_loss<kWide>(e, k, mx[0], inv_t, l, room, &turn);
        if (l == 0 && some) loss += (double)w * (double)tt * ((double)part + (double)logf(sum[0]));
        if (dz) {
            for (int64_t col = l * V; col < m; col += kWide * V) {
                Piece<T, V> v = load_piece<T, V>(zr + col);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    v.e[i] = to_elem<T>(some ? scale * (__builtin_amdgcn_exp2f((elem(v.e[i]) - mx[0]) * c2) * inv_sum) : 0.f);
                store_piece<T, V>(dz + row * m + col, v);
            }
            __syncthreads();
            if (some) teacher_columns<T, kWide>(e, dz + row * m, k, c2, mx[0], inv_sum, scale, l);
        }
        __syncthreads();
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
    const float inv_t = 1.f / a.temperature, tt = a.temperature * a.temperature, each = 1.f / (float)a.n;
    auto kernel = distill_kernel<T, V, LANES, R>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kBlock<LANES>), (size_t)kGroups * 4 * a.k * 4, a.s, static_cast<const T*>(a.z), a.n, a.m,
                       a.top, a.index, a.k, inv_t, tt, a.weight, each, ptr<double>(partial), static_cast<T*>(a.dz));
    return finish(a, ptr<double>(partial), blocks);
}

template <typename T, int V>
int launch_wide(const DistillArgs& a) {
    const int blocks = (int)std::min<int64_t>(a.n, 1024);
    Buf partial = dev_alloc((size_t)blocks * 8, a.s);
    if (!partial) return SP_ERR_ALLOC;
    const float inv_t = 1.f / a.temperature, tt = a.temperature * a.temperature, each = 1.f / (float)a.n;
    auto kernel = distill_wide_kernel<T, V>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kWide), (size_t)4 * a.k * 4, a.s, static_cast<const T*>(a.z), a.n, a.m, a.top, a.index, a.k,
                       inv_t, tt, a.weight, each, ptr<double>(partial), static_cast<T*>(a.dz));
    return finish(a, ptr<double>(partial), blocks);
}

// The fewest lanes that hold a row in at most 4 pieces (up to a wavefront), then at most 16; with many entries no fewer than a
// wavefront, which go over the pairs of entries (16 rows a workgroup would also need 16 times the LDS for them).
template <typename T, int V>
int sized(const DistillArgs& a) {
    const int pieces = (a.m + V - 1) / V;
    if (pieces <= 16 && a.k <= 64) return launch<T, V, 16, 1>(a);
    if (pieces <= 64 && a.k <= 64) return launch<T, V, 16, 4>(a);
    if (pieces <= 256) return launch<T, V, 64, 4>(a);
    if (pieces <= 1024) return launch<T, V, 256, 4>(a);
    if (pieces <= 4096) return launch<T, V, 256, 16>(a);
    if (pieces <= 8192) return launch<T, V, 1024, 8>(a);
    if (pieces <= 16384) return launch<T, V, 1024, 16>(a);
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
    if (!(temperature > 0.f) || !(temperature <= 3.0e38f)) return fail(SP_ERR_INVALID_ARG, "the temperature must be positive and finite");
    if (!d_loss || (n > 0 && (!d_logits || !d_top || !d_index))) return fail(SP_ERR_INVALID_ARG, "a logit/teacher/loss pointer is NULL");
    const DistillArgs a{d_logits, n, m, d_top, d_index, k, temperature, d_weight, d_loss, d_dlogits, (hipStream_t)stream};
    if (n == 0) return finish(a, nullptr, 0);
    return dt == SP_F32 ? typed<float>(a) : typed<bf16_t>(a);
}
