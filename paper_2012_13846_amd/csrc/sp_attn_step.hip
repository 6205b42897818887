// One new token of each sequence: its key and value go to the ring cache, and it attends over the window and the first tokens.
#include "sp_attn.h"

namespace sp {
namespace {

constexpr int kThreads = 256;

template <typename T>
struct StepArgs {
    const T *q, *k_new, *v_new;
    T *k_cache, *v_cache, *o;
    const int32_t* lens;
    int batch, cap, heads, kv_heads, group, dim, left, sinks;
    float scale;
};

// A wavefront a sequence and query head.  The new token's rows are read from k_new and v_new: another wavefront may be writing them
// to the cache.
template <typename T>
__global__ __launch_bounds__(kThreads) void attn_step_rows_kernel(StepArgs<T> a) {
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (at >= (int64_t)a.batch * a.heads) return;
    const int b = (int)(at / a.heads), h = (int)(at % a.heads), kh = h / a.group, p = a.lens[b], ring = a.cap - a.sinks;
    const int64_t fresh = ((int64_t)b * a.kv_heads + kh) * a.dim, slot_step = (int64_t)a.kv_heads * a.dim;
    const int64_t cache = (int64_t)b * a.cap * slot_step + (int64_t)kh * a.dim;
    auto slot = [&](int j) { return j < a.sinks ? j : a.sinks + (j - a.sinks) % ring; };
    T* o = a.o + at * a.dim;
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    if (p >= 0) {
        if (h % a.group == 0)
            for (int e = lane; e < a.dim; e += 64) {
                a.k_cache[cache + slot(p) * slot_step + e] = a.k_new[fresh + e];
                a.v_cache[cache + slot(p) * slot_step + e] = a.v_new[fresh + e];
            }
        const int lo = max(max(p - a.left, p - ring + 1), 0), first = min(a.sinks, lo), n = first + p + 1 - lo;
        auto row = [&](const T* all, const T* now, int t) {
            const int j = t < first ? t : lo + t - first;
            return j == p ? now + fresh : all + cache + slot(j) * slot_step;
        };
        const float c2 = a.scale * kLog2e;
        for (int t0 = 0; t0 < n; t0 += 64) {
            const bool in = t0 + lane < n;
            const float s = in ? dot(a.q + at * a.dim, row(a.k_cache, a.k_new, t0 + lane), a.dim) * c2 : -INFINITY;
            const float top = fmaxf(m, wave_reduce<Max>(s)), base = top == -INFINITY ? 0.f : top;
            const float old = __builtin_amdgcn_exp2f(m - base), e = in ? __builtin_amdgcn_exp2f(s - base) : 0.f;
            l = l * old + wave_reduce<Add>(e);
            acc[0] *= old;
            acc[1] *= old;
            add_rows<T>(acc, e, min(64, n - t0), a.dim, [&](int t) { return row(a.v_cache, a.v_new, t0 + t); });
            m = top;
        }
        acc[0] /= l;
        acc[1] /= l;
    }
    put_row(o, acc, a.dim);
}

template <typename T>
int step(const StepArgs<T>& a, hipStream_t s) {
    hipLaunchKernelGGL(attn_step_rows_kernel<T>, dim3((unsigned)(((int64_t)a.batch * a.heads + 3) / 4)), dim3(kThreads), 0, s, a);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" int sp_window_attn_step(const void* d_q, const void* d_k_new, const void* d_v_new, void* d_k_cache, void* d_v_cache,
                                   const int32_t* d_lens, int32_t batch, int32_t cap, int32_t heads, int32_t kv_heads, int32_t dim,
                                   int32_t left, int32_t sinks, float scale, void* d_o, sp_dtype dt, void* stream) {
    if (batch < 0) return fail(SP_ERR_INVALID_ARG, "negative batch");
    if (dt != SP_F32 && dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (heads < 1 || kv_heads < 1 || heads % kv_heads) return fail(SP_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
    if (dim < 1) return fail(SP_ERR_INVALID_ARG, "bad head width");
    if (left < 0 || sinks < 0 || cap <= sinks) return fail(SP_ERR_INVALID_ARG, "left and sinks must not be negative, the cache longer than sinks");
    if (!(scale > -3.0e38f && scale < 3.0e38f)) return fail(SP_ERR_INVALID_ARG, "the scale must be finite");
    if (dim > kMaxDim || heads > 65535 || batch > 65535)
        return fail(SP_ERR_UNSUPPORTED, "head widths above %d, more than 65535 heads or sequences", kMaxDim);
    if (batch == 0) return SP_OK;
    if (!d_q || !d_k_new || !d_v_new || !d_k_cache || !d_v_cache || !d_lens || !d_o) return fail(SP_ERR_INVALID_ARG, "a pointer is NULL");
    hipStream_t s = (hipStream_t)stream;
    if (dt == SP_F32)
        return step<float>({(const float*)d_q, (const float*)d_k_new, (const float*)d_v_new, (float*)d_k_cache, (float*)d_v_cache, (float*)d_o,
                            d_lens, batch, cap, heads, kv_heads, heads / kv_heads, dim, left, sinks, scale}, s);
    return step<bf16_t>({(const bf16_t*)d_q, (const bf16_t*)d_k_new, (const bf16_t*)d_v_new, (bf16_t*)d_k_cache, (bf16_t*)d_v_cache,
                         (bf16_t*)d_o, d_lens, batch, cap, heads, kv_heads, heads / kv_heads, dim, left, sinks, scale}, s);
}
