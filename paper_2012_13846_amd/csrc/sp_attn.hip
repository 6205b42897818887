// Attention with a sliding window and a few first rows that stay visible, over packed clouds: forward pass and gradients.
#include <algorithm>

#include "sp_attn.h"

namespace sp {
namespace {

constexpr int kThreads = 256;

template <typename T>
__global__ __launch_bounds__(kThreads) void attn_fwd_rows_kernel(AttnFwd<T> f) {
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = at / f.w.heads;
    if (row >= f.w.n_q) return;
    const Cloud c(f.w, cloud_of<1>(f.w.q_starts, f.w.clouds, f.w.n_q, (int)row));
    forward_row(f, c, (int)row - c.q0, (int)(at % f.w.heads));
}

// delta = dout . o of every query and head: a wavefront a row and head
template <typename T>
__global__ __launch_bounds__(kThreads) void attn_delta_kernel(AttnBwd<T> g) {
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = at / g.w.heads;
    if (row >= g.w.n_q) return;
    const int h = (int)(at % g.w.heads), lane = threadIdx.x & 63;
    const T *o = g.o.at(row, h, g.w.dim), *d = g.dout.at(row, h, g.w.dim);
    float s = 0.f;
    for (int e = lane; e < g.w.dim; e += 64) s += elem(o[e]) * elem(d[e]);
    s = wave_reduce<Add>(s);
    if (lane == 0) g.delta[at] = s;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void attn_dq_rows_kernel(AttnBwd<T> g) {
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = at / g.w.heads;
    if (row >= g.w.n_q) return;
    const Cloud c(g.w, cloud_of<1>(g.w.q_starts, g.w.clouds, g.w.n_q, (int)row));
    query_gradient_row(g, c, (int)row - c.q0, (int)(at % g.w.heads));
}

template <typename T>
__global__ __launch_bounds__(kThreads) void attn_dkv_rows_kernel(AttnBwd<T> g) {
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = at / g.w.kv_heads;
    if (row >= g.w.n_k) return;
    const Cloud c(g.w, cloud_of<1>(g.w.k_starts, g.w.clouds, g.w.n_k, (int)row));
    key_gradient_row(g, c, (int)row - c.k0, (int)(at % g.w.kv_heads));
}

unsigned row_blocks(int64_t rows, int heads) { return (unsigned)((rows * heads + 3) / 4); }

template <typename T>
int forward(const AttnFwd<T>& f, hipStream_t s) {
    if (f.w.n_q == 0) return SP_OK;
    hipLaunchKernelGGL(attn_fwd_rows_kernel<T>, dim3(row_blocks(f.w.n_q, f.w.heads)), dim3(kThreads), 0, s, f);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T>
int backward(AttnBwd<T> g, hipStream_t s) {
    Buf delta = dev_alloc((size_t)g.w.n_q * g.w.heads * 4, s);
    if (!delta) return SP_ERR_ALLOC;
    g.delta = ptr<float>(delta);
    if (g.w.n_q > 0) {
        hipLaunchKernelGGL(attn_delta_kernel<T>, dim3(row_blocks(g.w.n_q, g.w.heads)), dim3(kThreads), 0, s, g);
        hipLaunchKernelGGL(attn_dq_rows_kernel<T>, dim3(row_blocks(g.w.n_q, g.w.heads)), dim3(kThreads), 0, s, g);
    }
    if (g.w.n_k > 0) hipLaunchKernelGGL(attn_dkv_rows_kernel<T>, dim3(row_blocks(g.w.n_k, g.w.kv_heads)), dim3(kThreads), 0, s, g);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

int check(const sp_window_attn* a, Window* w) {
    if (!a) return fail(SP_ERR_INVALID_ARG, "the description is NULL");
    if (a->n_q < 0 || a->n_k < 0 || a->n_clouds < 0) return fail(SP_ERR_INVALID_ARG, "negative row or cloud count");
    if (a->dt != SP_F32 && a->dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads) return fail(SP_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
    if (a->dim < 1) return fail(SP_ERR_INVALID_ARG, "bad head width");
    if (a->left < 0 || a->right < 0 || a->sinks < 0) return fail(SP_ERR_INVALID_ARG, "left, right and sinks must not be negative");
    if (!(a->scale > -3.0e38f && a->scale < 3.0e38f)) return fail(SP_ERR_INVALID_ARG, "the scale must be finite");
    if (a->dim > kMaxDim || a->heads > 65535 || a->n_q > 1 << 30 || a->n_k > 1 << 30)
        return fail(SP_ERR_UNSUPPORTED, "head widths above %d, more than 65535 heads or more than 2^30 rows", kMaxDim);
    if (!a->d_q_starts || !a->d_k_starts) return fail(SP_ERR_INVALID_ARG, "the starts are NULL");
    w->q_starts = a->d_q_starts;
    w->k_starts = a->d_k_starts;
    w->n_q = (int)a->n_q;
    w->n_k = (int)a->n_k;
    w->clouds = a->n_clouds;
    w->heads = a->heads;
    w->kv_heads = a->kv_heads;
    w->group = a->heads / a->kv_heads;
    w->dim = a->dim;
    w->left = (int)std::min<int64_t>(a->left, a->n_k);
    w->right = (int)std::min<int64_t>(a->right, a->n_q);
    w->sinks = (int)std::min<int64_t>(a->sinks, a->n_k);
    w->scale = a->scale;
    return SP_OK;
}

struct Named {
    const void* p;
    int64_t ld, rows, heads;
    const char* name;
};
int check_rows(const Named* arrays, int n, int dim) {
    for (int i = 0; i < n; ++i) {
        const Named& a = arrays[i];
        if (a.rows > 0 && !a.p) return fail(SP_ERR_INVALID_ARG, "%s is NULL", a.name);
        if (a.rows > 1 && a.ld < a.heads * dim) return fail(SP_ERR_INVALID_ARG, "the rows of %s overlap", a.name);
        if (a.ld > (int64_t)1 << 32) return fail(SP_ERR_UNSUPPORTED, "the rows of %s are more than 2^32 elements apart", a.name);
    }
    return SP_OK;
}

template <typename T>
Rows<const T> in(const void* p, int64_t ld) { return {static_cast<const T*>(p), ld}; }
template <typename T>
Rows<T> out(void* p, int64_t ld) { return {static_cast<T*>(p), ld}; }

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" {

int sp_window_attn_fwd(const sp_window_attn* a, const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v,
                       int64_t ldv, void* d_o, int64_t ldo, float* d_lse, void* stream) {
    Window w;
    SP_TRY(check(a, &w));
    const Named arrays[] = {{d_q, ldq, w.n_q, w.heads, "q"}, {d_k, ldk, w.n_k, w.kv_heads, "k"}, {d_v, ldv, w.n_k, w.kv_heads, "v"},
                            {d_o, ldo, w.n_q, w.heads, "o"}, {d_lse, w.heads, w.n_q, 0, "lse"}};
    SP_TRY(check_rows(arrays, 5, w.dim));
    hipStream_t s = (hipStream_t)stream;
    if (a->dt == SP_F32) return forward<float>({w, in<float>(d_q, ldq), in<float>(d_k, ldk), in<float>(d_v, ldv), out<float>(d_o, ldo), d_lse}, s);
    return forward<bf16_t>({w, in<bf16_t>(d_q, ldq), in<bf16_t>(d_k, ldk), in<bf16_t>(d_v, ldv), out<bf16_t>(d_o, ldo), d_lse}, s);
}

int sp_window_attn_bwd(const sp_window_attn* a, const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v,
                       int64_t ldv, const void* d_o, int64_t ldo, const void* d_dout, int64_t lddout, const float* d_lse, void* d_dq,
                       int64_t lddq, void* d_dk, int64_t lddk, void* d_dv, int64_t lddv, void* stream) {
    Window w;
    SP_TRY(check(a, &w));
    const Named arrays[] = {{d_q, ldq, w.n_q, w.heads, "q"},          {d_k, ldk, w.n_k, w.kv_heads, "k"},   {d_v, ldv, w.n_k, w.kv_heads, "v"},
                            {d_o, ldo, w.n_q, w.heads, "o"},          {d_dout, lddout, w.n_q, w.heads, "dout"}, {d_lse, w.heads, w.n_q, 0, "lse"},
                            {d_dq, lddq, w.n_q, w.heads, "dq"},       {d_dk, lddk, w.n_k, w.kv_heads, "dk"}, {d_dv, lddv, w.n_k, w.kv_heads, "dv"}};
    SP_TRY(check_rows(arrays, 9, w.dim));
    hipStream_t s = (hipStream_t)stream;
    if (a->dt == SP_F32)
        return backward<float>({w, in<float>(d_q, ldq), in<float>(d_k, ldk), in<float>(d_v, ldv), in<float>(d_o, ldo), in<float>(d_dout, lddout),
                                d_lse, nullptr, out<float>(d_dq, lddq), out<float>(d_dk, lddk), out<float>(d_dv, lddv)}, s);
    return backward<bf16_t>({w, in<bf16_t>(d_q, ldq), in<bf16_t>(d_k, ldk), in<bf16_t>(d_v, ldv), in<bf16_t>(d_o, ldo),
                             in<bf16_t>(d_dout, lddout), d_lse, nullptr, out<bf16_t>(d_dq, lddq), out<bf16_t>(d_dk, lddk),
                             out<bf16_t>(d_dv, lddv)}, s);
}

}  // extern "C"
