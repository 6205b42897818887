// Attention with a sliding window and a few first rows that stay visible, over packed clouds: the forward pass (sp_attn_bwd.hip: the gradients).
#include <algorithm>

#include "sp_attn_rows.h"

namespace sp {
namespace {

// One pass over the keys with a running maximum and sum.  The maximum in use may lag the true one by 8 powers of two (probabilities up
// to 256, sums in fp32): the accumulators are multiplied again only when it falls behind, not whenever one of 32 rows has a new one.
// Bound by the vector pipe and the matrix pipe together: 16384 tokens, 32 heads of 128 over 8, window 1024: 316 - 343 us, 760 - 820 TFLOP/s, matrix
// pipe busy 37 %, vector pipe 43 %, no LDS bank conflicts; heads of 32 (373601 rows, 8 heads, 513 keys a row): 600 - 660 us, vector pipe
// 83 % (an exponential and four operations a pair against 128 multiply-adds).  64 keys a step: 32 leave a barrier for every 16 products;
// three wavefronts a SIMD for heads of 64, which need 165 registers; heads of 32 take 122 and get a fourth.  Row sums as products
// with ones would be free on the matrix pipe, but of probabilities rounded to bf16: lse must not be.
template <typename T, int NT, bool VEC, int W>
__global__ __launch_bounds__(64 * W, NT <= 2 ? 3 : 2) void attn_fwd_kernel(AttnFwd<T> f, int tiles) {
    using Tl = Tile<T, NT>;
    constexpr int kN = kKeys<T, W>, kB = kN / 32, kTileBytes = kN * Tl::kRowBytes;
    __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes];  // keys and values, two of each
    const Window& w = f.w;
    const RowTile<W> rt(w, tiles);
    const Cloud c(w, rt.cloud);
    const int64_t rows = (int64_t)c.a * w.group;
    if (!in_cloud(rt.r0, rows)) return;
    const WaveRows<W> wr(w, c, (uint32_t)rt.r0, (uint32_t)rows);
    const Reach& reach = wr.reach;
    const int lane = threadIdx.x & 63, kh = rt.kh, h = kh * w.group + wr.head;
    const auto pl = Tl::place();
    const KeyTiles<T, NT, VEC, W> kt(w, reach, f.k, f.v, c, kh);
    if (reach.n > 0) kt.load(lds, 0, 0);
    typename Tl::Frag q[Tl::kSteps];
    Tl::template load_row<VEC>(q, f.q.at(c.q0 + wr.query, h, w.dim), w.dim, wr.there, w.scale < 0.f);
    const float c2 = exponent_scale(w);
    const bool none = reach.n == 0 || wr.p + w.right < 0;  // the row sees nothing (else the last of its keys is seen at least)

    f32x16 acc[NT];
    float m, l;          // at most 8 powers of two below the row's largest score so far; this lane's half of the sum of exponentials
    bool other = false;  // there are values that are not finite
    // again: sums that were not finite, by `part` of the values
    auto pass = [&](auto again, int part) {
#pragma unroll
        for (int d = 0; d < NT; ++d) acc[d] = f32x16{};
        m = -INFINITY;
        l = 0.f;
        for (int slot = 0, buf = 0; slot < reach.n; slot += kN, buf ^= 1) {
            const char *keys = lds + buf * 2 * kTileBytes, *values = keys + kTileBytes;
            wait_tiles();
            if (slot + kN < reach.n) kt.load(lds, slot + kN, buf ^ 1);
            if (reach.none(w, slot, kN, wr.p_min, wr.p_max)) continue;
            f32x16 s[kB] = {};
            if (again && part != kFinite) {
                const SeenInTile seen(w, reach, slot, wr.p);
#pragma unroll
                for (int b = 0; b < kB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = seen.sees(b * 32 + 8 * (i / 4) + i % 4) ? 1.f : 0.f;
            } else {
#pragma unroll
                for (int st = 0; st < Tl::kSteps; ++st)
#pragma unroll
                    for (int b = 0; b < kB; ++b) s[b] = Tl::mma(Tl::direct(keys, pl, b, st), q[st], s[b]);
                if (again || !(wr.whole & reach.all(w, slot, kN, wr.p_min, wr.p_max))) {
                    const SeenInTile seen(w, reach, slot, wr.p);
                    if (!again && !seen.heads) {
#pragma unroll
                        for (int b = 0; b < kB; ++b)
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[b][i] = seen.in_range(b * 32 + 8 * (i / 4) + i % 4) ? s[b][i] : -INFINITY;
                    } else {
#pragma unroll
                        for (int b = 0; b < kB; ++b)
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[b][i] = seen.sees(b * 32 + 8 * (i / 4) + i % 4) ? s[b][i] : -INFINITY;
                    }
                }
                float top = m;
#pragma unroll
                for (int b = 0; b < kB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
                top = halves<Max>(top);
                if (__any((top - m) * c2 > 8.f)) {
                    const float old = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * c2);
                    l *= old;
#pragma unroll
                    for (int d = 0; d < NT; ++d) acc[d] *= old;
                    m = top;
                }
                const float m2 = m == -INFINITY ? 0.f : m * c2;
                // one operation less than the difference first; m2's rounding, which stands in the exponents and in lse, is below 2^-17 then
                if (__all(fabsf(m2) < 64.f)) {
#pragma unroll
                    for (int b = 0; b < kB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c2, -m2));
                } else {
                    const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int b = 0; b < kB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[b][i] = __builtin_amdgcn_exp2f((s[b][i] - from) * c2);
                }
                float sum[4] = {};
#pragma unroll
                for (int b = 0; b < kB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[i % 4] += s[b][i];
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            }
#pragma unroll
            for (int b = 0; b < kB; ++b)
#pragma unroll
                for (int st = 0; st < Tl::kTSteps; ++st) {
                    const auto pr = Tl::operand(s[b], st);
#pragma unroll
                    for (int d = 0; d < NT; ++d) {
                        auto rows = Tl::turned(values, pl, b, st, d);
                        if constexpr (again) rows = Tl::part_of(rows, part, &other);
                        acc[d] = Tl::mma(rows, pr, acc[d]);
                    }
                }
        }
        if (again && part != kFinite) {
            __syncthreads();
            return;
        }
        l = halves<Add>(l);
        const float inv = none ? 0.f : 1.f / l;
#pragma unroll
        for (int d = 0; d < NT; ++d) acc[d] *= inv;
        if (!wr.there) return;
        put_column<T, NT, VEC>(f.o.at(c.q0 + wr.query, h, w.dim), acc, w.dim);
        if (lane < 32) f.lse[(int64_t)(c.q0 + wr.query) * w.heads + h] = none ? -INFINITY : (m * c2 + __builtin_amdgcn_logf(l)) * kLn2;
    };
    pass(std::false_type{}, kFinite);
    if (__builtin_expect(!any_of_workgroup(wr.there & other_than_finite(acc)), 1)) return;
    kt.load(lds, 0, 0);
    pass(std::true_type{}, kFinite);
    // a row whose sum of exponentials is NaN is that altogether
    if (!any_of_workgroup(other) || !any_of_workgroup(wr.there & (l == l))) return;
#pragma unroll 1
    for (int part = kPlus; part <= kMinus; ++part) {
        kt.load(lds, 0, 0);
        pass(std::true_type{}, part);
        if (wr.there) join_column<T, NT>(f.o.at(c.q0 + wr.query, h, w.dim), acc, w.dim, part == kPlus ? INFINITY : -INFINITY);
    }
}

template <typename T, int NT, bool VEC, int W>
int forward_sized(const AttnFwd<T>& f, hipStream_t s) {
    const int64_t tiles = tile_numbers(f.w.n_q, f.w.clouds, f.w.group, W * kWaveRows);
    if (tiles * f.w.kv_heads > INT32_MAX) return fail(SP_ERR_UNSUPPORTED, "more than 2^31 tiles of rows");
    hipLaunchKernelGGL((attn_fwd_kernel<T, NT, VEC, W>), dim3((unsigned)(tiles * f.w.kv_heads)), dim3(64 * W), 0, s, f, (int)tiles);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T, bool VEC, int W>
int forward_wide(const AttnFwd<T>& f, hipStream_t s) {
    const int nt = (f.w.dim + 31) / 32;
    return nt == 1 ? forward_sized<T, 1, VEC, W>(f, s) : nt == 2 ? forward_sized<T, 2, VEC, W>(f, s) : nt == 3 ? forward_sized<T, 3, VEC, W>(f, s) : forward_sized<T, 4, VEC, W>(f, s);
}

template <typename T>
int forward(const AttnFwd<T>& f, hipStream_t s) {
    if (f.w.n_q == 0) return SP_OK;
    const bool vec = f.w.dim * sizeof(T) % 16 == 0 && in_pieces(f.q) && in_pieces(f.k) && in_pieces(f.v) && in_pieces(f.o);
    if (few_tiles(tile_numbers(f.w.n_q, f.w.clouds, f.w.group, 4 * kWaveRows), f.w.kv_heads))
        return vec ? forward_wide<T, true, 1>(f, s) : forward_wide<T, false, 1>(f, s);
    return vec ? forward_wide<T, true, 4>(f, s) : forward_wide<T, false, 4>(f, s);
}

int check(const sp_window_attn* a, Window* w) {
    if (!a) return fail(SP_ERR_INVALID_ARG, "the description is NULL");
    if (a->n_q < 0 || a->n_k < 0 || a->n_clouds < 0) return fail(SP_ERR_INVALID_ARG, "negative row or cloud count");
    if (a->dt != SP_F32 && a->dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads) return fail(SP_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
    if (a->dim < 1) return fail(SP_ERR_INVALID_ARG, "bad head width");
    if (a->left < 0 || a->right < 0 || a->sinks < 0) return fail(SP_ERR_INVALID_ARG, "left, right and sinks must not be negative");
    if (!(a->scale > -3.0e38f && a->scale < 3.0e38f)) return fail(SP_ERR_INVALID_ARG, "the scale must be finite");
    if (a->dim > kMaxDim || a->heads > 65535 || a->n_q > 1 << 29 || a->n_k > 1 << 29 || a->n_clouds > 1 << 29)
        return fail(SP_ERR_UNSUPPORTED, "head widths above %d, more than 65535 heads or more than 2^29 rows or clouds", kMaxDim);
    if (a->n_q * (a->heads / a->kv_heads) > 1 << 30) return fail(SP_ERR_UNSUPPORTED, "more than 2^30 rows and heads that share a key head");
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
        return attn_backward<float>({w, in<float>(d_q, ldq), in<float>(d_k, ldk), in<float>(d_v, ldv), in<float>(d_o, ldo), in<float>(d_dout, lddout),
                                d_lse, nullptr, out<float>(d_dq, lddq), out<float>(d_dk, lddk), out<float>(d_dv, lddv)}, s);
    return attn_backward<bf16_t>({w, in<bf16_t>(d_q, ldq), in<bf16_t>(d_k, ldk), in<bf16_t>(d_v, ldv), in<bf16_t>(d_o, ldo),
                             in<bf16_t>(d_dout, lddout), d_lse, nullptr, out<bf16_t>(d_dq, lddq), out<bf16_t>(d_dk, lddk),
                             out<bf16_t>(d_dv, lddv)}, s);
}

}  // extern "C"
