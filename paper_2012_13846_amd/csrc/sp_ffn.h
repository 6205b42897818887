// The gated feed-forward block's passes over a storage type; included by one file a type.
//   forward   [g u] = x W_in^T, h = act(g) * u (one product, its last step), y = h W_out^T
//   backward  dh = dy W_out, whose last step makes dg = dh * u * act'(g) and du = dh * act(g) from the g and u that were kept;
//             dx = [dg du] W_in, dW_in = [dg du]^T x, dW_out = dy^T h, which do not wait for each other: in one launch where that is faster
// Forward 6 n c m operations, with the gradients 18 n c m, at 8192 x 2048 x 8192 in bf16 2.1 ms (1170 TFLOP/s; the products alone by a library 1.7).
// h is kept beside g and u: made again from these as they were rounded it would be off by their rounding, too (dW_out 4e-3 instead of 2e-3).
#pragma once

#include "sp_mm.h"

namespace sp {

template <typename T>
int ffn_fwd(const Ffn& f, hipStream_t s) {
    constexpr int E = sizeof(T);
    T* h = f.kept ? static_cast<T*>(f.kept) + 2 * f.m : reinterpret_cast<T*>(f.work);
    const int64_t ldh = f.kept ? kKept<T> * (int64_t)f.m : f.m;
    float* part = reinterpret_cast<float*>(f.work + (f.kept ? 0 : up256(f.n * f.m * E)));
    Mm a{};
    a.first = f.w_in, a.ld_first = (int64_t)f.c * E, a.second = f.x, a.ld_second = (int64_t)f.c * E;
    a.m = f.m, a.n = (int)f.n, a.k = f.c, a.last = kGate, a.out = h, a.ld = ldh, a.kept = f.kept, a.act = f.act;
    SP_TRY((mm<T, false, false>(a, part, s)));
    Mm b{};
    b.first = f.w_out, b.ld_first = (int64_t)f.m * E, b.second = h, b.ld_second = ldh * E;
    b.m = f.c, b.n = (int)f.n, b.k = f.m, b.last = kStore, b.out = f.y, b.ld = f.c;
    return mm<T, false, false>(b, part, s);
}

template <typename T>
int ffn_bwd(const Ffn& f, hipStream_t s) {
    constexpr int E = sizeof(T);
    const T* h = static_cast<const T*>(f.kept) + 2 * f.m;
    T* dgu = reinterpret_cast<T*>(f.work);
    char* part = f.work + up256(2 * f.n * f.m * E);
    const int64_t row_c = (int64_t)f.c * E, row_m = (int64_t)f.m * E;
    Mm of[3] = {};
    Mm &x = of[0], &in = of[1], &out = of[2];
    x.first = f.w_in, x.ld_first = row_c, x.second = dgu, x.ld_second = 2 * row_m;
    x.m = f.c, x.n = (int)f.n, x.k = 2 * f.m, x.last = kStore, x.out = f.dx, x.ld = f.c;
    in.first = f.x, in.ld_first = row_c, in.second = dgu, in.ld_second = 2 * row_m;
    in.m = f.c, in.n = 2 * f.m, in.k = (int)f.n, in.last = kStore, in.out = f.dw_in, in.ld = f.c;
    out.first = h, out.ld_first = kKept<T> * row_m, out.second = f.dy, out.ld_second = row_c;
    out.m = f.m, out.n = f.c, out.k = (int)f.n, out.last = kStore, out.out = f.dw_out, out.ld = f.m;
    if (f.n == 0) {
        SP_TRY((mm<T, true, true>(in, reinterpret_cast<float*>(part), s)));
        return mm<T, true, true>(out, reinterpret_cast<float*>(part), s);
    }
    Mm a{};
    a.first = f.w_out, a.ld_first = row_m, a.second = f.dy, a.ld_second = row_c;
    a.m = f.m, a.n = (int)f.n, a.k = f.c, a.last = kGateBack, a.kept = f.kept, a.dgu = dgu, a.act = f.act;
    SP_TRY((mm<T, true, false>(a, reinterpret_cast<float*>(part), s)));
    return mm_three<T>(of, part, s);
}

}  // namespace sp
