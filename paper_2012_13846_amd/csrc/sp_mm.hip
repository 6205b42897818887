// The entry points of the feed-forward block and of products in 8 bits, and the rule by which a product takes its workgroups.
#include <algorithm>

#include "sp_mm.h"

namespace sp {

Plan mm_plan(int64_t rows, int64_t n, int64_t k_bytes, int size, bool pieces) {
    const int64_t steps = (k_bytes + kStepBytes - 1) / kStepBytes;
    struct Kind2 {
        ShapeName name;
        int bm, bn;
        double step;  // clocks a step of a workgroup takes of a CU that is full of them
        double alone; // ... and of a CU that has no other
    };
    // A CU multiplies 64 x 64 blocks of a step of 128 bytes in 128 clocks (fp32: 1024).
    const double unit = size == 4 ? 1024 : 128;
    const Kind2 kinds[] = {{kLarge, 256, 256, 16 * unit * 1.25, 16 * unit * 1.25},
                           {kMiddle, 128, 128, 4 * unit * 1.5, std::max(4 * unit * 1.5, 1000.0)},
                           {kNarrow, 64, 128, 2 * unit * 1.7, std::max(2 * unit * 1.7, 800.0)},
                           {kFew, 128, 32, std::max(unit * 2, 2000.0), std::max(unit * 2, 2000.0)}};
    Plan best{kMiddle, 1, (int)steps, 1, 1};
    double least = 1e300;
    for (const Kind2& kind : kinds) {
        if (kind.name == kLarge && !pieces) continue;
        if ((kind.name == kFew) != (n <= 32)) continue;
        const int64_t tiles_m = (rows + kind.bm - 1) / kind.bm, tiles_n = (n + kind.bn - 1) / kind.bn, tiles = tiles_m * tiles_n;
        if (tiles > 0x7fffffff) continue;
        int64_t last = 0;
        for (int64_t want = 1; want <= 64 && want <= std::max<int64_t>(1, steps / 2); want = want < 4 ? want + 1 : want + want / 2) {
            const int64_t each = std::max<int64_t>(1, (steps + want - 1) / want), splits = std::max<int64_t>(1, (steps + each - 1) / each);
            if (splits == last || tiles * splits > 0x7fffffff) continue;
            last = splits;
            const bool join = splits > 1;
            const double rounds = (double)((tiles * splits + 255) / 256);
            const double time = rounds * each * (rounds > 1 ? kind.step : kind.alone) + 3000 + (join ? 8000 + 8.0 * splits * rows * n / 2300 : 0);
            if (time < least) {
                least = time;
                best = Plan{kind.name, (int)splits, (int)each, (int)tiles_m, (int)tiles_n};
            }
        }
    }
    return best;
}

static int64_t ffn_work(int64_t n, int c, int m, int size, bool backward) {
    int64_t part = 0;
    for (const bool pieces : {false, true}) {  // the arrays' alignment is not known yet
        if (!backward) {
            part = std::max({part, mm_work(2 * (int64_t)m, n, (int64_t)c * size, size, true, pieces), mm_work(c, n, (int64_t)m * size, size, true, pieces)});
        } else {
            part = std::max({part, mm_work(m, n, (int64_t)c * size, size, false, pieces), mm_work(c, n, 2 * (int64_t)m * size, size, false, pieces),
                             mm_work(c, 2 * (int64_t)m, n * size, size, false, pieces), mm_work(m, c, n * size, size, false, pieces)});
        }
    }
    return up256((backward ? 2 : 1) * n * m * size) + up256(part) + 256;
}

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;
constexpr int64_t kMostRow = (int64_t)1 << 22;  // bytes: 256 rows lie within the 2^31 that a load's offset may say

int check(const sp_ffn* f) {
    if (!f) return fail(SP_ERR_INVALID_ARG, "the description is NULL");
    if (f->dt != SP_F32 && f->dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (f->act != SP_GATE_SILU && f->act != SP_GATE_GELU) return fail(SP_ERR_INVALID_ARG, "bad gate");
    if (f->n < 0 || f->c < 1 || f->m < 1) return fail(SP_ERR_INVALID_ARG, "bad row or channel count");
    if (f->n > kMostRows || f->c > 1 << 18 || f->m > 1 << 18)
        return fail(SP_ERR_UNSUPPORTED, "more than 2^30 rows, or a width beyond 2^18");
    return SP_OK;
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" {

int64_t sp_ffn_work_bytes(const sp_ffn* f, int32_t backward) {
    if (check(f) != SP_OK) return -1;
    return ffn_work(f->n, f->c, f->m, f->dt == SP_F32 ? 4 : 2, backward != 0);
}

int sp_ffn_fwd(const sp_ffn* f, const void* d_x, const void* d_w_in, const void* d_w_out, void* d_kept, void* d_y, void* d_work, void* stream) {
    SP_TRY(check(f));
    if (f->n == 0) return SP_OK;
    if (!d_x || !d_w_in || !d_w_out || !d_y || !d_work) return fail(SP_ERR_INVALID_ARG, "a feature/weight/work pointer is NULL");
    if ((uintptr_t)d_work % 256) return fail(SP_ERR_INVALID_ARG, "the work memory must be 256-byte aligned");
    const Ffn a{f->n, f->c, f->m, f->act, d_x, d_w_in, d_w_out, nullptr, d_kept, d_y, nullptr, nullptr, nullptr, static_cast<char*>(d_work)};
    return f->dt == SP_F32 ? ffn_fwd<float>(a, (hipStream_t)stream) : ffn_fwd<bf16_t>(a, (hipStream_t)stream);
}

int sp_ffn_bwd(const sp_ffn* f, const void* d_x, const void* d_w_in, const void* d_w_out, const void* d_kept, const void* d_dy, void* d_dx,
               void* d_dw_in, void* d_dw_out, void* d_work, void* stream) {
    SP_TRY(check(f));
    if (!d_w_in || !d_w_out || !d_dw_in || !d_dw_out || !d_work || (f->n > 0 && (!d_x || !d_kept || !d_dy || !d_dx)))
        return fail(SP_ERR_INVALID_ARG, "a feature/weight/gradient/work pointer is NULL");
    if ((uintptr_t)d_work % 256) return fail(SP_ERR_INVALID_ARG, "the work memory must be 256-byte aligned");
    const Ffn a{f->n, f->c, f->m, f->act, d_x, d_w_in, d_w_out, d_dy, const_cast<void*>(d_kept), nullptr, d_dx, d_dw_in, d_dw_out, static_cast<char*>(d_work)};
    return f->dt == SP_F32 ? ffn_bwd<float>(a, (hipStream_t)stream) : ffn_bwd<bf16_t>(a, (hipStream_t)stream);
}

int64_t sp_q8_linear_work(int64_t n, int64_t c, int64_t m) {
    if (n < 0 || n > kMostRows || c < 1 || c > kMostRow || m < 1 || m > kMostRows) return -1;
    const int64_t wide = q8_blocks(c) * kQ8Block;  // the results' type is not known yet
    return up256(std::max(mm_work(m, n, wide, 1, true, true), mm_work(m, n, wide, 1, true, false))) + 256;
}

int sp_q8_linear(const uint8_t* d_q, const uint8_t* d_scales, int64_t n, int64_t c, const uint8_t* d_wq, const uint8_t* d_wscales, int64_t m,
                 void* d_y, sp_dtype dt, void* d_work, void* stream) {
    if (n < 0 || c < 1 || m < 1) return fail(SP_ERR_INVALID_ARG, "bad row or channel count");
    if (dt != SP_F32 && dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (n > kMostRows || m > kMostRows || c > kMostRow) return fail(SP_ERR_UNSUPPORTED, "more than 2^30 rows, or rows of more than 2^22 elements");
    if (n == 0) return SP_OK;
    if (!d_q || !d_scales || !d_wq || !d_wscales || !d_y || !d_work) return fail(SP_ERR_INVALID_ARG, "a code/scale/feature/work pointer is NULL");
    if (!aligned16(d_q) || !aligned16(d_wq) || (uintptr_t)d_scales % 4 || (uintptr_t)d_wscales % 4 || (uintptr_t)d_work % 256)
        return fail(SP_ERR_INVALID_ARG, "codes must be 16-byte, scales 4-byte and the work memory 256-byte aligned");
    Mm a{};
    const int64_t wide = q8_blocks(c) * kQ8Block;
    a.first = d_wq, a.ld_first = wide, a.second = d_q, a.ld_second = wide;
    a.m = (int)m, a.n = (int)n, a.k = (int)wide, a.last = kStore, a.out = d_y, a.ld = m, a.out_f32 = dt == SP_F32;
    a.first_scales = d_wscales, a.second_scales = d_scales, a.scales = (int)q8_scales(c);
    return mm<q8_t, false, false>(a, static_cast<float*>(d_work), (hipStream_t)stream);
}

}  // extern "C"
