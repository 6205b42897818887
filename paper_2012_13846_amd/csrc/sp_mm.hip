// The entry points of the feed-forward block and of products in 8 bits, and the rule by which a product takes its workgroups.
#include <algorithm>

#include "sp_mm.h"

namespace sp {

// Workgroups of each shape, and the microseconds that a step of 128 bytes takes of one that has a CU to itself and of two that share it, as measured
// over products of 64 to 70001 rows and widths of 64 to 8192; what a product takes beside them: 3.5 us, for each round of workgroups what the first
// tiles wait for and the results' way out (2 us, 8 us where no other workgroup of the CU works meanwhile), and to join parts 3.5 us and their way to
// memory and back at 4 bytes a picosecond.
namespace {
struct Cost {
    ShapeName name;
    int bm, bn, threads;
    double alone[4], shared[4];  // by type; shared 0: a CU holds one
};
//                                f32   bf16  8 bits, and exactly
constexpr Cost kCosts[] = {{kLarge, 256, 256, 512, {7.9, 1.35, 1.7, 0}, {0, 0, 0, 0}},
                           {kMiddle, 128, 128, 256, {2.0, 0.55, 0.68, 1.15}, {4.06, 1.0, 1.13, 1.96}},
                           {kNarrow, 64, 128, 256, {1.15, 0.37, 0.55, 0.85}, {2.1, 0.65, 0.81, 1.26}},
                           {kFew, 128, 32, 256, {0.7, 0.35, 0, 0}, {1.1, 0.55, 0, 0}}};
constexpr double kLaunch = 3.5, kRound = 2, kRoundAlone = 8;
double join_time(int64_t splits, int64_t rows, int64_t n) { return 8.0 * (double)splits * (double)rows * (double)n / 4e6; }
}  // namespace

Plan mm_plan(int64_t rows, int64_t n, int64_t k_bytes, MmType type, bool pieces) {
    const int64_t steps = (k_bytes + kStepBytes - 1) / kStepBytes;
    Plan best{kMiddle, 0, (int)steps, 0, 0, kNoPlan};
    for (const Cost& kind : kCosts) {
        if (kind.name == kLarge && (!pieces || type == kQ8Exact)) continue;
        if ((kind.name == kFew) != (n <= kThinRows && type < kQ8)) continue;
        const int64_t tiles_m = (rows + kind.bm - 1) / kind.bm, tiles_n = (n + kind.bn - 1) / kind.bn, tiles = tiles_m * tiles_n;
        const int64_t most = kMostThreads / kind.threads;
        const double alone = kind.alone[type], shared = kind.shared[type];
        int64_t last = 0;
        for (int64_t want = 1; want <= 128 && want <= std::max<int64_t>(1, steps / 2); want = want < 4 ? want + 1 : want + want / 2) {
            int64_t each = std::max<int64_t>(1, (steps + want - 1) / want);
            if (type >= kQ8 && want > 1) each = (each + 3) / 4 * 4;  // a word of scales is four steps'
            const int64_t splits = std::max<int64_t>(1, (steps + each - 1) / each);
            if (splits == last || tiles * splits > most) continue;
            last = splits;
            const int64_t groups = tiles * splits, slots = shared > 0 ? 512 : 256, rest = groups % slots;
            const double round = shared > 0 ? kRound : kRoundAlone;
            double time = kLaunch + (double)(groups / slots) * ((double)each * (shared > 0 ? shared : alone) + round);
            if (rest) time += (double)each * (rest <= 256 ? alone : shared) + round;
            if (splits > 1) time += kLaunch + join_time(splits, rows, n);
            if (time < best.time) best = Plan{kind.name, (int)splits, (int)each, (int)tiles_m, (int)tiles_n, time};
        }
    }
    return best;
}

// Every workgroup has at most so many steps, whichever product it is of: those are handed out as CUs come free.
PlanThree mm_plan_three(const Size (&of)[3], MmType type, bool pieces) {
    PlanThree best{};
    double least = 0;
    for (const Size& o : of) least += mm_plan(o.rows, o.n, o.k_bytes, type, pieces).time;
    for (const Cost& kind : kCosts) {
        if (kind.name != kMiddle && kind.name != kNarrow) continue;
        const double alone = kind.alone[type], shared = kind.shared[type];
        for (int64_t most = 4; most <= 4096; most += most < 16 ? 4 : most / 2) {
            PlanThree t{true, {}};
            double work = 0, joins = 0;
            int64_t groups = 0, longest = 0;
            for (int i = 0; i < 3; ++i) {
                const int64_t steps = (of[i].k_bytes + kStepBytes - 1) / kStepBytes;
                const int64_t tiles_m = (of[i].rows + kind.bm - 1) / kind.bm, tiles_n = (of[i].n + kind.bn - 1) / kind.bn;
                const int64_t want = (steps + most - 1) / most, each = (steps + want - 1) / want, splits = (steps + each - 1) / each;
                if (tiles_m > 1 << 20 || tiles_n > 1 << 20 || splits > 128) {
                    groups = (int64_t)1 << 40;
                    break;
                }
                groups += tiles_m * tiles_n * splits;
                longest = std::max(longest, each);
                work += (double)(tiles_m * tiles_n) * ((double)steps * shared + (double)splits * kRound);
                if (splits > 1) joins += join_time(splits, of[i].rows, of[i].n) + (joins > 0 ? 0 : kLaunch);
                t.p[i] = Plan{kind.name, (int)splits, (int)each, (int)tiles_m, (int)tiles_n, 0};
            }
            if (groups > 1 << 20) continue;
            // (an uneven end: half a workgroup's time)
            const double time = kLaunch + joins + (groups <= 256 ? (double)longest * alone + kRound : std::max(work / 512 + (double)longest * shared / 2, (double)longest * shared + kRound));
            if (time < least) least = time, best = t;
        }
    }
    return best;
}

static int64_t ffn_work(int64_t n, int c, int m, int size, bool backward) {
    const MmType type = size == 4 ? kF32 : kBf16;
    int64_t part = 0;
    for (const bool pieces : {false, true}) {  // the arrays' alignment is not known yet
        if (!backward) {
            part = std::max({part, mm_work(2 * (int64_t)m, n, (int64_t)c * size, type, true, pieces), mm_work(c, n, (int64_t)m * size, type, true, pieces)});
        } else {
            const int64_t c_bytes = (int64_t)c * size, n_bytes = n * size;
            const Size of[3] = {{c, n, 2 * (int64_t)m * size}, {c, 2 * (int64_t)m, n_bytes}, {m, c, n_bytes}};
            part = std::max(part, mm_work(m, n, c_bytes, type, false, pieces));
            for (const Size& o : of) part = std::max(part, mm_work(o.rows, o.n, o.k_bytes, type, false, pieces));
            if (n > 0) part = std::max(part, mm_work_three(of, type, pieces));
        }
    }
    return part == kNoWork ? -1 : up256((backward ? 2 : 1) * n * m * size) + up256(part) + 256;
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
    const int64_t part = std::max(mm_work(m, n, wide, kQ8, true, true), mm_work(m, n, wide, kQ8Exact, true, true));
    return part == kNoWork ? -1 : up256(part) + 256;
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
