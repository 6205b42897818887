// Attention with a sliding window and a few first rows that stay visible, over packed clouds: gradients.
#include <algorithm>

#include "sp_attn_rows.h"

namespace sp {
namespace {

constexpr int kThreads = 256;  // of a workgroup that joins

// Two kernels compute the scores again, each for what it can sum without atomics: dq by rows like the forward pass (and delta = dout . o
// on the way), dk and dv by keys.  The second goes over the rows of all query heads that share the key head, so their sum needs no
// second step.

// delta = dout . o = sum of p (dout . v).  From o it has the error of o's rounding, half a step, which stands in every dS of the row and
// does not average out where few keys share it: dq and dk are 0.0027 off in bf16 with 5 to 16 keys a row and 0.0037 with two (relative
// norms; the results' own rounding is 0.0017, that of dS 0.0017 again).  Rows of at most this many keys take the sum itself, in a pass of
// its own over keys that are close by then; with more of them o's part is below 0.0007.
constexpr int kExactKeys = 128;

// Three products a pair of tiles: scores, dout . v, dS . k; accumulators, q and dout stay in registers.  The forward pass's case: 440 - 475 us
// (840 - 900 TFLOP/s of the three products), matrix pipe busy 40 %, vector pipe 36 %; heads of 32: 710 - 790 us, vector pipe 80 %.
template <typename T, int NT, bool VEC, int W>
__global__ __launch_bounds__(64 * W, NT == 1 ? 4 : sizeof(T) * NT == 4 ? 3 : sizeof(T) * NT < 16 ? 2 : 1) void attn_dq_kernel(AttnBwd<T> g, int tiles) {
    using Tl = Tile<T, NT>;
    constexpr int kN = kKeys<T, W>, kB = kN / 32, kTileBytes = kN * Tl::kRowBytes;
    __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes];
    const Window& w = g.w;
    const RowTile<W> rt(w, tiles);
    const Cloud c(w, rt.cloud);
    const int64_t rows = (int64_t)c.a * w.group;
    if (!in_cloud(rt.r0, rows)) return;
    const WaveRows<W> wr(w, c, (uint32_t)rt.r0, (uint32_t)rows);
    const Reach& reach = wr.reach;
    const int lane = threadIdx.x & 63, kh = rt.kh, h = kh * w.group + wr.head;
    const auto pl = Tl::place();
    const KeyTiles<T, NT, VEC, W> kt(w, reach, g.k, g.v, c, kh);
    int first_buf = 0;  // where the first tile is
    if (reach.n > 0) kt.load(lds, 0, 0);
    typename Tl::Frag q[Tl::kSteps], dout[Tl::kSteps];
    Tl::template load_row<VEC>(q, g.q.at(c.q0 + wr.query, h, w.dim), w.dim, wr.there, w.scale < 0.f);
    Tl::template load_row<VEC>(dout, g.dout.at(c.q0 + wr.query, h, w.dim), w.dim, wr.there, false);
    const int64_t stat = (int64_t)(c.q0 + wr.query) * w.heads + h;
    const float l2 = wr.there ? g.lse[stat] * kLog2e : 0.f, c2 = exponent_scale(w);
    float delta = 0.f;
    if (sizeof(T) == 2 && min(w.left + w.right + 1 + w.sinks, c.b) <= kExactKeys) {
        for (int slot = 0, buf = 0; slot < reach.n; slot += kN, buf ^= 1) {
            const char *keys = lds + buf * 2 * kTileBytes, *values = keys + kTileBytes;
            wait_tiles();
            kt.load(lds, slot + kN < reach.n ? slot + kN : 0, buf ^ 1);  // at last the first again
            const SeenInTile seen(w, reach, slot, wr.p);
#pragma unroll 1
            for (int b = 0; b < kB; ++b) {
                f32x16 s = {}, dp = {};
#pragma unroll
                for (int st = 0; st < Tl::kSteps; ++st) {
                    s = Tl::mma(Tl::direct(keys, pl, b, st), q[st], s);
                    dp = Tl::mma(Tl::direct(values, pl, b, st), dout[st], dp);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -l2)) * dp[i];
                    delta += seen.sees(b * 32 + 8 * (i / 4) + i % 4) ? x : 0.f;
                }
            }
            first_buf = buf ^ 1;
        }
        delta = halves<Add>(delta);
    } else {
        typename Tl::Frag o[Tl::kSteps];
        Tl::template load_row<VEC>(o, g.o.at(c.q0 + wr.query, h, w.dim), w.dim, wr.there, false);
#pragma unroll
        for (int st = 0; st < Tl::kSteps; ++st)
#pragma unroll
            for (int i = 0; i < Tl::kPer; ++i) delta = fmaf((float)o[st][i], (float)dout[st][i], delta);
        delta = halves<Add>(delta);
    }
    if (wr.there && lane < 32) g.delta[stat] = delta;
    f32x16 acc[NT];
    bool other = false;  // there are keys that are not finite
    // As in the forward pass.  Such a key's score is -infinity, its dS 0 and the product NaN, or all of the row is NaN: no signs.
    auto pass = [&](auto again, int part) {
#pragma unroll
        for (int d = 0; d < NT; ++d) acc[d] = f32x16{};
        for (int slot = 0, buf = again ? 0 : first_buf; slot < reach.n; slot += kN, buf ^= 1) {
            const char *keys = lds + buf * 2 * kTileBytes, *values = keys + kTileBytes;
            wait_tiles();
            if (slot + kN < reach.n) kt.load(lds, slot + kN, buf ^ 1);
            if (reach.none(w, slot, kN, wr.p_min, wr.p_max)) continue;
            const bool all = !again && (wr.whole & reach.all(w, slot, kN, wr.p_min, wr.p_max));
            const SeenInTile seen(w, reach, slot, wr.p);
#pragma unroll
            for (int b = 0; b < kB; ++b) {
                f32x16 s = {}, dp = {};
#pragma unroll
                for (int st = 0; st < Tl::kSteps; ++st) s = Tl::mma(Tl::direct(keys, pl, b, st), q[st], s);
#pragma unroll
                for (int st = 0; st < Tl::kSteps; ++st) dp = Tl::mma(Tl::direct(values, pl, b, st), dout[st], dp);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -l2)) * (dp[i] - delta);
                if (!all) {
                    if (!again && !seen.heads) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = seen.in_range(b * 32 + 8 * (i / 4) + i % 4) ? s[i] : 0.f;
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float x = again && part != kFinite ? 1.f : s[i];
                            s[i] = seen.sees(b * 32 + 8 * (i / 4) + i % 4) ? x : 0.f;
                        }
                    }
                }
#pragma unroll
                for (int st = 0; st < Tl::kTSteps; ++st) {
                    const auto ds = Tl::operand(s, st);
#pragma unroll
                    for (int d = 0; d < NT; ++d) {
                        auto rows = Tl::turned(keys, pl, b, st, d);
                        if constexpr (again) rows = Tl::part_of(rows, part, &other);
                        acc[d] = Tl::mma(rows, ds, acc[d]);
                    }
                }
            }
        }
        if (again && part != kFinite) return;
#pragma unroll
        for (int d = 0; d < NT; ++d) acc[d] *= w.scale;
        if (wr.there) put_column<T, NT, VEC>(g.dq.at(c.q0 + wr.query, h, w.dim), acc, w.dim);
    };
    pass(std::false_type{}, kFinite);
    if (__builtin_expect(!any_of_workgroup(wr.there & other_than_finite(acc)), 1)) return;
    kt.load(lds, 0, 0);
    pass(std::true_type{}, kFinite);
    if (!any_of_workgroup(other) || !any_of_workgroup(wr.there & (fabsf(l2) < INFINITY))) return;
    kt.load(lds, 0, 0);
    pass(std::true_type{}, kEither);
    if (wr.there) join_column<T, NT>(g.dq.at(c.q0 + wr.query, h, w.dim), acc, w.dim, NAN);
}

// The first keys of a cloud are seen by all later queries: a tile with them would take many times the others' time.  For few of them
// (at most kSplitSinks) in a long cloud the keys' kernel leaves their pairs beyond the window out and its sums in fp32 (`first`);
// attn_far_kernel adds up those pairs, a chunk of rows to a wavefront (`far`), and attn_join_kernel adds both, the chunks in order.
constexpr int kSplitSinks = 128;
// Clouds of 561 rows beyond the window: 103 us without the split, 123 with it (four clouds, 4 heads of 32, fp32, forward and
// backward); of 745 rows: 88 and 81 (one cloud, 8 heads of 64, bf16); of 1745: 144 and 119.
constexpr int kLongBeyond = 640;
// The host knows the clouds' mean, not the longest: with a lower mean the kernels look for long clouds in calls of more keys beyond the window than
// this.  Where there are none that costs 5 us (4096 to 65536 keys in clouds of 256: 31 - 1288 us in all); a cloud of 4000 keys among 100 of
// 100 takes 132 us instead of 645 (8 heads of 64 over 2), one of 60000 370 instead of 9800, with 32 heads of 128 over 8 5.1 ms instead of 21.
// In fewer keys in all, one long cloud loses 0.2 - 0.6 ms at most, and clouds a little beyond kLongBeyond gain nothing (2500 keys: 109 us, 118 split).
constexpr int kLongTotal = 4096;
struct Split {
    int sinks;           // 0: not split
    LongClouds clouds;
    float *first, *far;  // by sums_at(): [place or chunk]...
};
__device__ __forceinline__ int64_t split_at(const Window& w, const Split& sp, int64_t part, int kh, int key) {
    return sums_at(w.kv_heads, sp.sinks, w.dim, part, kh, key);
}
// the first row that sees a key of the 32 from `key` on beyond its window
__device__ __forceinline__ int64_t far_begin(const Window& w, const Cloud& c, int key) {
    return (int64_t)max(w.left + key + 1 - c.off, 0) * w.group;
}

// The rows (queries and dout) that a workgroup of the keys' kernels goes over, `step` of at most N at a time: whole queries, so that a
// row's place in its tile does not change, unless a query's heads are more than N.
template <typename T, int NT, bool VEC, int N, int THREADS>
struct QueryTiles {
    using Tl = Tile<T, NT>;
    static constexpr int kTileBytes = N * Tl::kRowBytes;
    const AttnBwd<T>& g;
    const Cloud& c;
    int kh, step;
    int end;  // the rows' end, a multiple of `group`
    TileLoads<T, NT, N, THREADS> lq, ld;
    __device__ __forceinline__ QueryTiles(const AttnBwd<T>& g_, const Cloud& c_, int kh_, int end_) : g(g_), c(c_), kh(kh_), end(end_) {
        const int group = g.w.group, row = g.w.dim * (int)sizeof(T);
        step = group <= N ? N / group * group : N;
        if constexpr (VEC) {
            const uint32_t ldq = (uint32_t)(g.q.ld * sizeof(T)), ldd = (uint32_t)(g.dout.ld * sizeof(T));
            lq.place(g.w.dim, [&](int r) { return r < step ? r / group * ldq + r % group * row : kOutside; });
            ld.place(g.w.dim, [&](int r) { return r < step ? r / group * ldd + r % group * row : kOutside; });
        }
    }
    __device__ __forceinline__ void one(char* tile, const TileLoads<T, NT, N, THREADS>& l, const Rows<const T>& t, int row) const {
        const int group = g.w.group;
        if constexpr (VEC) {
            const uint32_t i = (uint32_t)row / (uint32_t)group, left = (uint32_t)min(step, end - row) / (uint32_t)group;  // queries
            l.load(lds_address(tile), memory_of(t.at(c.q0 + i, kh * group, g.w.dim),
                                                (uint32_t)((left - 1) * t.ld + group * g.w.dim) * (uint32_t)sizeof(T)));
        } else {
            load_elements<T, NT, N, THREADS>(tile, g.w.dim, [&](int r) {
                return r < step && row + r < end ? t.at(c.q0 + (row + r) / group, kh * group + (int)((row + r) % group), g.w.dim) : nullptr;
            });
        }
    }
    __device__ __forceinline__ void load(char* tiles, int row) const {
        one(tiles, lq, g.q, row);
        one(tiles + kTileBytes, ld, g.dout, row);
    }
};

// A row's statistics on their way from memory to LDS
struct RowStat {
    float l2, delta;
    int p;
};
template <typename T>
__device__ __forceinline__ RowStat row_stat(const AttnBwd<T>& g, const Cloud& c, int kh, int row, bool there) {
    RowStat r{0.f, 0.f, kNowhere};
    if (there) {
        const int i = (int)((uint32_t)row / (uint32_t)g.w.group);
        const int64_t at = (int64_t)(c.q0 + i) * g.w.heads + kh * g.w.group + (int)((uint32_t)row % (uint32_t)g.w.group);
        r = {g.lse[at] * kLog2e, g.delta[at], i + c.off};
    }
    return r;
}
template <int N>
struct RowStats {
    __attribute__((aligned(16))) float l2[N], minus_delta[N];
    __attribute__((aligned(16))) int p[N];
    __device__ __forceinline__ void put(const RowStat& r, int at) {
        l2[at] = r.l2;
        minus_delta[at] = -r.delta;
        p[at] = r.p;
    }
};

// Keys' gradients from 32 rows after another.  VLDS: the values are read from LDS when they are needed, for heads so wide that
// registers for both would leave a SIMD one wavefront.
template <typename T, int NT, bool VLDS>
struct KeyGrads {
    using Tl = Tile<T, NT>;
    typename Tl::Frag k[Tl::kSteps], v[VLDS ? 1 : Tl::kSteps];
    const char* v_tile;  // this wavefront's 32 rows
    f32x16 dk[NT], dv[NT];
    // Probabilities and dS of rows 32 b .. of the tiles q and dout; `counts`: 1 for each pair that is seen
    template <int N, typename Seen>
    __device__ __forceinline__ void scores(f32x16& s, f32x16& dp, const char* q, const char* dout, const RowStats<N>& stats,
                                           const typename Tl::Place& pl, int b, float c2, bool all, Seen seen, bool counts = false) const {
        const int half = b * 32 + 4 * ((threadIdx.x & 63) >> 5);
        s = f32x16{};  // dp begins at -delta
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 de = *reinterpret_cast<const f32x4*>(stats.minus_delta + half + 8 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) dp[4 * g + i] = de[i];
        }
#pragma unroll
        for (int st = 0; st < Tl::kSteps; ++st) s = Tl::mma(Tl::direct(q, pl, b, st), k[st], s);
#pragma unroll
        for (int st = 0; st < Tl::kSteps; ++st)
            dp = Tl::mma(Tl::direct(dout, pl, b, st), VLDS ? Tl::direct(v_tile, pl, 0, st) : v[VLDS ? 0 : st], dp);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 l = *reinterpret_cast<const f32x4*>(stats.l2 + half + 8 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[4 * g + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + i], c2, -l[i]));
                dp[4 * g + i] *= s[4 * g + i];
            }
        }
        if (!all)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int4 p = *reinterpret_cast<const int4*>(stats.p + half + 8 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool sees = seen(i == 0 ? p.x : i == 1 ? p.y : i == 2 ? p.z : p.w);
                    s[4 * g + i] = !sees ? 0.f : counts ? 1.f : s[4 * g + i];
                    dp[4 * g + i] = !sees ? 0.f : counts ? 1.f : dp[4 * g + i];
                }
            }
    }
    __device__ __forceinline__ void products(const f32x16& s, const f32x16& dp, const char* q, const char* dout, const typename Tl::Place& pl, int b) {
#pragma unroll
        for (int st = 0; st < Tl::kTSteps; ++st) {
            const auto p = Tl::operand(s, st), ds = Tl::operand(dp, st);
#pragma unroll
            for (int d = 0; d < NT; ++d) {
                dv[d] = Tl::mma(Tl::turned(dout, pl, b, st, d), p, dv[d]);
                dk[d] = Tl::mma(Tl::turned(q, pl, b, st, d), ds, dk[d]);
            }
        }
    }
    // Where sums were not finite, one of these instead (Part): into `dv`, from rows 32 b .. of `rows`, q's or dout's.  Returns whether they had others.
    __device__ __forceinline__ bool product_of(const f32x16& shares, const char* rows, const typename Tl::Place& pl, int b, int part) {
        bool other = false;
#pragma unroll
        for (int st = 0; st < Tl::kTSteps; ++st) {
            const auto x = Tl::operand(shares, st);
#pragma unroll
            for (int d = 0; d < NT; ++d) dv[d] = Tl::mma(Tl::part_of(Tl::turned(rows, pl, b, st, d), part, &other), x, dv[d]);
        }
        return other;
    }
};

// The sums that a workgroup takes again, one after another, where they were not finite: dk's and dv's finite part; and, where rows of dout are not
// finite, how often +infinity and -infinity join dv.  A query that is not finite has scores that are not, and all of its shares are NaN: no signs.
enum Again { kDk, kDv, kDvPlus, kDvMinus, kAgain };
__device__ __forceinline__ int part_of_again(int what) { return what <= kDv ? kFinite : what == kDvPlus ? kPlus : kMinus; }

template <typename T, int NT>
constexpr bool kValuesInLds = sizeof(T) == 2 && NT >= 3;
// rows of a step: 32 where 64 do not fit the LDS beside the values of two workgroups
template <typename T, int NT, int W>
constexpr int kStepRows = sizeof(T) == 2 && NT <= 2 && W > 1 ? 64 : 32;

// Four products a pair of tiles.  A wavefront has 32 keys: 128 registers of accumulators and 32 of keys at a width of 128, which with
// the values in LDS leaves room for two wavefronts a SIMD (1455 -> 697 us on the forward pass's case; 680 - 750 now).  Bound by the latency of
// LDS reads, each right before its product for want of registers to read ahead: matrix pipe busy 31 %, vector pipe 19 %.  Reads asked
// for ahead of their products spill (2103 us in all against 1538), a higher priority for products costs 15 %; the two score products one
// after another instead of by turns give 1 - 7 %.  Heads of 32: 770 - 850 us.
template <typename T, int NT, bool VEC, int W>
__global__ __launch_bounds__(64 * W, NT == 1 ? (sizeof(T) == 2 ? 4 : 3) : sizeof(T) * NT == 4 ? 3 : sizeof(T) * NT <= 8 ? 2 : 1) void attn_dkv_kernel(AttnBwd<T> g, Split split, int tiles) {
    using Tl = Tile<T, NT>;
    constexpr bool kVLds = kValuesInLds<T, NT>;
    constexpr int kRows = W * kWaveRows, kN = kStepRows<T, NT, W>, kB = kN / 32, kTileBytes = kN * Tl::kRowBytes;
    __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes];
    __shared__ __attribute__((aligned(1024))) char values[kVLds ? kRows * Tl::kRowBytes : 16];
    __shared__ RowStats<kN> stats[2];
    const Window& w = g.w;
    const uint32_t item = item_of_block(blockIdx.x, gridDim.x), t = item % (uint32_t)tiles;
    const int kh = (int)(item / (uint32_t)tiles);
    const CloudTile ct(w.k_starts, w.clouds, w.n_k, t, 1, kRows);
    const int cn = ct.cloud;
    const Cloud c(w, cn);
    if (!in_cloud(ct.row, c.b)) return;
    const int j0 = (int)ct.row, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int jw = j0 + wave * kWaveRows, j = jw + (lane & 31);
    const bool there = j < c.b, split_here = split.sinks > 0 && split.clouds.has(cn);
    const int sinks = split_here ? 0 : w.sinks;
    // the rows that see a key of the workgroup's
    const int a = c.partners ? c.a : 0;
    const int i0 = min(max(j0 - w.right - c.off, 0), a), i1 = j0 < sinks ? a : max(i0, min(max(min(j0 + kRows, c.b) + w.left - c.off, 0), a));
    const int begin = i0 * w.group, end = i1 * w.group;
    const auto pl = Tl::place();
    const QueryTiles<T, NT, VEC, kN, 64 * W> qt(g, c, kh, end);
    KeyGrads<T, NT, kVLds> kg;
    const float c2 = exponent_scale(w);
    bool other = false;  // there are rows of dout that are not finite
    auto stat_of = [&](int row) {
        const int thread = threadIdx.x;
        return row_stat(g, c, kh, row + thread, (thread < qt.step) & (row + thread < end));
    };
    // Workgroups of neighbouring keys see mostly the same rows, more of them than a chiplet's L2 holds.  Each goes round its steps from
    // the one whose number among all rows' steps is a multiple of their count, so that those that run together read a row together.
    const int steps = (end - begin + qt.step - 1) / qt.step, past = steps > 0 ? begin / qt.step % steps : 0, turn = past ? steps - past : 0;
    auto row_of = [&](int n) { return begin + (n + turn < steps ? n + turn : n + turn - steps) * qt.step; };
    auto start = [&] {
        if (begin < end) {
            qt.load(lds, row_of(0));
            const RowStat r = stat_of(row_of(0));
            if (threadIdx.x < kN) stats[0].put(r, threadIdx.x);
        }
    };
    start();
    Tl::template load_row<VEC>(kg.k, g.k.at(c.k0 + j, kh, w.dim), w.dim, there, w.scale < 0.f);
    if constexpr (kVLds) {
        const T* v = g.v.at(c.k0 + j0, kh, w.dim);
        const int64_t ldv = g.v.ld;
        if constexpr (VEC) {
            TileLoads<T, NT, kRows, 64 * W> lv;
            lv.place(w.dim, [&](int r) { return r * (uint32_t)(ldv * sizeof(T)); });
            lv.load(lds_address(values), memory_of(v, (uint32_t)((min(kRows, c.b - j0) - 1) * ldv + w.dim) * (uint32_t)sizeof(T)));
        } else {
            load_elements<T, NT, kRows, 64 * W>(values, w.dim, [&](int r) { return j0 + r < c.b ? v + r * ldv : nullptr; });
        }
        kg.v_tile = values + wave * kWaveRows * Tl::kRowBytes;
        if (begin >= end) wait_tiles();  // no workgroup ends with a load on its way
    } else {
        Tl::template load_row<VEC>(kg.v, g.v.at(c.k0 + j, kh, w.dim), w.dim, there, false);
    }
    // j - right <= p <= j + left, for the first keys all p behind
    const int low = j - w.right;
    const uint32_t width = j < sinks ? 0x7fffffffu : (uint32_t)(w.left + w.right);
    auto pass = [&](auto again, int what) {
#pragma unroll
        for (int d = 0; d < NT; ++d) kg.dk[d] = kg.dv[d] = f32x16{};
        int buf = 0;
        for (int n = 0; n < steps; ++n, buf ^= 1) {
            const int row = row_of(n);
            const char *q = lds + buf * 2 * kTileBytes, *dout = q + kTileBytes;
            wait_tiles();
            RowStat next{};
            const bool more = n + 1 < steps;
            if (more) {
                qt.load(lds + (buf ^ 1) * 2 * kTileBytes, row_of(n + 1));
                next = stat_of(row_of(n + 1));
            }
            const int p_min = (int)((uint32_t)row / (uint32_t)w.group) + c.off;
            const int p_max = (int)((uint32_t)(min(row + qt.step, end) - 1) / (uint32_t)w.group) + c.off;
            const bool none = (jw >= c.b) | (jw > p_max + w.right) | ((jw + kWaveRows - 1 < p_min - w.left) & (jw >= sinks));
            const bool all = !again && ((row + kN <= end) & (qt.step == kN) & (jw + kWaveRows - 1 <= p_min + w.right) & (jw >= p_max - w.left));
            const auto seen = [&](int p) { return (uint32_t)(p - low) <= width; };
            if (!none)
#pragma unroll 1
                for (int b = 0; b < kB; ++b) {
                    f32x16 s, dp;
                    kg.scores(s, dp, q, dout, stats[buf], pl, b, c2, all, seen, again && what > kDv);
                    if constexpr (again) other |= kg.product_of(what == kDk ? dp : s, what == kDk ? q : dout, pl, b, part_of_again(what)) & (what == kDv);
                    else kg.products(s, dp, q, dout, pl, b);
                }
            if (more && threadIdx.x < kN) stats[buf ^ 1].put(next, threadIdx.x);
        }
        if (again) __syncthreads();
    };
    const bool part = split_here && j < split.sinks;
    // of this key's dk (0) and dv (1)
    auto sums = [&](int which) { return split.first + split_at(w, split, split.clouds.place(cn), kh, j) + which * w.dim; };
    auto row = [&](int which) { return which ? g.dv.at(c.k0 + j, kh, w.dim) : g.dk.at(c.k0 + j, kh, w.dim); };
    auto store = [&](int which, const f32x16(&acc)[NT]) {
        if (there && part) put_column<float, NT, false>(sums(which), acc, w.dim);
        else if (there) put_column<T, NT, VEC>(row(which), acc, w.dim);
    };
    auto scaled = [&](f32x16(&acc)[NT]) {
#pragma unroll
        for (int d = 0; d < NT; ++d) acc[d] *= w.scale;
    };
    pass(std::false_type{}, 0);
    scaled(kg.dk);
    store(0, kg.dk);
    store(1, kg.dv);
    if (__builtin_expect(!any_of_workgroup(there & other_than_finite(kg.dk, kg.dv)), 1)) return;
#pragma unroll 1
    for (int what = kDk; what < kAgain; ++what) {
        if (what == kDvPlus && !any_of_workgroup(other)) break;
        start();
        pass(std::true_type{}, what);
        if (what <= kDv) {
            if (what == kDk) scaled(kg.dv);
            store(what, kg.dv);
        } else if (there && part) {
            join_column<float, NT>(sums(1), kg.dv, w.dim, what == kDvPlus ? INFINITY : -INFINITY);
        } else if (there) {
            join_column<T, NT>(row(1), kg.dv, w.dim, what == kDvPlus ? INFINITY : -INFINITY);
        }
    }
}

// Reads every row once for a few keys: bound by memory's latency at one or two wavefronts a SIMD (373601 rows of 8 heads of 32: 147 us,
// 2.6 TB/s; 16384 of 32 of 128: 55 - 59 us, 4.6 - 4.9 TB/s).  Without the split the tile of the first keys alone would go over all rows.
template <typename T, int NT, bool VEC>
__global__ __launch_bounds__(64, 1) void attn_far_kernel(AttnBwd<T> g, Split split, int tiles) {
    using Tl = Tile<T, NT>;
    constexpr int kTileBytes = 32 * Tl::kRowBytes;
    __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes];
    __shared__ RowStats<32> stats[2];
    const Window& w = g.w;
    const uint32_t item = item_of_block(blockIdx.x, gridDim.x), t = item % (uint32_t)tiles;
    const int groups = (split.sinks + 31) / 32, key0 = (int)(item / (uint32_t)tiles) % groups * 32, kh = (int)(item / (uint32_t)tiles) / groups;
    const LongClouds& lc = split.clouds;
    const int cn = find_cloud(w.clouds, t, [&](int i) { return lc.first_chunk(i); });
    const Cloud c(w, cn);
    const int64_t r0 = (t - lc.first_chunk(cn)) * lc.chunk, rows = (int64_t)c.a * w.group;
    if (!lc.has(cn) || !in_cloud(r0, rows)) return;
    const int64_t from = max(r0, far_begin(w, c, key0)), to_row = min(r0 + lc.chunk, rows);
    if (from >= to_row) return;
    const int begin = (int)from, end = (int)to_row;
    const int lane = threadIdx.x, j = key0 + (lane & 31);
    const bool there = j < min(split.sinks, c.b);
    const auto pl = Tl::place();
    const QueryTiles<T, NT, VEC, 32, 64> qt(g, c, kh, end);
    KeyGrads<T, NT, false> kg;
    auto stat_of = [&](int row) { return row_stat(g, c, kh, row + lane, (lane < qt.step) & (row + lane < end)); };
    auto start = [&] {
        wait_own_tiles();  // nothing of an earlier pass is still read
        qt.load(lds, begin);
        const RowStat r = stat_of(begin);
        if (lane < 32) stats[0].put(r, lane);
    };
    start();
    Tl::template load_row<VEC>(kg.k, g.k.at(c.k0 + j, kh, w.dim), w.dim, there, w.scale < 0.f);
    Tl::template load_row<VEC>(kg.v, g.v.at(c.k0 + j, kh, w.dim), w.dim, there, false);
    const float c2 = exponent_scale(w);
    bool other = false;
    auto pass = [&](auto again, int what) {  // as in the keys' kernel
#pragma unroll
        for (int d = 0; d < NT; ++d) kg.dk[d] = kg.dv[d] = f32x16{};
        int buf = 0;
        for (int row = begin; row < end; row += qt.step, buf ^= 1) {
            wait_own_tiles();
            RowStat next{};
            const bool more = row + qt.step < end;
            if (more) {
                qt.load(lds + (buf ^ 1) * 2 * kTileBytes, row + qt.step);
                next = stat_of(row + qt.step);
            }
            const char *q = lds + buf * 2 * kTileBytes, *dout = q + kTileBytes;
            const bool all = !again && ((row + 32 <= end) & (qt.step == 32) & (key0 + 31 < (int)((uint32_t)row / (uint32_t)w.group) + c.off - w.left));
            f32x16 s, dp;
            kg.scores(s, dp, q, dout, stats[buf], pl, 0, c2, all, [&](int p) { return j < p - w.left; }, again && what > kDv);
            if constexpr (again) other |= kg.product_of(what == kDk ? dp : s, what == kDk ? q : dout, pl, 0, part_of_again(what)) & (what == kDv);
            else kg.products(s, dp, q, dout, pl, 0);
            if (more && lane < 32) stats[buf ^ 1].put(next, lane);
        }
    };
    float* const sums = split.far + split_at(w, split, t, kh, j);  // dk's, then dv's
    auto scaled = [&](f32x16(&acc)[NT]) {
#pragma unroll
        for (int d = 0; d < NT; ++d) acc[d] *= w.scale;
    };
    pass(std::false_type{}, 0);
    scaled(kg.dk);
    if (there) {
        put_column<float, NT, false>(sums, kg.dk, w.dim);
        put_column<float, NT, false>(sums + w.dim, kg.dv, w.dim);
    }
    if (__builtin_expect(!__any(there & other_than_finite(kg.dk, kg.dv)), 1)) return;
#pragma unroll 1
    for (int what = kDk; what < kAgain; ++what) {
        if (what == kDvPlus && !__any(other)) break;
        start();
        pass(std::true_type{}, what);
        if (what == kDk) scaled(kg.dv);
        if (!there) continue;
        if (what <= kDv) put_column<float, NT, false>(sums + what * w.dim, kg.dv, w.dim);
        else join_column<float, NT>(sums + w.dim, kg.dv, w.dim, what == kDvPlus ? INFINITY : -INFINITY);
    }
}

// a workgroup a place, key head and one of the first keys: every wavefront a quarter of the chunks
template <typename T>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnBwd<T> g, Split split) {
    __shared__ float sums[4][2 * kMaxDim];
    const Window& w = g.w;
    const LongClouds& lc = split.clouds;
    const int place = blockIdx.x, kh = blockIdx.y, j = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int cn = lc.by_number() ? place + 1 : find_cloud(w.clouds, place, [&](int i) { return lc.place(i); });
    if (!lc.has(cn) || lc.place(cn) != place) return;
    const Cloud c(w, cn);
    if (j >= c.b) return;
    const int64_t t0 = lc.first_chunk(cn), rows = (int64_t)c.a * w.group;
    const int64_t far0 = far_begin(w, c, j / 32 * 32);
    // chunks with a row behind far0 were written
    const int64_t u0 = min(far0, rows) / lc.chunk, u1 = far0 < rows ? (rows + lc.chunk - 1) / lc.chunk : u0;
    const int64_t quarter = (u1 - u0 + 3) / 4, v0 = min(u0 + wave * quarter, u1), v1 = min(v0 + quarter, u1);
    const float* far = split.far + split_at(w, split, t0, kh, j);
    const int64_t step = split_at(w, split, 1, 0, 0);
    for (int at = lane; at < 2 * w.dim; at += 64) {
        float s = 0.f;
#pragma unroll 16
        for (int64_t u = v0; u < v1; ++u) s += far[u * step + at];
        sums[wave][at] = s;
    }
    __syncthreads();
    if (wave) return;
    const float* first = split.first + split_at(w, split, place, kh, j);
    T* const to[2] = {g.dk.at(c.k0 + j, kh, w.dim), g.dv.at(c.k0 + j, kh, w.dim)};
    for (int q = 0; q < 2; ++q)
        for (int e = lane; e < w.dim; e += 64) {
            const int at = q * w.dim + e;
            float s = first[at];
            for (int k = 0; k < 4; ++k) s += sums[k][at];
            to[q][e] = to_elem<T>(s);
        }
}

template <typename T, int NT, bool VEC, int W>
int backward_sized(AttnBwd<T> g, hipStream_t s) {
    const Window& w = g.w;
    const int64_t q_tiles = tile_numbers(w.n_q, w.clouds, w.group, W * kWaveRows), k_tiles = tile_numbers(w.n_k, w.clouds, 1, W * kWaveRows);
    if (std::max(q_tiles, k_tiles) * w.kv_heads > INT32_MAX) return fail(SP_ERR_UNSUPPORTED, "more than 2^31 tiles of rows");
    Buf delta = dev_alloc((size_t)w.n_q * w.heads * 4, s), parts;
    if (!delta) return SP_ERR_ALLOC;
    g.delta = ptr<float>(delta);
    // rows of a chunk: enough chunks to fill the chip, whose sums are a quarter of the rows that they read at most
    const int64_t fill = (int64_t)w.n_q * w.heads / 1024;
    const int chunk = (int)std::min<int64_t>(std::max<int64_t>(fill, std::max(128, 8 * std::min(w.sinks, kSplitSinks))), 1024);
    Split split{0, {w.q_starts, w.k_starts, w.n_q, w.n_k, w.clouds, w.group, (chunk + w.group - 1) / w.group * w.group, w.left + kLongBeyond + 1}, nullptr, nullptr};
    const LongClouds& lc = split.clouds;
    const int groups = (w.sinks + 31) / 32;
    if (w.sinks > 0 && w.sinks <= kSplitSinks && w.n_q > 0 && w.clouds > 0 &&
        (w.n_k / w.clouds >= lc.least || w.n_k - w.left > kLongTotal)) {
        const size_t each = (size_t)w.kv_heads * w.sinks * 2 * w.dim;
        parts = dev_alloc((lc.chunks() + lc.places()) * each * 4, s);
        if (parts) {  // else the slow way, which needs no memory
            split.sinks = w.sinks;
            split.first = ptr<float>(parts);
            split.far = split.first + lc.places() * each;
        }
    }
    if (w.n_q > 0)
        hipLaunchKernelGGL((attn_dq_kernel<T, NT, VEC, W>), dim3((unsigned)(q_tiles * w.kv_heads)), dim3(64 * W), 0, s, g, (int)q_tiles);
    if (w.n_k > 0)
        hipLaunchKernelGGL((attn_dkv_kernel<T, NT, VEC, W>), dim3((unsigned)(k_tiles * w.kv_heads)), dim3(64 * W), 0, s, g, split, (int)k_tiles);
    if (split.sinks) {
        hipLaunchKernelGGL((attn_far_kernel<T, NT, VEC>), dim3((unsigned)(lc.chunks() * w.kv_heads * groups)), dim3(64), 0, s, g, split, (int)lc.chunks());
        hipLaunchKernelGGL(attn_join_kernel<T>, dim3(lc.places(), w.kv_heads, split.sinks), dim3(kThreads), 0, s, g, split);
    }
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T, bool VEC, int W>
int backward_wide(const AttnBwd<T>& g, hipStream_t s) {
    const int nt = (g.w.dim + 31) / 32;
    return nt == 1 ? backward_sized<T, 1, VEC, W>(g, s) : nt == 2 ? backward_sized<T, 2, VEC, W>(g, s) : nt == 3 ? backward_sized<T, 3, VEC, W>(g, s) : backward_sized<T, 4, VEC, W>(g, s);
}

}  // namespace

template <typename T>
int attn_backward(const AttnBwd<T>& g, hipStream_t s) {
    const bool vec = g.w.dim * sizeof(T) % 16 == 0 && in_pieces(g.q) && in_pieces(g.k) && in_pieces(g.v) && in_pieces(g.o) && in_pieces(g.dout) &&
                     in_pieces(g.dq) && in_pieces(g.dk) && in_pieces(g.dv) && g.w.group <= 32;
    const int64_t tiles = std::max(tile_numbers(g.w.n_q, g.w.clouds, g.w.group, 4 * kWaveRows), tile_numbers(g.w.n_k, g.w.clouds, 1, 4 * kWaveRows));
    if (few_tiles(tiles, g.w.kv_heads)) return vec ? backward_wide<T, true, 1>(g, s) : backward_wide<T, false, 1>(g, s);
    return vec ? backward_wide<T, true, 4>(g, s) : backward_wide<T, false, 4>(g, s);
}
template int attn_backward<float>(const AttnBwd<float>&, hipStream_t);
template int attn_backward<bf16_t>(const AttnBwd<bf16_t>&, hipStream_t);

}  // namespace sp
