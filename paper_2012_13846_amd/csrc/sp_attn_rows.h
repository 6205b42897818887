// A workgroup's rows of the windowed attention, the keys that they see, and these keys' way to LDS.
#pragma once

#include "sp_attn_tile.h"

namespace sp {

// A workgroup of W wavefronts has 32 W rows of one key head: a row is a query and one of the `group` query heads that share the key head, so that keys
// and values in LDS serve all of them and a tile of few queries sees few keys.  A wavefront has 32 of these rows, and goes over the
// keys that any row of the workgroup sees, 64 (bf16, W = 4) or 32 at a time; the next keys are on their way to LDS meanwhile.
template <typename T, int W>
constexpr int kKeys = sizeof(T) == 2 && W > 1 ? 64 : 32;
constexpr int kWaveRows = 32;
constexpr int kNowhere = -(1 << 30);  // the position of a row that is none: sees nothing

// What a workgroup's rows see: the slots of its tiles are the first keys, then a stretch.
struct Reach {
    int first, lo, n;
    __device__ __forceinline__ Reach(const Window& w, const Cloud& c, int p_min, int p_max) {
        const int hi = c.partners ? min(max(p_max + w.right + 1, 0), c.b) : 0;
        lo = min(max(p_min - w.left, 0), hi);
        first = min(w.sinks, lo);
        n = first + hi - lo;
    }
    __device__ __forceinline__ int key(int slot) const { return slot + (slot < first ? 0 : lo - first); }
    // whether rows at positions p_min .. p_max see all (none) of the `count` keys from `slot` on
    __device__ __forceinline__ bool all(const Window& w, int slot, int count, int p_min, int p_max) const {
        const int k = key(slot);
        return (slot >= first) & (slot + count <= n) & (k >= p_max - w.left) & (k + count - 1 <= p_min + w.right);
    }
    __device__ __forceinline__ bool none(const Window& w, int slot, int count, int p_min, int p_max) const {
        const int k = key(slot);
        return (k >= w.sinks) & ((k > p_max + w.right) | (k + count - 1 < p_min - w.left));
    }
};

// Whether a lane's row sees the keys of a tile, by the key's number in the tile (8 g + i: the lane's half is in the borders): a range,
// and the first `head` of them where the tile has first keys (`heads`).  First keys before a gap are seen by every row of the workgroup:
// the window of its first row begins behind them.  Without a gap a slot is its key, and its border is the range's upper one too.
struct SeenInTile {
    int low, head;
    uint32_t width;
    bool heads;
    __device__ __forceinline__ SeenInTile(const Window& w, const Reach& reach, int slot, int p) {
        const int half = 4 * ((int)(threadIdx.x & 63) >> 5), k = slot + reach.lo - reach.first;
        const int high = min(p + w.right - k, reach.n - slot - 1);
        low = p - w.left - k;
        width = high >= low ? (uint32_t)(high - low) + 1 : 0;
        const bool gap = reach.lo >= w.sinks;
        head = gap ? reach.first - slot : min(w.sinks - slot, high + 1);
        heads = (gap ? reach.first : w.sinks) > slot;
        low -= half;
        head -= half;
    }
    __device__ __forceinline__ bool in_range(int r) const { return (uint32_t)(r - low) < width; }
    __device__ __forceinline__ bool sees(int r) const { return in_range(r) | (r < head); }
};

__device__ __forceinline__ float exponent_scale(const Window& w) {
    // exp2 of score * this; not quite zero for a scale of zero, so that a hidden key's -infinity stays one.  The scale's sign is the
    // operand's: rows are negated when they are loaded.
    return fmaxf(fabsf(w.scale) * kLog2e, 1e-30f);
}

// A workgroup's tile of rows
template <int W>
struct RowTile {
    int kh, cloud;
    int64_t r0;
    __device__ __forceinline__ RowTile(const Window& w, int tiles) {
        const uint32_t item = item_of_block(blockIdx.x, gridDim.x), t = item % (uint32_t)tiles;
        kh = (int)(item / (uint32_t)tiles);
        const CloudTile ct(w.q_starts, w.clouds, w.n_q, t, w.group, W * kWaveRows);
        cloud = ct.cloud;
        r0 = ct.row;
    }
};

// A lane's row of a workgroup's tile, its wavefront's positions and what the workgroup sees.  (Rows of a cloud are counted from its
// first; a cloud has at most 2^31 of them.)
template <int W>
struct WaveRows {
    uint32_t w0;       // the wavefront's first row
    bool there, whole; // this lane's row exists; all of the wavefront's do
    int query, head, p;
    int p_min, p_max;  // of the wavefront; one that has no row sees nothing
    Reach reach;
    __device__ __forceinline__ WaveRows(const Window& w, const Cloud& c, uint32_t r0, uint32_t rows)
        : reach(w, c, (int)(r0 / w.group) + c.off, (int)((min(r0 + W * kWaveRows, rows) - 1) / w.group) + c.off) {
        w0 = r0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kWaveRows;
        const uint32_t row = w0 + (threadIdx.x & 31);
        there = row < rows;
        whole = w0 + kWaveRows <= rows;
        query = (int)(row / w.group);
        head = (int)(row % w.group);
        p = there ? query + c.off : kNowhere;
        p_min = w0 < rows ? (int)(w0 / w.group) + c.off : kNowhere;
        p_max = w0 < rows ? (int)((min(w0 + kWaveRows, rows) - 1) / w.group) + c.off : kNowhere;
    }
};

// The keys and values of a workgroup's slots, kN at a time, into LDS
template <typename T, int NT, bool VEC, int W>
struct KeyTiles {
    static constexpr int kN = kKeys<T, W>, kTileBytes = kN * Tile<T, NT>::kRowBytes;
    const Window& w;
    const Reach& reach;
    const T *k, *v;  // the cloud's first rows of this key head
    uint32_t ldk, ldv;  // bytes between rows
    int64_t ldk_elements, ldv_elements;
    TileLoads<T, NT, kN, 64 * W> lk, lv;
    __device__ __forceinline__ KeyTiles(const Window& w_, const Reach& reach_, const Rows<const T>& k_, const Rows<const T>& v_, const Cloud& c, int kh)
        : w(w_), reach(reach_), k(k_.at(c.k0, kh, w_.dim)), v(v_.at(c.k0, kh, w_.dim)), ldk((uint32_t)(k_.ld * sizeof(T))),
          ldv((uint32_t)(v_.ld * sizeof(T))), ldk_elements(k_.ld), ldv_elements(v_.ld) {
        if constexpr (VEC) {
            lk.place(w.dim, [&](int r) { return r * ldk; });
            lv.place(w.dim, [&](int r) { return r * ldv; });
        }
    }
    __device__ __forceinline__ void one(char* tile, const TileLoads<T, NT, kN, 64 * W>& l, const T* p, uint32_t ld, int64_t ld_elements, int slot) const {
        const uint32_t row = w.dim * (uint32_t)sizeof(T);
        if constexpr (VEC) {
            const uint32_t at = lds_address(tile);
            if (slot >= reach.first) {
                l.load(at, memory_of(p + reach.key(slot) * ld_elements, (min(kN, reach.n - slot) - 1) * ld + row));
            } else {
                const int split = min(kN, reach.first - slot), rest = min(kN, reach.n - slot) - split;
                l.load_two(at, memory_of(p + slot * ld_elements, (split - 1) * ld + row), split,
                           memory_of(p + reach.lo * ld_elements, rest > 0 ? (rest - 1) * ld + row : 0), split * ld);
            }
        } else {
            load_elements<T, NT, kN, 64 * W>(tile, w.dim, [&](int r) { return slot + r < reach.n ? p + reach.key(slot + r) * ld_elements : nullptr; });
        }
    }
    __device__ __forceinline__ void load(char* lds, int slot, int buf) const {
        one(lds + buf * 2 * kTileBytes, lk, k, ldk, ldk_elements, slot);
        one(lds + (buf * 2 + 1) * kTileBytes, lv, v, ldv, ldv_elements, slot);
    }
};

template <typename T>
bool in_pieces(const Rows<T>& r) { return r.ld * (int64_t)sizeof(T) % 16 == 0 && r.ld * (int64_t)sizeof(T) <= kMostRowBytes && aligned16(r.p); }

// Workgroups of four wavefronts share what they read; where they are fewer than the chip's compute units, workgroups of one are four
// times as many, each with a shorter way.  Forward and backward in us, four / one: 1601 rows in 8 clouds, 4 heads of 16, fp32 79 / 68; 2500
// rows in 4 clouds, 4 heads of 32, fp32 124 / 104; 256 rows, 8 heads of 64, bf16 55 / 55.
inline bool few_tiles(int64_t tiles_of_four, int kv_heads) { return tiles_of_four * kv_heads <= 256; }

}  // namespace sp
