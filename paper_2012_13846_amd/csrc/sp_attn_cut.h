// How the windowed attention cuts packed clouds into tiles of rows, and where the sums of the first keys lie: arithmetic that the
// host and the kernels share.  No device code and no other header, so that a test on the CPU can check every index.
//
// Starts come from device memory and may be anything: every function takes what they give into the arrays, and a tile that a workgroup
// finds for itself is used only if in_cloud() says so.
#pragma once

#include <cstdint>

#ifndef SP_HOST_DEVICE
#ifdef __HIPCC__
#define SP_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define SP_HOST_DEVICE inline
#endif
#endif

namespace sp {

// Clouds 1 .. clouds are the caller's; 0 and clouds + 1 hold the rows before the first and after the last.
SP_HOST_DEVICE int cloud_begin(const int32_t* starts, int clouds, int n, int c) {
    if (c <= 0) return 0;
    if (c > clouds + 1) return n;
    const int s = starts[c - 1];
    return s < 0 ? 0 : s < n ? s : n;
}
// Rows of cloud c: none where the starts descend
SP_HOST_DEVICE int cloud_rows(const int32_t* starts, int clouds, int n, int c) {
    const int rows = cloud_begin(starts, clouds, n, c + 1) - cloud_begin(starts, clouds, n, c);
    return rows > 0 ? rows : 0;
}
// Rows cut cloud by cloud into tiles of `tile`, each row of the array standing for `per` rows of the cut: cloud c has the tile
// numbers from begin(c) * per / tile + c on, which are at least as many as its tiles.
SP_HOST_DEVICE int64_t first_tile(const int32_t* starts, int clouds, int n, int c, int per, int tile) {
    return (int64_t)cloud_begin(starts, clouds, n, c) * per / tile + c;
}
SP_HOST_DEVICE int64_t tile_numbers(int64_t n, int clouds, int per, int tile) { return n * per / tile + clouds + 2; }

// The last cloud whose first tile is <= t, 64 clouds at a time: `count(lo, step, hi)` says how many of the clouds lo + step, lo + 2 step,
// .., lo + 64 step that are no more than `hi` have such a first tile.  Where the starts do not ascend it is some cloud, whose first tile may be behind t.
template <typename Count>
SP_HOST_DEVICE int last_cloud(int clouds, Count count) {
    int lo = 0, hi = clouds + 1;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64;
        lo += step * count(lo, step, hi);
        hi = hi < lo + step - 1 ? hi : lo + step - 1;
    }
    return lo;
}
// A tile's first row, counted from its cloud's: of that cloud?  Not for the numbers between two clouds' tiles, and before the cloud's
// first row where the starts do not ascend.
SP_HOST_DEVICE bool in_cloud(int64_t row, int64_t rows) { return row >= 0 && row < rows; }

// Sums of the first keys: [part][kv_heads][sinks][dk, dv][dim]
SP_HOST_DEVICE int64_t sums_at(int kv_heads, int sinks, int dim, int64_t part, int kh, int key) {
    return (((part * kv_heads + kh) * sinks + key) * 2) * dim;
}

// The clouds whose first keys' sums are split: those of at least `least` keys.  How many there are stands in device memory; they have places
// (parts of the keys' own sums) by the clouds' numbers, or, of more clouds than there can be long ones, by where they begin: two that
// begin in the same `least` keys are not both long.
struct LongClouds {
    const int32_t *q_starts, *k_starts;
    int n_q, n_k, clouds;
    int per, chunk;  // rows of a query; of a chunk
    int least;
    SP_HOST_DEVICE bool by_number() const { return clouds <= n_k / least + 1; }
    SP_HOST_DEVICE int places() const { return by_number() ? clouds : n_k / least + 1; }
    SP_HOST_DEVICE int place(int c) const { return by_number() ? c - 1 : cloud_begin(k_starts, clouds, n_k, c) / least; }
    SP_HOST_DEVICE bool has(int c) const { return c >= 1 && c <= clouds && cloud_rows(k_starts, clouds, n_k, c) >= least; }
    // Their rows cut into chunks: a long cloud has the numbers from here on, at least as many as its chunks before the next cloud's
    SP_HOST_DEVICE int64_t first_chunk(int c) const { return (int64_t)cloud_begin(q_starts, clouds, n_q, c) * per / chunk + place(c); }
    SP_HOST_DEVICE int64_t chunks() const { return (int64_t)n_q * per / chunk + places() + 1; }
};

}  // namespace sp
