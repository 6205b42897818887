// What the kernels of the windowed attention share: their arguments, and which cloud a row belongs to.
#pragma once

#include "sp_elem.h"

#include "sp_attn_cut.h"

namespace sp {

constexpr int kMaxDim = 128;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Row r, head h of an array starts at p + r * ld + h * dim.
template <typename T>
struct Rows {
    T* p;
    int64_t ld;
    __device__ __forceinline__ T* at(int64_t r, int h, int dim) const { return p + r * ld + (int64_t)h * dim; }
};

struct Window {
    const int32_t *q_starts, *k_starts;
    int n_q, n_k, clouds;
    int heads, kv_heads, group, dim;
    int left, right, sinks;  // at most n_k, n_q and n_k: more changes nothing, and positions +- these fit 32 bits
    float scale;
};

template <typename T>
struct AttnFwd {
    Window w;
    Rows<const T> q, k, v;
    Rows<T> o;
    float* lse;  // [n_q][heads]
};

template <typename T>
struct AttnBwd {
    Window w;
    Rows<const T> q, k, v, o, dout;
    const float* lse;
    float* delta;  // [n_q][heads]: dout . o
    Rows<T> dq, dk, dv;
};

template <typename T>
int attn_backward(const AttnBwd<T>& g, hipStream_t s);  // sp_attn_bwd.hip

// The last cloud c of which first(c) <= t, by a wavefront.  All lanes must come here together.
template <typename First>
__device__ __forceinline__ int find_cloud(int clouds, int64_t t, First first) {
    return __builtin_amdgcn_readfirstlane(last_cloud(clouds, [&](int lo, int step, int hi) {
        const int at = lo + ((int)(threadIdx.x & 63) + 1) * step;
        return (int)__popcll(__ballot(at <= hi && first(at) <= t));
    }));
}
// A tile number's cloud and the tile's first row, counted from the cloud's (see in_cloud).
struct CloudTile {
    int cloud;
    int64_t row;
    __device__ __forceinline__ CloudTile(const int32_t* starts, int clouds, int n, int64_t t, int per, int tile) {
        cloud = find_cloud(clouds, t, [&](int c) { return first_tile(starts, clouds, n, c, per, tile); });
        row = (t - first_tile(starts, clouds, n, cloud, per, tile)) * tile;
    }
};

struct Cloud {
    int q0, a, k0, b;  // first query row, queries, first key row, keys
    int off;           // query i stands at position i + off
    __device__ __forceinline__ Cloud(const Window& w, int c) {
        q0 = cloud_begin(w.q_starts, w.clouds, w.n_q, c);
        a = cloud_rows(w.q_starts, w.clouds, w.n_q, c);
        k0 = cloud_begin(w.k_starts, w.clouds, w.n_k, c);
        b = cloud_rows(w.k_starts, w.clouds, w.n_k, c);
        off = b - a;
        partners = c >= 1 && c <= w.clouds;
    }
    bool partners;  // false: these rows belong to no cloud, see nothing and are seen by nobody
};

}  // namespace sp
