// What the kernels of the windowed attention share: which cloud a row belongs to, which keys a query sees, and one row's results
// computed by one wavefront, key by key.
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

// A tile number's cloud and the tile's first row, counted from the cloud's (see in_cloud).  All lanes must come here together.
struct CloudTile {
    int cloud;
    int64_t row;
    __device__ __forceinline__ CloudTile(const int32_t* starts, int clouds, int n, int64_t t, int per, int tile) {
        const int c = last_cloud(clouds, [&](int lo, int step, int hi) {
            const int at = lo + ((int)(threadIdx.x & 63) + 1) * step;
            return (int)__popcll(__ballot(at <= hi && first_tile(starts, clouds, n, at, per, tile) <= t));
        });
        cloud = __builtin_amdgcn_readfirstlane(c);
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

// The keys that query i of a cloud sees, in order: t-th of n
struct Seen {
    int first, lo, n;
    __device__ __forceinline__ Seen(const Window& w, const Cloud& c, int i) {
        const int p = i + c.off;
        const int hi = c.partners ? min(max(p + w.right + 1, 0), c.b) : 0;
        lo = min(max(p - w.left, 0), hi);
        first = min(w.sinks, lo);
        n = first + hi - lo;
    }
    __device__ __forceinline__ int key(int t) const { return t < first ? t : lo + t - first; }
};

__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
// ---- one row by one wavefront: lanes are keys (or queries) for the scores and elements for the products with rows --------------
// All lanes must come here together.

template <typename T>
__device__ __forceinline__ float dot(const T* a, const T* b, int dim) {
    float s = 0.f;
    for (int e = 0; e < dim; ++e) s = fmaf(elem(a[e]), elem(b[e]), s);
    return s;
}
// acc[e] += value of lane t * row t's elements, for the n rows that at(t) gives
template <typename T, typename At>
__device__ __forceinline__ void add_rows(float (&acc)[2], float value, int n, int dim, At at) {
    const int lane = threadIdx.x & 63;
    for (int t = 0; t < n; ++t) {
        const T* row = at(t);
        const float x = lane_value(value, t);
        if (lane < dim) acc[0] = fmaf(x, elem(row[lane]), acc[0]);
        if (lane + 64 < dim) acc[1] = fmaf(x, elem(row[lane + 64]), acc[1]);
    }
}
template <typename T>
__device__ __forceinline__ void put_row(T* row, const float (&acc)[2], int dim) {
    const int lane = threadIdx.x & 63;
    if (lane < dim) row[lane] = to_elem<T>(acc[0]);
    if (lane + 64 < dim) row[lane + 64] = to_elem<T>(acc[1]);
}

template <typename T>
__device__ __forceinline__ void key_gradient_row(const AttnBwd<T>& g, const Cloud& c, int j, int kh) {
    const Window& w = g.w;
    const int lane = threadIdx.x & 63;
    // queries at positions j - right .. j + left (all later ones for the first keys)
    const int end = c.partners ? c.a : 0;
    const int lo = min(max(j - w.right - c.off, 0), end);
    const int hi = j < w.sinks ? end : min(max(j + w.left + 1 - c.off, lo), end);
    float ak[2] = {0.f, 0.f}, av[2] = {0.f, 0.f};
    const T *k = g.k.at(c.k0 + j, kh, w.dim), *v = g.v.at(c.k0 + j, kh, w.dim);
    for (int h = kh * w.group; h < (kh + 1) * w.group; ++h)
        for (int i0 = lo; i0 < hi; i0 += 64) {
            float p = 0.f, ds = 0.f;
            if (i0 + lane < hi) {
                const int64_t r = c.q0 + i0 + lane;
                p = __builtin_amdgcn_exp2f((dot(g.q.at(r, h, w.dim), k, w.dim) * w.scale - g.lse[r * w.heads + h]) * kLog2e);
                ds = p * (dot(g.dout.at(r, h, w.dim), v, w.dim) - g.delta[r * w.heads + h]) * w.scale;
            }
            const int n = min(64, hi - i0);
            add_rows<T>(ak, ds, n, w.dim, [&](int t) { return g.q.at(c.q0 + i0 + t, h, w.dim); });
            add_rows<T>(av, p, n, w.dim, [&](int t) { return g.dout.at(c.q0 + i0 + t, h, w.dim); });
        }
    put_row(g.dk.at(c.k0 + j, kh, w.dim), ak, w.dim);
    put_row(g.dv.at(c.k0 + j, kh, w.dim), av, w.dim);
}

}  // namespace sp
