// One new token of each sequence: its key and value go to the ring cache, and it attends over the window and the first tokens.
#include <algorithm>

#include "sp_attn_tile.h"

namespace sp {
namespace {

constexpr int kThreads = 256;

template <typename T>
struct StepArgs {
    const T *q, *k_new, *v_new;
    T *k_cache, *v_cache, *o;
    const int32_t* lens;
    int batch, cap, heads, kv_heads, group, dim, left, sinks;
    float scale;
};

constexpr int kHeads = 32;  // query heads of a workgroup: the columns of a product
constexpr int kKeys = 32;   // of a wavefront's tile

// The keys a token at position p sees, in order: t-th of n; and the cache's row of a position
struct StepSeen {
    int p, first, lo, n, sinks, ring, from, at;  // position `from`, the first behind the first keys, lies in row sinks + at
    template <typename T>
    __device__ __forceinline__ StepSeen(const StepArgs<T>& a, int b) : p(a.lens[b]), sinks(a.sinks), ring(a.cap - a.sinks) {
        lo = max(max(p - a.left, p - ring + 1), 0);
        first = min(sinks, lo);
        n = p < 0 ? 0 : first + (p - lo + 1);
        from = max(lo, sinks);
        at = (from - sinks) % ring;
    }
    __device__ __forceinline__ int key(int t) const { return t + (t < first ? 0 : lo - first); }
    // of a key that is seen: fewer than `ring` behind `from`
    __device__ __forceinline__ int row(int j) const {
        const int r = at + (j - from);
        return j < sinks ? j : sinks + (r < ring ? r : r - ring);
    }
};

// fp32 heads above 64 have room for one tile of keys and values a wavefront
template <typename T, int NT>
constexpr int kStepBufs = Tile<T, NT>::kRowBytes > 256 ? 1 : 2;

// Reads a sequence's window once and does little else: bound by memory (96 sequences of up to 30000 tokens, 8 key heads of 128, window
// 4096: 243 us, 5.4 TB/s, as a large copy).  Keys as the first operand of 32 x 32 products waste the columns that have no query head; even
// one in 32 leaves the matrix pipes idle nine tenths of the time.  A workgroup has up to 32 query heads of one key head and a
// part of the sequence's keys; its four wavefronts take tiles of 32 keys by turns, each through LDS of its own (two tiles of keys
// and values, the next on its way while one is used), with no barrier until their sums are joined.  The new token's rows are read
// from k_new and v_new: another workgroup may be writing them to the cache.
template <typename T, int NT, bool VEC>
__global__ __launch_bounds__(kThreads, 1) void attn_step_kernel(StepArgs<T> a, int parts, int bufs, float* __restrict__ partial) {
    using Tl = Tile<T, NT>;
    constexpr int kTileBytes = kKeys * Tl::kRowBytes;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = blockIdx.x, columns = (a.group + kHeads - 1) / kHeads, kh = blockIdx.y / columns, h0 = blockIdx.y % columns * kHeads, b = blockIdx.z;
    const int here = min(kHeads, a.group - h0);
    const StepSeen seen(a, b);
    const int64_t fresh = ((int64_t)b * a.kv_heads + kh) * a.dim, slot_step = (int64_t)a.kv_heads * a.dim;
    const int64_t cache = (int64_t)b * a.cap * slot_step + (int64_t)kh * a.dim;
    if (part == 0 && h0 == 0 && seen.p >= 0)
        for (int e = threadIdx.x; e < a.dim; e += kThreads) {
            a.k_cache[cache + seen.row(seen.p) * slot_step + e] = a.k_new[fresh + e];
            a.v_cache[cache + seen.row(seen.p) * slot_step + e] = a.v_new[fresh + e];
        }
    const int each = ((seen.n + parts - 1) / parts + kKeys - 1) / kKeys * kKeys, begin = min(part * each, seen.n), end = min(begin + each, seen.n);
    char* mine = lds + wave * 2 * bufs * kTileBytes;
    const auto pl = Tl::place();
    typename Tl::Frag q[Tl::kSteps];
    const int column = lane & 31;
    Tl::template load_row<VEC>(q, a.q + ((int64_t)b * a.heads + kh * a.group + h0 + column) * a.dim, a.dim, column < here, a.scale < 0.f);
    const float c2 = fmaxf(fabsf(a.scale) * kLog2e, 1e-30f);  // as in the packed form
    // rows of the cache by 32 bits from the sequence's first (step() sees to it); the new token's from another place
    const uint32_t row_bytes = (uint32_t)(slot_step * sizeof(T)), head_bytes = a.dim * (uint32_t)sizeof(T);
    auto load = [&](int t, int buf) {
        char *keys = mine + buf * 2 * kTileBytes, *values = keys + kTileBytes;
        if constexpr (VEC) {
            using Ld = TileLoads<T, NT, kKeys, 64>;
            const uint32_t bytes = (uint32_t)(a.cap - 1) * row_bytes + head_bytes;
            const u32x4 k_ring = memory_of(a.k_cache + cache, bytes), v_ring = memory_of(a.v_cache + cache, bytes);
            const u32x4 k_token = memory_of(a.k_new + fresh, head_bytes), v_token = memory_of(a.v_new + fresh, head_bytes);
#pragma unroll
            for (int k = 0; k < Ld::kLoads; ++k) {
                const int at = t + Ld::row(k), j = seen.key(at), piece = Ld::piece(k);
                const uint32_t k_at = Ld::lds_of(lds_address(keys), k), v_at = Ld::lds_of(lds_address(values), k);
                const bool in = (at < end) & (piece * Tl::kPer < a.dim);
                if (j == seen.p) {
                    memory_to_lds(k_token, in ? piece * 16 : kOutside, k_at);
                    memory_to_lds(v_token, in ? piece * 16 : kOutside, v_at);
                } else {
                    const uint32_t off = in ? seen.row(j) * row_bytes + piece * 16 : 0xffffff00u;
                    memory_to_lds(k_ring, off, k_at);
                    memory_to_lds(v_ring, off, v_at);
                }
            }
        } else {
            auto from = [&](const T* all, const T* now, int r) -> const T* {
                if (t + r >= end) return nullptr;
                const int j = seen.key(t + r);
                return j == seen.p ? now + fresh : all + cache + seen.row(j) * slot_step;
            };
            load_elements<T, NT, kKeys, 64>(keys, a.dim, [&](int r) { return from(a.k_cache, a.k_new, r); });
            load_elements<T, NT, kKeys, 64>(values, a.dim, [&](int r) { return from(a.v_cache, a.v_new, r); });
        }
    };
    f32x16 acc[NT] = {};
    float m = -INFINITY, l = 0.f;
    int t = begin + wave * kKeys, buf = 0;
    if (t < end) load(t, 0);
    for (; t < end; t += 4 * kKeys, buf ^= bufs - 1) {
        wait_own_tiles();
        if (bufs == 2 && t + 4 * kKeys < end) load(t + 4 * kKeys, buf ^ 1);
        const char *keys = mine + buf * 2 * kTileBytes, *values = keys + kTileBytes;
        f32x16 s = {};
#pragma unroll
        for (int st = 0; st < Tl::kSteps; ++st) s = Tl::mma(Tl::direct(keys, pl, 0, st), q[st], s);
        if (t + kKeys > end)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = t + 8 * (i / 4) + 4 * (lane >> 5) + i % 4 < end ? s[i] : -INFINITY;
        float top = m;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
        top = halves<Max>(top);
        const float base = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f((m - base) * c2);
        l *= old;
#pragma unroll
        for (int d = 0; d < NT; ++d) acc[d] *= old;
        m = top;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f((s[i] - base) * c2);
            l += s[i];
        }
#pragma unroll
        for (int st = 0; st < Tl::kTSteps; ++st) {
            const auto pr = Tl::operand(s, st);
#pragma unroll
            for (int d = 0; d < NT; ++d) acc[d] = Tl::mma(Tl::turned(values, pl, 0, st, d), pr, acc[d]);
        }
        if (bufs == 1 && t + 4 * kKeys < end) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            load(t + 4 * kKeys, 0);
        }
    }
    l = halves<Add>(l);
    // [wavefront][column][NT * 32 sums, maximum, sum of exponentials]
    constexpr int kRow = NT * 32 + 2;
    float* sums = reinterpret_cast<float*>(lds);
    __syncthreads();
    if (column < here) {
        float* to = sums + (wave * kHeads + column) * kRow;
        put_column<float, NT, false>(to, acc, NT * 32);
        if (lane < 32) {
            to[NT * 32] = m;
            to[NT * 32 + 1] = l;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < here * a.dim; i += kThreads) {
        const int col = i / a.dim, e = i % a.dim;
        const float* from = sums + col * kRow;
        float top = -INFINITY, v = 0.f, total = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, from[k * kHeads * kRow + NT * 32]);
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float* f = from + k * kHeads * kRow;
            const float x = __builtin_amdgcn_exp2f((f[NT * 32] - base) * c2);
            v = fmaf(f[e], x, v);
            total = fmaf(f[NT * 32 + 1], x, total);
        }
        const int64_t out = (int64_t)b * a.heads + kh * a.group + h0 + col;
        if (parts == 1) {
            a.o[out * a.dim + e] = to_elem<T>(seen.n > 0 ? v / total : 0.f);
        } else {
            float* to = partial + (out * parts + part) * (a.dim + 2);
            to[e] = v;
            if (e == 0) {
                to[a.dim] = top;
                to[a.dim + 1] = total;
            }
        }
    }
}

// the parts of a sequence and head, in order
template <typename T>
__global__ __launch_bounds__(128) void attn_step_join_kernel(StepArgs<T> a, int parts, const float* __restrict__ partial) {
    const int64_t out = (int64_t)blockIdx.y * a.heads + blockIdx.x;
    const float *from = partial + out * parts * (a.dim + 2), c2 = fmaxf(fabsf(a.scale) * kLog2e, 1e-30f);
    const int e = threadIdx.x, lane = e & 63;
    float top = -INFINITY;
    for (int k = lane; k < parts; k += 64) top = fmaxf(top, from[k * (a.dim + 2) + a.dim]);
    top = lanes_reduce<64, Max>(top);
    if (e >= a.dim) return;
    const float base = top == -INFINITY ? 0.f : top;
    float v = 0.f, total = 0.f;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) {
        const float* f = from + k * (a.dim + 2);
        const float x = __builtin_amdgcn_exp2f((f[a.dim] - base) * c2);
        v = fmaf(f[e], x, v);
        total = fmaf(f[a.dim + 1], x, total);
    }
    a.o[out * a.dim + e] = to_elem<T>(a.lens[blockIdx.y] >= 0 ? v / total : 0.f);
}

template <typename T, int NT, bool VEC>
int step_sized(const StepArgs<T>& a, hipStream_t s) {
    using Tl = Tile<T, NT>;
    const int columns = (a.group + kHeads - 1) / kHeads;
    const int64_t items = (int64_t)a.batch * a.kv_heads * columns, most = std::min<int64_t>(a.cap, (int64_t)a.left + 1 + a.sinks);
    // enough workgroups to fill the chip several times, of at least one tile for each wavefront
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>((1024 + items - 1) / items, (most + 4 * kKeys - 1) / (4 * kKeys)));
    Buf partial;
    if (parts > 1) {
        partial = dev_alloc((size_t)a.batch * a.heads * parts * (a.dim + 2) * 4, s);
        if (!partial) return SP_ERR_ALLOC;
    }
    auto kernel = attn_step_kernel<T, NT, VEC>;
    // one tile a wavefront leaves a CU room for two workgroups: 264 of them, one sequence of 8 key heads, run at a time
    const int bufs = (most + parts - 1) / parts <= 4 * kKeys ? 1 : kStepBufs<T, NT>;
    const size_t lds = std::max<size_t>((size_t)8 * bufs * kKeys * Tl::kRowBytes, (size_t)4 * kHeads * (NT * 32 + 2) * 4);
    {
        static std::mutex mu;
        static size_t attr_lds = 64 * 1024;  // largest dynamic LDS size opted into so far
        std::lock_guard<std::mutex> lk(mu);
        if (lds > attr_lds) {
            SP_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
            attr_lds = lds;
        }
    }
    hipLaunchKernelGGL(kernel, dim3(parts, a.kv_heads * columns, a.batch), dim3(kThreads), lds, s, a, parts, bufs, ptr<float>(partial));
    if (parts > 1) hipLaunchKernelGGL(attn_step_join_kernel<T>, dim3(a.heads, a.batch), dim3(128), 0, s, a, parts, ptr<float>(partial));
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T>
int step(const StepArgs<T>& a, hipStream_t s) {
    const bool vec = a.dim * sizeof(T) % 16 == 0 && (int64_t)a.cap * a.kv_heads * a.dim * (int64_t)sizeof(T) < 0xf0000000ll && aligned16(a.q) && aligned16(a.k_new) && aligned16(a.v_new) && aligned16(a.k_cache) && aligned16(a.v_cache);
    const int nt = (a.dim + 31) / 32;
    if (vec) return nt == 1 ? step_sized<T, 1, true>(a, s) : nt == 2 ? step_sized<T, 2, true>(a, s) : nt == 3 ? step_sized<T, 3, true>(a, s) : step_sized<T, 4, true>(a, s);
    return nt == 1 ? step_sized<T, 1, false>(a, s) : nt == 2 ? step_sized<T, 2, false>(a, s) : nt == 3 ? step_sized<T, 3, false>(a, s) : step_sized<T, 4, false>(a, s);
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" int sp_window_attn_step(const void* d_q, const void* d_k_new, const void* d_v_new, void* d_k_cache, void* d_v_cache,
                                   const int32_t* d_lens, int32_t batch, int32_t cap, int32_t heads, int32_t kv_heads, int32_t dim,
                                   int32_t left, int32_t sinks, float scale, void* d_o, sp_dtype dt, void* stream) {
    if (batch < 0) return fail(SP_ERR_INVALID_ARG, "negative batch");
    if (dt != SP_F32 && dt != SP_BF16) return fail(SP_ERR_INVALID_ARG, "bad dtype");
    if (heads < 1 || kv_heads < 1 || heads % kv_heads) return fail(SP_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
    if (dim < 1) return fail(SP_ERR_INVALID_ARG, "bad head width");
    if (left < 0 || sinks < 0 || cap <= sinks) return fail(SP_ERR_INVALID_ARG, "left and sinks must not be negative, the cache longer than sinks");
    if (!(scale > -3.0e38f && scale < 3.0e38f)) return fail(SP_ERR_INVALID_ARG, "the scale must be finite");
    if (dim > kMaxDim || heads > 65535 || batch > 65535)
        return fail(SP_ERR_UNSUPPORTED, "head widths above %d, more than 65535 heads or sequences", kMaxDim);
    if (batch == 0) return SP_OK;
    if (!d_q || !d_k_new || !d_v_new || !d_k_cache || !d_v_cache || !d_lens || !d_o) return fail(SP_ERR_INVALID_ARG, "a pointer is NULL");
    hipStream_t s = (hipStream_t)stream;
    if (dt == SP_F32)
        return step<float>({(const float*)d_q, (const float*)d_k_new, (const float*)d_v_new, (float*)d_k_cache, (float*)d_v_cache, (float*)d_o,
                            d_lens, batch, cap, heads, kv_heads, heads / kv_heads, dim, left, sinks, scale}, s);
    return step<bf16_t>({(const bf16_t*)d_q, (const bf16_t*)d_k_new, (const bf16_t*)d_v_new, (bf16_t*)d_k_cache, (bf16_t*)d_v_cache,
                         (bf16_t*)d_o, d_lens, batch, cap, heads, kv_heads, heads / kv_heads, dim, left, sinks, scale}, s);
}
