// cache_append: rotation of queries and keys by their positions, keys and values into a paged cache.
//
//   (x, y) -> (x cos a - y sin a, y cos a + x sin a),  a = position * inv_freq[pair]
//
// The product is formed in double and reduced to [-pi, pi] there: at position 131072 an fp32 product would be off
// by 0.008 rad.  Sine and cosine are those of the reduced angle rounded to fp32 (by up to 2^-23 rad), the rotation is fp32, and
// results are rounded once.
// Bound by memory: every element is read once and written once.  One CTA has one node (all heads of a token share
// its angles, which are formed once into shared memory).  A thread asks for its first vectors before it looks up where
// they go: the length, the parents, the page and the angles take some 2000 clocks one after the other.
// 256 x 17 nodes, 32/8 heads of 128, bf16: 21.4 us; 4 prompts of 8000, adjacent pairs: 137 us, 5.7 TB/s.
#include "common.cuh"
#include "draft_tree.cuh"
#include "host_util.h"
#include "launch.h"

namespace spr {

namespace {

constexpr int kAppendThreads = 256;
constexpr int kMaxRotPairs = 512;        // head dimension up to 1024

struct AppendParams {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;    // elements from one node to the next
    DraftNodes nodes;
    const int32_t *slots;
    const float *inv_freq;
    const int32_t *page_table;
    void *k_cache, *v_cache, *q_out;
    int *status;
    int Hq, Hkv, D, pairs;                   // pairs = rotated elements / 2
    int interleaved;
    int max_pages, num_pages, page_size;
    int wide;                                // heads are made of pairs of vectors
    int rotated, copied;                     // units of a rotated head, of a value head (see append_kernel)
    uint32_t rotated_inv, copied_inv;        // 2^32 / these, rounded up
};

// what a thread moves at once, as it lies in memory, and as numbers
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int n = 4;
    float4 raw;
    __device__ __forceinline__ void load(const float *p) { raw = __ldcs(reinterpret_cast<const float4 *>(p)); }
    __device__ __forceinline__ void store(float *p) const { __stcs(reinterpret_cast<float4 *>(p), raw); }
    __device__ __forceinline__ void get(float (&x)[4]) const { x[0] = raw.x, x[1] = raw.y, x[2] = raw.z, x[3] = raw.w; }
    __device__ __forceinline__ void set(const float (&x)[4]) { raw = make_float4(x[0], x[1], x[2], x[3]); }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    uint4 raw;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { raw = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { __stcs(reinterpret_cast<uint4 *>(p), raw); }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
            w[e] = *reinterpret_cast<const uint32_t *>(&b);
        }
        raw = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
// one element at a time, for rows that are not made of whole aligned vectors
template <typename T>
struct One {
    static constexpr int n = 1;
    T raw;
    __device__ __forceinline__ void load(const T *p) { raw = *p; }
    __device__ __forceinline__ void store(T *p) const { *p = raw; }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = (float)raw; }
    __device__ __forceinline__ void set(const float (&x)[1]) { raw = (T)x[0]; }
};

__device__ __forceinline__ int divide(int x, int by, uint32_t inv) { return by == 1 ? x : (int)__umulhi((uint32_t)x, inv); }

// n cosines and sines from `turn` on
template <int n>
__device__ __forceinline__ void angles(const float *turn, float (&c)[n], float (&s)[n])
{
    if constexpr (n % 4 == 0) {
#pragma unroll
        for (int e = 0; e < n; e += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(turn + e), y = *reinterpret_cast<const float4 *>(turn + kMaxRotPairs + e);
            c[e] = x.x, c[e + 1] = x.y, c[e + 2] = x.z, c[e + 3] = x.w;
            s[e] = y.x, s[e + 1] = y.y, s[e + 2] = y.z, s[e + 3] = y.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < n; ++e) c[e] = turn[e], s[e] = turn[kMaxRotPairs + e];
    }
}

// A unit is what a thread moves at once: two vectors V where there are two.  Pairs of halves: a vector and its partner `pairs`
// elements on; behind them, in the rest of a head, one vector.  Adjacent pairs, and value heads: neighbours.
template <typename T, typename V, bool ADJACENT>
struct Unit {
    static constexpr int n = V::n;
    static constexpr bool kPartners = !ADJACENT || n == 1;     // the two vectors of a rotated unit turn with each other
    V a, o;
    int head, col, by;                                         // by: distance of the second vector, 0 where there is none
    __device__ __forceinline__ void place(const AppendParams &p, int u)
    {
        const int turned = (p.Hq + p.Hkv) * p.rotated;
        const bool is_v = u >= turned;
        if (is_v) u -= turned;
        const int h = is_v ? divide(u, p.copied, p.copied_inv) : divide(u, p.rotated, p.rotated_inv);
        const int j = u - h * (is_v ? p.copied : p.rotated);
        head = is_v ? h + p.Hq + p.Hkv : h;
        if (is_v || !kPartners) {
            by = p.wide ? n : 0;
            col = j * (n + by);
        } else {
            const int two = p.pairs / n;
            by = j < two ? (ADJACENT ? 1 : p.pairs) : 0;
            col = j < two ? (ADJACENT ? 2 * j : j * n) : 2 * p.pairs + (j - two) * n;
        }
    }
    __device__ __forceinline__ void load(const AppendParams &p, int64_t node)
    {
        const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.Hkv;
        const T *src = is_q   ? static_cast<const T *>(p.q) + node * p.q_stride + (int64_t)head * p.D
                       : is_v ? static_cast<const T *>(p.v) + node * p.v_stride + (int64_t)(head - p.Hq - p.Hkv) * p.D
                              : static_cast<const T *>(p.k) + node * p.k_stride + (int64_t)(head - p.Hq) * p.D;
        a.load(src + col);
        if (by) o.load(src + col + by);
    }
    // pairs within a vector that begins at column col
    __device__ __forceinline__ void turn_within(V &v, int col, const AppendParams &p, const float *turn)
    {
        if (col >= 2 * p.pairs) return;
        float x[n], c[n > 1 ? n / 2 : 1], w[n > 1 ? n / 2 : 1];
        v.get(x);
        angles<(n > 1 ? n / 2 : 1)>(turn + col / 2, c, w);
#pragma unroll
        for (int e = 0; e + 1 < n; e += 2)
            if ((col + e) / 2 < p.pairs) {
                const float z = x[e], y = x[e + 1];
                x[e] = z * c[e / 2] - y * w[e / 2];
                x[e + 1] = y * c[e / 2] + z * w[e / 2];
            }
        v.set(x);
    }
    // entry: where head 0's row of the node lies in the caches, in rows; negative: nowhere
    __device__ __forceinline__ void store(const AppendParams &p, int64_t node, int64_t entry, const float *turn)
    {
        const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.Hkv;
        if (!is_q && entry < 0) return;
        T *dst = is_q   ? static_cast<T *>(p.q_out) + (node * p.Hq + head) * p.D
                 : is_v ? static_cast<T *>(p.v_cache) + (entry + (int64_t)(head - p.Hq - p.Hkv) * p.page_size) * p.D
                        : static_cast<T *>(p.k_cache) + (entry + (int64_t)(head - p.Hq) * p.page_size) * p.D;
        if (!is_v && kPartners && by) {
            float x[n], y[n], c[n], w[n];
            a.get(x);
            o.get(y);
            angles<n>(turn + (ADJACENT ? col / 2 : col), c, w);
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float z = x[e];
                x[e] = z * c[e] - y[e] * w[e];
                y[e] = y[e] * c[e] + z * w[e];
            }
            a.set(x);
            o.set(y);
        }
        if (!is_v && !kPartners) {
            turn_within(a, col, p, turn);
            if (by) turn_within(o, col + by, p, turn);
        }
        if (by) o.store(dst + col + by);
        a.store(dst + col);
    }
};

template <typename T, typename V, bool ADJACENT>
__global__ void __launch_bounds__(kAppendThreads, 5) append_kernel(const AppendParams p)
{
    constexpr int kAhead = 2;
    __shared__ __align__(16) float turn[2 * kMaxRotPairs];       // cosines, then sines
    __shared__ int tree[kMaxTreeNodes];
    const int64_t node = blockIdx.x;
    const int tid = threadIdx.x, units = (p.Hq + p.Hkv) * p.rotated + p.Hkv * p.copied;
    Unit<T, V, ADJACENT> unit[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (tid + k * kAppendThreads < units) {
            unit[k].place(p, tid + k * kAppendThreads);
            unit[k].load(p, node);
        }
    const int b = (int)(node / p.nodes.T), i = (int)(node - (int64_t)b * p.nodes.T);
    const int given = p.slots ? __ldg(p.slots + node) : 0;
    const int len = __ldg(p.nodes.lens + b);
    const bool used = len >= 0 && i < node_count(p.nodes, b);
    if (!used) {
        T *q_out = static_cast<T *>(p.q_out) + node * p.Hq * p.D;
        for (int c = tid; c < p.Hq * p.D; c += kAppendThreads) q_out[c] = (T)0.f;
        return;
    }
    // the page and the entry in it; nothing is kept where there is none
    const int64_t slot = p.slots ? (int64_t)given : (int64_t)len + i;
    int64_t entry = -1;
    if (slot >= 0) {
        const int64_t at = slot >> 31 ? slot / p.page_size : (int64_t)((uint32_t)slot / (uint32_t)p.page_size);
        const int page = at < p.max_pages ? __ldg(p.page_table + (int64_t)b * p.max_pages + at) : -1;
        if (page >= 0 && page < p.num_pages)
            entry = (int64_t)page * p.Hkv * p.page_size + (slot - at * p.page_size);
        else if (tid == 0)
            raise_status(p.status, SPR_ERR_BAD_PAGE);
    }
    int depth = i;
    if (p.nodes.parents) {
        for (int j = tid; j <= i; j += kAppendThreads) tree[j] = p.nodes.parents[(int64_t)b * p.nodes.T + j];
        __syncthreads();
        depth = 0;
        for (int j = checked_parent(tree[i], i, p.status); j >= 0; j = checked_parent(tree[j], j, p.status)) ++depth;
    }
    const double position = (double)len + depth;
    for (int j = tid; j < p.pairs; j += kAppendThreads) {
        double a = position * (double)__ldg(p.inv_freq + j);
        a = fma(-6.283185307179586477, rint(a * 0.15915494309189533577), a);
        sincosf((float)a, &turn[kMaxRotPairs + j], &turn[j]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (tid + k * kAppendThreads < units) {
            unit[k].place(p, tid + k * kAppendThreads);         // (again: cheaper than registers to keep it)
            unit[k].store(p, node, entry, turn);
        }
    for (int u = tid + kAhead * kAppendThreads; u < units; u += kAppendThreads) {
        unit[0].place(p, u);
        unit[0].load(p, node);
        unit[0].store(p, node, entry, turn);
    }
}

template <typename T>
cudaError_t launch_append(AppendParams &p, int64_t nodes, cudaStream_t st)
{
    constexpr int n = 16 / sizeof(T);
    auto whole = [&](const void *t, int64_t stride) { return !t || (aligned(t, 16) && stride % n == 0); };
    const bool vec = whole(p.q, p.q_stride) && whole(p.k, p.k_stride) && whole(p.v, p.v_stride) && whole(p.q_out, 0) &&
                     whole(p.k_cache, 0) && whole(p.v_cache, 0) && p.D % n == 0 &&
                     (p.interleaved || p.pairs % n == 0);
    const int w = vec ? n : 1;
    p.wide = p.D % (2 * w) == 0;
    p.copied = p.D / w / (p.wide ? 2 : 1);
    p.rotated = !p.interleaved || w == 1 ? p.pairs / w + (p.D - 2 * p.pairs) / w : p.copied;      // (as Unit::kPartners)
    p.rotated_inv = (uint32_t)((((uint64_t)1 << 32) + p.rotated - 1) / p.rotated);
    p.copied_inv = (uint32_t)((((uint64_t)1 << 32) + p.copied - 1) / p.copied);
    const unsigned ctas = (unsigned)nodes;
    if (vec && p.interleaved)
        append_kernel<T, Vec<T>, true><<<ctas, kAppendThreads, 0, st>>>(p);
    else if (vec)
        append_kernel<T, Vec<T>, false><<<ctas, kAppendThreads, 0, st>>>(p);
    else if (p.interleaved)
        append_kernel<T, One<T>, true><<<ctas, kAppendThreads, 0, st>>>(p);
    else
        append_kernel<T, One<T>, false><<<ctas, kAppendThreads, 0, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

}  // namespace spr

using namespace spr;

extern "C" int cache_append(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                            int B, int T, int Hq, int Hkv, int D, int dt, const int32_t *lens, const int32_t *counts,
                            const int32_t *parents, const int32_t *slots, const float *inv_freq, int rot, int interleaved,
                            const int32_t *page_table, int max_pages, int num_pages, int page_size, void *k_cache,
                            void *v_cache, void *q_out, void *ws, size_t ws_bytes, void *cuda_stream)
{
    if (!dtype_ok(dt)) return SPR_ERR_UNSUPPORTED;
    if (B < 0 || T < 0 || Hq < 0 || Hkv <= 0 || D <= 0 || D > 2 * kMaxRotPairs || rot < 0 || rot % 2 || rot > D || max_pages <= 0 ||
        num_pages <= 0 || page_size <= 0 || (int64_t)B * T > 0x7fffffff || (int64_t)Hq + 2 * (int64_t)Hkv > 4096)
        return SPR_ERR_INVALID_ARG;
    if (parents && T > kMaxTreeNodes) return SPR_ERR_UNSUPPORTED;
    if (B == 0 || T == 0) return SPR_OK;
    const size_t es = elem_size(dt);
    if (!k || !v || !lens || !page_table || !k_cache || !v_cache || (rot && !inv_freq) || !q != !q_out || (q && Hq == 0))
        return SPR_ERR_INVALID_ARG;
    if (!aligned(k, es) || !aligned(v, es) || !aligned(k_cache, es) || !aligned(v_cache, es) || !aligned(q, es) || !aligned(q_out, es) ||
        !aligned(lens, 4) || !aligned(counts, 4) || !aligned(parents, 4) || !aligned(slots, 4) || !aligned(inv_freq, 4) ||
        !aligned(page_table, 4))
        return SPR_ERR_INVALID_ARG;
    if (k_stride < (int64_t)Hkv * D || v_stride < (int64_t)Hkv * D || (q && q_stride < (int64_t)Hq * D)) return SPR_ERR_INVALID_ARG;
    // in place a node's queries would be written over another's that are still to be read
    if (q && q == q_out && q_stride != (int64_t)Hq * D && (int64_t)B * T > 1) return SPR_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < (size_t)kHeaderBytes) return SPR_ERR_WORKSPACE;
    const int rc = device_supported();
    if (rc != SPR_OK) return rc;
    AppendParams p = {};
    p.q = q, p.k = k, p.v = v;
    p.q_stride = q ? q_stride : 0, p.k_stride = k_stride, p.v_stride = v_stride;
    p.nodes = DraftNodes{lens, counts, parents, T};
    p.slots = slots, p.inv_freq = inv_freq, p.page_table = page_table;
    p.k_cache = k_cache, p.v_cache = v_cache, p.q_out = q_out;
    p.status = static_cast<int *>(ws);
    p.Hq = q ? Hq : 0, p.Hkv = Hkv, p.D = D, p.pairs = rot / 2, p.interleaved = interleaved != 0;
    p.max_pages = max_pages, p.num_pages = num_pages, p.page_size = page_size;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return finish(dt == SPR_F32 ? launch_append<float>(p, (int64_t)B * T, st) : launch_append<__nv_bfloat16>(p, (int64_t)B * T, st));
}
