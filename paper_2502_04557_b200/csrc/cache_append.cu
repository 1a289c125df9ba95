// cache_append: rotation of queries and keys by their positions, keys and values into a paged cache.
//
//   (x, y) -> (x cos a - y sin a, y cos a + x sin a),  a = position * inv_freq[pair]
//
// The product is formed in double and reduced to [-pi, pi] there: at position 131072 an fp32 product would be off
// by 0.008 rad.  Sine and cosine of the reduced angle are fp32, and so is the rotation; results are rounded once.
// Bound by memory: every element is read once and written once.  One CTA has one node (all heads of a token share
// its angles, which are formed once into shared memory).
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
};

template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int n = 4;
    float x[4];
    __device__ __forceinline__ void load(const float *p)
    {
        const float4 a = *reinterpret_cast<const float4 *>(p);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    }
    __device__ __forceinline__ void store(float *p) const { *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]); }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    float x[8];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p)
    {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const
    {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
            w[e] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
// one element at a time, for rows that are not made of whole aligned vectors
template <typename T>
struct One {
    static constexpr int n = 1;
    float x[1];
    __device__ __forceinline__ void load(const T *p) { x[0] = (float)*p; }
    __device__ __forceinline__ void store(T *p) const { *p = (T)x[0]; }
};

// V: the vector that a thread moves; x runs over a head's vectors, y over heads
template <typename T, typename V>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendParams p)
{
    __shared__ float2 turn[kMaxRotPairs];
    __shared__ int tree[kMaxTreeNodes];
    const int64_t node = blockIdx.x;
    const int b = (int)(node / p.nodes.T), i = (int)(node - (int64_t)b * p.nodes.T);
    const int len = __ldg(p.nodes.lens + b);
    const bool used = len >= 0 && i < node_count(p.nodes, b);
    const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
    T *q_out = static_cast<T *>(p.q_out) + node * p.Hq * p.D;
    if (!used) {
        if (p.q_out)
            for (int c = tid; c < p.Hq * p.D; c += threads) q_out[c] = (T)0.f;
        return;
    }
    int depth = i;
    if (p.nodes.parents) {
        for (int j = tid; j <= i; j += threads) tree[j] = p.nodes.parents[(int64_t)b * p.nodes.T + j];
        __syncthreads();
        depth = 0;
        for (int j = checked_parent(tree[i], i, p.status); j >= 0; j = checked_parent(tree[j], j, p.status)) ++depth;
    }
    // the page and the entry in it; nothing is kept where there is none
    const int64_t slot = p.slots ? (int64_t)__ldg(p.slots + node) : (int64_t)len + i;
    int64_t entry = -1;
    if (slot >= 0) {
        const int64_t at = slot / p.page_size;
        const int page = at < p.max_pages ? __ldg(p.page_table + (int64_t)b * p.max_pages + at) : -1;
        if (page >= 0 && page < p.num_pages)
            entry = (int64_t)page * p.Hkv * p.page_size + (slot - at * p.page_size);
        else if (tid == 0)
            raise_status(p.status, SPR_ERR_BAD_PAGE);
    }
    const double position = (double)len + depth;
    for (int j = tid; j < p.pairs; j += threads) {
        double a = position * (double)__ldg(p.inv_freq + j);
        a = fma(-6.283185307179586477, rint(a * 0.15915494309189533577), a);
        sincosf((float)a, &turn[j].y, &turn[j].x);
    }
    __syncthreads();
    const T *q = static_cast<const T *>(p.q) + node * p.q_stride;
    const T *k = static_cast<const T *>(p.k) + node * p.k_stride;
    const T *v = static_cast<const T *>(p.v) + node * p.v_stride;
    T *k_cache = static_cast<T *>(p.k_cache), *v_cache = static_cast<T *>(p.v_cache);
    constexpr int n = V::n;
    const int heads = p.Hq + 2 * p.Hkv;
    for (int h = threadIdx.y; h < heads; h += blockDim.y) {
        const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
        const int hk = is_q ? h : is_v ? h - p.Hq - p.Hkv : h - p.Hq;
        if (is_q ? !p.q_out : entry < 0) continue;
        const T *src = (is_q ? q : is_v ? v : k) + (int64_t)hk * p.D;
        T *dst = is_q ? q_out + (int64_t)hk * p.D
                      : (is_v ? v_cache : k_cache) + (entry + (int64_t)hk * p.page_size) * p.D;
        const int pairs = is_v ? 0 : p.pairs;
        if (p.interleaved && n > 1) {
            for (int c = threadIdx.x * n; c < p.D; c += blockDim.x * n) {
                V a;
                a.load(src + c);
#pragma unroll
                for (int e = 0; e + 1 < n; e += 2)
                    if ((c + e) / 2 < pairs) {
                        const float2 t = turn[(c + e) / 2];
                        const float x = a.x[e], y = a.x[e + 1];
                        a.x[e] = x * t.x - y * t.y;
                        a.x[e + 1] = y * t.x + x * t.y;
                    }
                a.store(dst + c);
            }
        } else {
            // element c and its partner: `pairs` further on, or the next one
            const int by = p.interleaved ? 1 : pairs, step = p.interleaved ? 2 : 1;
            for (int c = threadIdx.x * n; c < pairs; c += blockDim.x * n) {
                V a, o;
                a.load(src + c * step);
                o.load(src + c * step + by);
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    const float2 t = turn[c + e];
                    const float x = a.x[e], y = o.x[e];
                    a.x[e] = x * t.x - y * t.y;
                    o.x[e] = y * t.x + x * t.y;
                }
                a.store(dst + c * step);
                o.store(dst + c * step + by);
            }
            for (int c = 2 * pairs + threadIdx.x * n; c < p.D; c += blockDim.x * n) {
                V a;
                a.load(src + c);
                a.store(dst + c);
            }
        }
    }
}

template <typename T>
cudaError_t launch_append(const AppendParams &p, int64_t nodes, cudaStream_t st)
{
    constexpr int n = 16 / sizeof(T);
    auto whole = [&](const void *t, int64_t stride) { return !t || (aligned(t, 16) && stride % n == 0); };
    const bool vec = whole(p.q, p.q_stride) && whole(p.k, p.k_stride) && whole(p.v, p.v_stride) && whole(p.q_out, 0) &&
                     whole(p.k_cache, 0) && whole(p.v_cache, 0) && p.D % n == 0 &&
                     (p.interleaved || p.pairs % n == 0);
    const int per_head = vec ? p.D / n : p.D;
    int x = 1;
    while (x < per_head && x < 32) x *= 2;
    if (!p.interleaved && p.pairs && x > 1) x /= 2;
    const dim3 threads((unsigned)x, (unsigned)(kAppendThreads / x));
    if (vec)
        append_kernel<T, Vec<T>><<<(unsigned)nodes, threads, 0, st>>>(p);
    else
        append_kernel<T, One<T>><<<(unsigned)nodes, threads, 0, st>>>(p);
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
        num_pages <= 0 || page_size <= 0 || (int64_t)B * T > 0x7fffffff || (int64_t)Hq + 2 * (int64_t)Hkv > 65536)
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
