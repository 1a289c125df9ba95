// logits_rules: penalties for repeated tokens, biases and grammar masks on rows of logits.
//
// Row i of sequence b is what the target (or the draft) says after node i.  With c_v the number of times that token v
// stands in the sequence's history and on node i's path, the node itself included:
//   l' = l                                                   where c_v = 0
//        (l > 0 ? l / r : l r) - f c_v - s                   where c_v > 0   (r, f, s: repetition, frequency, presence)
//   l' = l' + bias_v, and -inf where the row's mask has no bit for v
//
// Bound by memory: a row is read and written once.  A CTA has one stretch of the vocabulary of one sequence, for a
// run of its rows: counts and biases of the stretch are gathered into shared memory once (history and biases are
// read by every stretch, from L2), with integer atomics, so that their order does not matter.  Nearly all tokens are
// touched by neither: a bitmap says which vectors of a row hold one that is, and all others go by as they came.
#include "common.cuh"
#include "draft_tree.cuh"
#include "host_util.h"
#include "launch.h"

namespace spr {

namespace {

constexpr int kRuleThreads = 256;

struct RuleParams {
    const void *logits;
    void *out;
    int64_t ldv, ld_out;
    int V, B;
    DraftNodes nodes;            // lens is not used
    const int32_t *history;
    int64_t ld_history;
    const int32_t *history_len;
    const int32_t *tokens;       // [B,T] or null
    const float *penalties;      // [B,3] or null
    const int32_t *bias_tokens;  // [B,n_bias]
    const float *bias_values;
    int n_bias;
    const uint32_t *masks;       // [num_masks, ld_mask]
    int64_t ld_mask;
    int num_masks;
    const int32_t *mask_rows;    // [B,T]
    int *status;
    int chunks, row_groups, rows_per_group;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T>
struct Lanes;            // a 16-byte vector as elements
template <>
struct Lanes<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ float get(const uint32_t (&w)[4], int e) { return __uint_as_float(w[e]); }
    static __device__ __forceinline__ void set(uint32_t (&w)[4], int e, float x) { w[e] = __float_as_uint(x); }
    static __device__ __forceinline__ void forbid(uint32_t (&w)[4], uint32_t allowed)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(allowed >> e & 1)) w[e] = 0xff800000u;
    }
};
template <>
struct Lanes<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ float get(const uint32_t (&w)[4], int e)
    {
        return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
    static __device__ __forceinline__ void set(uint32_t (&w)[4], int e, float x)
    {
        const uint32_t b = __bfloat16_as_ushort(__float2bfloat16(x));
        w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | b << 16 : (w[e >> 1] & 0xffff0000u) | b;
    }
    static __device__ __forceinline__ void forbid(uint32_t (&w)[4], uint32_t allowed)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!(allowed >> (2 * e) & 1)) w[e] = (w[e] & 0xffff0000u) | 0xff80u;
            if (!(allowed >> (2 * e + 1) & 1)) w[e] = (w[e] & 0xffffu) | 0xff800000u;
        }
    }
};

// n <= 8 bits of a bit row from bit `at` on (bits before 0 and behind `words` words read as zero)
__device__ __forceinline__ uint32_t bits_at(const uint32_t *row, int at, int words)
{
    const int w = at >> 5;
    const uint32_t lo = w >= 0 && w < words ? row[w] : 0u, hi = w + 1 >= 0 && w + 1 < words ? row[w + 1] : 0u;
    return __funnelshift_r(lo, hi, at & 31);
}

// A CTA's stretch: 16-byte vectors [chunk * VECS, (chunk + 1) * VECS) of a row, counted from the 16-byte boundary at or
// before the row's first element, so that the stretch begins up to n - 1 tokens earlier in some rows.
template <typename T, int VECS, bool ALIGNED>
__global__ void __launch_bounds__(kRuleThreads) rules_kernel(const RuleParams p)
{
    constexpr int n = Lanes<T>::n, es = sizeof(T);
    constexpr int kTokens = VECS * n + n;               // tokens first .. first + kTokens - 1 can be met
    constexpr int kWords = (kTokens + 31) / 32;
    extern __shared__ int sm[];
    int *count = sm;                                    // [kTokens]
    int *bias = sm + kTokens;                           // [kTokens] 1 + index of the bias that counts; only with biases
    __shared__ uint32_t touched[kWords + 1];
    __shared__ int near[kMaxTreeNodes];                 // nodes whose token lies in the stretch
    __shared__ int tree[kMaxTreeNodes];
    __shared__ int n_near;

    const int tid = threadIdx.x;
    const int chunk = blockIdx.x % p.chunks, group = blockIdx.x / p.chunks % p.row_groups, b = blockIdx.x / p.chunks / p.row_groups;
    const int TT = p.nodes.T, used = node_count(p.nodes, b);
    const int first = chunk * VECS * n - n;             // (n - 1 tokens would do; whole vectors are easier on the eye)
    const int row0 = group * p.rows_per_group, row1 = min(row0 + p.rows_per_group, TT);

    for (int i = tid; i < kTokens; i += kRuleThreads) {
        count[i] = 0;
        if (p.n_bias) bias[i] = 0;
    }
    for (int i = tid; i <= kWords; i += kRuleThreads) touched[i] = 0;
    if (tid == 0) n_near = 0;
    if (p.nodes.parents)
        for (int i = tid; i < TT; i += kRuleThreads) tree[i] = p.nodes.parents[(int64_t)b * TT + i];
    __syncthreads();

    auto touch = [&](int at) { atomicOr(&touched[at >> 5], 1u << (at & 31)); };
    if (p.penalties) {
        if (p.history) {
            const int len = min((int64_t)max(__ldg(p.history_len + b), 0), p.ld_history);
            const int32_t *h = p.history + (int64_t)b * p.ld_history;
            for (int i = tid; i < len; i += kRuleThreads) {
                const int t = __ldg(h + i);
                if (t >= p.V && chunk == 0) raise_status(p.status, SPR_ERR_BAD_TOKEN);
                if (t >= 0 && t < p.V && t >= first && t - first < kTokens) {
                    if (atomicAdd(&count[t - first], 1) == 0) touch(t - first);
                }
            }
        }
        if (p.tokens)
            for (int i = tid; i < used; i += kRuleThreads) {
                const int t = __ldg(p.tokens + (int64_t)b * TT + i);
                if (t >= p.V && chunk == 0) raise_status(p.status, SPR_ERR_BAD_TOKEN);
                if (t >= 0 && t < p.V && t >= first && t - first < kTokens) {
                    near[atomicAdd(&n_near, 1)] = i | (t - first) << 8;
                    touch(t - first);
                }
            }
    }
    for (int i = tid; i < p.n_bias; i += kRuleThreads) {
        const int t = __ldg(p.bias_tokens + (int64_t)b * p.n_bias + i);
        if (t >= p.V && chunk == 0) raise_status(p.status, SPR_ERR_BAD_TOKEN);
        if (t >= 0 && t < p.V && t >= first && t - first < kTokens) {
            atomicMax(&bias[t - first], i + 1);
            touch(t - first);
        }
    }
    __syncthreads();

    float repeat = 1.f, often = 0.f, there = 0.f;
    if (p.penalties) {
        repeat = __ldg(p.penalties + 3 * b);
        often = __ldg(p.penalties + 3 * b + 1);
        there = __ldg(p.penalties + 3 * b + 2);
    }
    const int nn = n_near;
    const int mask_words = (p.V + 31) / 32;

    // whether node j is node i or on its path
    auto on_path = [&](int j, int i) {
        if (!p.nodes.parents) return j <= i;
        while (i > j) i = checked_parent(tree[i], i, p.status);
        return i == j;
    };
    auto changed = [&](float x, int at, int row) {
        int c = count[at];
        for (int m = 0; m < nn; ++m)
            if (near[m] >> 8 == at && on_path(near[m] & 255, row)) ++c;
        if (c > 0) x = (x > 0.f ? x / repeat : x * repeat) - often * (float)c - there;
        if (p.n_bias) {
            const int k = bias[at];
            if (k) x += __ldg(p.bias_values + (int64_t)b * p.n_bias + k - 1);
        }
        return x;
    };

    for (int row = row0; row < row1; ++row) {
        const int64_t r = (int64_t)b * TT + row;
        const T *src = static_cast<const T *>(p.logits) + r * p.ldv;
        T *dst = static_cast<T *>(p.out) + r * p.ld_out;
        const bool rules = row < used;
        const uint32_t *mask = nullptr;
        if (rules && p.masks) {
            const int m = __ldg(p.mask_rows + r);
            if (m >= p.num_masks) {
                if (tid == 0 && chunk == 0) raise_status(p.status, SPR_ERR_BAD_ROW);
            } else if (m >= 0)
                mask = p.masks + (int64_t)m * p.ld_mask;
        }
        if (ALIGNED) {
            const int lead = (int)(reinterpret_cast<uintptr_t>(src) % 16) / es;   // the same in dst
#pragma unroll
            for (int u = 0; u < VECS / kRuleThreads; ++u) {
                const int v = chunk * VECS + u * kRuleThreads + tid;
                const int c = v * n - lead;                  // the vector's first token
                if (c >= p.V) continue;
                if (c >= 0 && c + n <= p.V) {
                    const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(src + c));
                    uint32_t w[4] = {a.x, a.y, a.z, a.w};
                    if (rules) {
                        uint32_t t = bits_at(touched, c - first, kWords + 1) & ((1u << n) - 1);
                        while (t) {
                            const int e = __ffs(t) - 1;
                            t &= t - 1;
#pragma unroll
                            for (int f = 0; f < n; ++f)
                                if (f == e) Lanes<T>::set(w, f, changed(Lanes<T>::get(w, f), c + f - first, row));
                        }
                        if (mask) Lanes<T>::forbid(w, bits_at(mask, c, mask_words));
                    }
                    __stcs(reinterpret_cast<uint4 *>(dst + c), make_uint4(w[0], w[1], w[2], w[3]));
                    continue;
                }
                for (int e = 0; e < n; ++e)
                    if (c + e >= 0 && c + e < p.V) {
                        T x = src[c + e];
                        if (rules) {
                            if (bits_at(touched, c + e - first, kWords + 1) & 1) x = (T)changed(to_float(x), c + e - first, row);
                            if (mask && !(bits_at(mask, c + e, mask_words) & 1)) x = (T)neg_inf();
                        }
                        dst[c + e] = x;
                    }
            }
        } else {
            // rows of input and output that lie differently on 16-byte boundaries: one element at a time
            for (int i = tid; i < VECS * n; i += kRuleThreads) {
                const int c = chunk * VECS * n + i;
                if (c >= p.V) break;
                T x = src[c];
                if (rules) {
                    if (bits_at(touched, c - first, kWords + 1) & 1) x = (T)changed(to_float(x), c - first, row);
                    if (mask && !(bits_at(mask, c, mask_words) & 1)) x = (T)neg_inf();
                }
                dst[c] = x;
            }
        }
    }
}

template <typename T, int VECS, bool ALIGNED>
cudaError_t launch_rules(const RuleParams &p, unsigned ctas, cudaStream_t st)
{
    constexpr int tokens = VECS * Lanes<T>::n + Lanes<T>::n;
    const size_t smem = (size_t)tokens * 4 * (p.n_bias ? 2 : 1);
    if (smem > 40000) {
        const cudaError_t e = cudaFuncSetAttribute(rules_kernel<T, VECS, ALIGNED>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * tokens * 4);
        if (e != cudaSuccess) return e;
    }
    rules_kernel<T, VECS, ALIGNED><<<ctas, kRuleThreads, smem, st>>>(p);
    return cudaGetLastError();
}

template <typename T>
cudaError_t pick_rules(RuleParams &p, bool same, cudaStream_t st)
{
    constexpr int n = Lanes<T>::n, kLong = 1024, kShort = 256;
    const int T_ = p.nodes.T;
    auto chunks_of = [&](int vecs) { return (int)(((int64_t)p.V + n - 1 + (int64_t)vecs * n - 1) / ((int64_t)vecs * n)); };
    const bool wide = (int64_t)p.B * chunks_of(kLong) >= 148 * 2;
    p.chunks = chunks_of(wide ? kLong : kShort);
    // few sequences: their rows are dealt out too
    int64_t groups = (148 * 4 + (int64_t)p.B * p.chunks - 1) / ((int64_t)p.B * p.chunks);
    if (groups > T_) groups = T_;
    p.rows_per_group = (int)((T_ + groups - 1) / groups);
    p.row_groups = (T_ + p.rows_per_group - 1) / p.rows_per_group;
    const int64_t ctas = (int64_t)p.B * p.chunks * p.row_groups;
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    if (wide) return same ? launch_rules<T, kLong, true>(p, (unsigned)ctas, st) : launch_rules<T, kLong, false>(p, (unsigned)ctas, st);
    return same ? launch_rules<T, kShort, true>(p, (unsigned)ctas, st) : launch_rules<T, kShort, false>(p, (unsigned)ctas, st);
}

}  // namespace

}  // namespace spr

using namespace spr;

extern "C" int logits_rules(const void *logits, int64_t ldv, int V, int B, int T, int dt, const int32_t *history, int64_t ld_history,
                            const int32_t *history_len, const int32_t *tokens, const int32_t *parents, const int32_t *counts,
                            const float *penalties, const int32_t *bias_tokens, const float *bias_values, int n_bias,
                            const uint32_t *masks, int64_t ld_mask, int num_masks, const int32_t *mask_rows, void *out,
                            int64_t ld_out, void *ws, size_t ws_bytes, void *cuda_stream)
{
    if (!dtype_ok(dt)) return SPR_ERR_UNSUPPORTED;
    if (B < 0 || T < 0 || V <= 0 || V > 1 << 30 || ldv < V || ld_out < V || (int64_t)B * T > 0x7fffffff || n_bias < 0 || n_bias > 1024)
        return SPR_ERR_INVALID_ARG;
    if (T > kMaxTreeNodes) return SPR_ERR_UNSUPPORTED;
    if (B == 0 || T == 0) return SPR_OK;
    const size_t es = elem_size(dt);
    if (!logits || !out || !aligned(logits, es) || !aligned(out, es)) return SPR_ERR_INVALID_ARG;
    if ((history && (!history_len || ld_history < 0)) || (n_bias && (!bias_tokens || !bias_values)) ||
        (masks && (!mask_rows || num_masks <= 0 || ld_mask < ((int64_t)V + 31) / 32)))
        return SPR_ERR_INVALID_ARG;
    if (!aligned(history, 4) || !aligned(history_len, 4) || !aligned(tokens, 4) || !aligned(parents, 4) || !aligned(counts, 4) ||
        !aligned(penalties, 4) || !aligned(bias_tokens, 4) || !aligned(bias_values, 4) || !aligned(masks, 4) || !aligned(mask_rows, 4))
        return SPR_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < (size_t)kHeaderBytes) return SPR_ERR_WORKSPACE;
    const int rc = device_supported();
    if (rc != SPR_OK) return rc;
    RuleParams p = {};
    p.logits = logits, p.out = out, p.ldv = ldv, p.ld_out = ld_out, p.V = V, p.B = B;
    p.nodes = DraftNodes{nullptr, counts, parents, T};
    p.history = history, p.ld_history = ld_history, p.history_len = history_len, p.tokens = tokens;
    p.penalties = penalties, p.bias_tokens = bias_tokens, p.bias_values = bias_values, p.n_bias = n_bias;
    p.masks = masks, p.ld_mask = ld_mask, p.num_masks = num_masks, p.mask_rows = mask_rows;
    p.status = static_cast<int *>(ws);
    // every row of both lies alike on 16-byte boundaries
    const bool same = (reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(out)) % 16 == 0 && (ldv - ld_out) * (int64_t)es % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return finish(dt == SPR_F32 ? pick_rules<float>(p, same, st) : pick_rules<__nv_bfloat16>(p, same, st));
}
