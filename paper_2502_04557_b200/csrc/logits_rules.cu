// logits_rules: penalties for repeated tokens, biases and grammar masks on rows of logits.
//
// Row i of sequence b is what the target (or the draft) says after node i.  With c_v the number of times that token v
// stands in the sequence's history and on node i's path, the node itself included:
//   l' = l                                                   where c_v = 0
//        (l > 0 ? l / r : l r) - f c_v - s                   where c_v > 0   (r, f, s: repetition, frequency, presence)
//   l' = l' + bias_v, and -inf where the row's mask has no bit for v
//
// Bound by memory: a row is read and written once.  A CTA has one stretch of the vocabulary of one sequence, for a run of
// its rows, which go through a ring in shared memory by bulk copies.  The stretch's counts and biases are gathered into tables
// once (history and biases are read by every stretch, from L2), with integer atomics, so that their order does not matter.
// Nearly all tokens are touched by neither: those that are stand in a list, up to four to a thread (or are looked for), and are put right in the
// ring; masks are applied there to vectors, with their bits read a row ahead.  Rows by 8 KB for many sequences, 4 KB for few.
// 256 x 17 rows of 128256 bf16 entries, a quarter masked: 410 us, 5.5 TB/s.  More rows in the ring take
// CTAs from the SM (4 stages 490 us), two leave the copies too little (508 us).
#include <atomic>

#include "host_util.h"
#include "launch.h"
#include "rules.cuh"
#include "tensor_pair.cuh"

namespace spr {

namespace {

using namespace pairtc;

constexpr int kMaxStages = 3;         // rows of a CTA that are on their way

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_addr(bar))
                 : "memory");
}
__device__ __forceinline__ void bulk_store(void *dst, uint32_t src, uint32_t bytes)
{
    asm volatile(
        "cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes)
        : "memory");
}

// A CTA's stretch: BYTES bytes of each row, counted from the 16-byte boundary at or before the row's first element, so that
// the stretch begins up to a vector less one token earlier in some rows.
template <typename T, int BYTES>
struct Stretch {
    static constexpr int n = 16 / sizeof(T), vecs = BYTES / 16;
    static constexpr int tokens = vecs * n + n;         // tokens first .. first + tokens - 1 can be met
    static constexpr int words = (tokens + 31) / 32;
    static constexpr int threads = BYTES / 32;          // two vectors each
    static size_t smem(int stages, int biases, int nodes)      // nodes of a tree
    {
        return (size_t)stages * BYTES + tokens * 4 + (biases ? tokens * 2 + 4 * biases : 0) + (nodes + 31) / 32 * nodes * 4;
    }
};

template <typename T, int BYTES>
__global__ void __launch_bounds__(Stretch<T, BYTES>::threads) rules_kernel(const RuleParams p)
{
    using S = Stretch<T, BYTES>;
    constexpr int n = S::n, es = sizeof(T), kTokens = S::tokens, kWords = S::words, kRuleThreads = S::threads, kListed = 4 * kRuleThreads;
    extern __shared__ __align__(128) uint8_t sm[];
    int *count = reinterpret_cast<int *>(sm + p.stages * BYTES);                      // [kTokens]; kRuleOnPath: some node has the token
    uint32_t *bias = reinterpret_cast<uint32_t *>(count + kTokens);                  // [kTokens] of 16 bits: 1 + the bias that counts
    float *bias_value = reinterpret_cast<float *>(bias + kTokens / 2);              // [n_bias]
    // [T][path_words]: a bit for each node on a node's path, where there is a tree
    uint32_t *path = p.n_bias ? reinterpret_cast<uint32_t *>(bias_value + p.n_bias) : bias;
    const int path_words = (p.nodes.T + 31) / 32;
    __shared__ uint64_t full[kMaxStages];
    __shared__ uint16_t listed[kListed];                // touched tokens, in any order
    __shared__ uint32_t touched[kWords];
    __shared__ int near[kMaxTreeNodes];                 // nodes whose token lies in the stretch
    __shared__ int tree[kMaxTreeNodes];
    __shared__ int mask_of[kMaxTreeNodes];              // the rows' masks, negative: none
    __shared__ int n_near, n_listed, abort;

    const int tid = threadIdx.x;
    const int chunk = blockIdx.x % p.pieces, group = blockIdx.x / p.pieces % p.row_groups, b = blockIdx.x / p.pieces / p.row_groups;
    const int TT = p.nodes.T, used = node_count(p.nodes, b);
    const int v0 = chunk * S::vecs;                     // the stretch's first vector
    const int first = v0 * n - n;                       // (n - 1 tokens would do; whole vectors are easier on the eye)
    const int row0 = group * p.rows_per_group, row1 = min(row0 + p.rows_per_group, TT);

    // a row's elements before its first 16-byte boundary, and its vectors [va, vb) in the stretch that are whole: those
    // are copied by the copy engine, others one element at a time
    struct Span {
        const T *src;
        T *dst;
        int lead, va, vb;
    };
    auto span = [&](int row) {
        Span s;
        const int64_t r = (int64_t)b * TT + row;
        s.src = static_cast<const T *>(p.logits) + r * p.ldv;
        s.dst = static_cast<T *>(p.out) + r * p.ld_out;
        s.lead = p.same ? (int)(reinterpret_cast<uintptr_t>(s.src) % 16) / es : 0;
        s.va = v0 + (v0 == 0 && s.lead ? 1 : 0);
        s.vb = p.same ? min(v0 + S::vecs, (p.V + s.lead) / n) : s.va;
        return s;
    };
    auto fetch = [&](int row) {
        const Span s = span(row);
        const int stage = (row - row0) % p.stages;
        const uint32_t bytes = s.vb > s.va ? (uint32_t)(s.vb - s.va) * 16 : 0u;
        bar_expect(&full[stage], bytes);        // (a phase for every row, whatever there is to copy)
        if (bytes) bulk_load(smem_addr(sm) + stage * BYTES + (s.va - v0) * 16, s.src + (s.va * n - s.lead), bytes, &full[stage]);
    };

    int fetched = min(row0 + p.stages, row1);            // thread 0: the row that is fetched next
    if (tid == 0) {
        for (int i = 0; i < kMaxStages; ++i) bar_init(&full[i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        n_near = n_listed = abort = 0;
        for (int row = row0; row < fetched; ++row) fetch(row);
    }
    // everything that the stretch's counts are made of is asked for before any of it is looked at
    constexpr int kAhead = 8;
    const bool counted = p.penalties && p.history;
    const int32_t *h = p.history + (int64_t)b * p.ld_history;
    int ahead[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) ahead[u] = counted && u * kRuleThreads + tid < p.ld_history ? __ldg(h + u * kRuleThreads + tid) : -1;
    const int64_t len = counted ? min((int64_t)max(__ldg(p.history_len + b), 0), p.ld_history) : 0;
    const int my_token = p.penalties && p.tokens && tid < used ? __ldg(p.tokens + (int64_t)b * TT + tid) : -1;
    const int my_bias = tid < p.n_bias ? __ldg(p.bias_tokens + (int64_t)b * p.n_bias + tid) : -1;
    for (int i = tid; i < p.n_bias; i += kRuleThreads) bias_value[i] = __ldg(p.bias_values + (int64_t)b * p.n_bias + i);
    float repeat = 1.f, often = 0.f, there = 0.f;
    if (p.penalties) {
        repeat = __ldg(p.penalties + 3 * b);
        often = __ldg(p.penalties + 3 * b + 1);
        there = __ldg(p.penalties + 3 * b + 2);
    }
    for (int i = tid; i < kTokens / 4; i += kRuleThreads) reinterpret_cast<int4 *>(count)[i] = make_int4(0, 0, 0, 0);
    if (p.n_bias)
        for (int i = tid; i < kTokens / 2; i += kRuleThreads) bias[i] = 0;
    for (int i = tid; i < kWords; i += kRuleThreads) touched[i] = 0;
    if (p.nodes.parents)
        for (int i = tid; i < used; i += kRuleThreads) tree[i] = checked_parent(__ldg(p.nodes.parents + (int64_t)b * TT + i), i, p.status);
    for (int i = row0 + tid; i < row1; i += kRuleThreads) {
        int m = p.masks && i < used ? __ldg(p.mask_rows + (int64_t)b * TT + i) : -1;
        if (m >= p.num_masks) {
            if (chunk == 0) raise_status(p.status, SPR_ERR_BAD_ROW);
            m = -1;
        }
        mask_of[i] = m;
    }
    __syncthreads();
    if (p.nodes.parents)
        for (int i = tid; i < used; i += kRuleThreads) {
            for (int w = 0; w < path_words; ++w) path[i * path_words + w] = 0;
            for (int j = i; j >= 0; j = tree[j]) path[i * path_words + (j >> 5)] |= 1u << (j & 31);
        }

    auto within = [&](int t) {
        if (t >= p.V && chunk == 0) raise_status(p.status, SPR_ERR_BAD_TOKEN);
        return t >= 0 && t < p.V && t >= first && t - first < kTokens;
    };
    auto touch = [&](int at) {
        const uint32_t bit = 1u << (at & 31);
        if (atomicOr(&touched[at >> 5], bit) & bit) return;
        const int i = atomicAdd(&n_listed, 1);
        if (i < kListed) listed[i] = (uint16_t)at;
    };
    auto count_one = [&](int t) {
        if (within(t)) {
            atomicAdd(&count[t - first], 1);
            touch(t - first);
        }
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (u * kRuleThreads + tid < len) count_one(ahead[u]);
    for (int64_t i = kAhead * kRuleThreads + tid; i < len; i += kRuleThreads) count_one(__ldg(h + i));
    auto node_token = [&](int i, int t) {
        if (within(t)) {
            near[atomicAdd(&n_near, 1)] = i | (t - first) << 8;
            atomicOr(&count[t - first], kRuleOnPath);
            touch(t - first);
        }
    };
    if (my_token >= 0) node_token(tid, my_token);
    if (p.penalties && p.tokens)
        for (int i = tid + kRuleThreads; i < used; i += kRuleThreads) node_token(i, __ldg(p.tokens + (int64_t)b * TT + i));
    auto bias_token = [&](int i, int t) {
        if (!within(t)) return;
        const int at = t - first, sh = 16 * (at & 1);
        uint32_t old = bias[at >> 1];
        while ((old >> sh & 0xffffu) < (uint32_t)i + 1) {        // the largest index stays
            const uint32_t seen = atomicCAS(&bias[at >> 1], old, (old & ~(0xffffu << sh)) | (uint32_t)(i + 1) << sh);
            if (seen == old) break;
            old = seen;
        }
        touch(at);
    };
    if (my_bias >= 0) bias_token(tid, my_bias);
    for (int i = tid + kRuleThreads; i < p.n_bias; i += kRuleThreads) bias_token(i, __ldg(p.bias_tokens + (int64_t)b * p.n_bias + i));
    __syncthreads();

    const int nn = n_near, nl = n_listed;
    const int mask_words = (p.V + 31) / 32;

    // whether node j is node i or on its path
    auto on_path = [&](int j, int i) { return p.nodes.parents ? (path[i * path_words + (j >> 5)] >> (j & 31) & 1) != 0 : j <= i; };

    auto bias_of = [&](int at) {
        const uint32_t i = p.n_bias ? bias[at >> 1] >> (16 * (at & 1)) & 0xffffu : 0u;
        return i ? make_float2(bias_value[i - 1], 1.f) : make_float2(0.f, 0.f);
    };
    // the rules for one token of a row; c: its count with kRuleOnPath, w: its bias and whether there is one
    auto fix = [&](int at, int c, float2 w, int shift, int row, T *buf) {
        const int pos = at + first + shift;
        if (pos < 0 || pos >= S::vecs * n) return;
        if (c & kRuleOnPath) {
            c &= ~kRuleOnPath;
            for (int m = 0; m < nn; ++m)
                if (near[m] >> 8 == at && on_path(near[m] & 255, row)) ++c;
        }
        if (c == 0 && w.y == 0.f) return;           // on other paths only: its bits stay as they are
        float x = (float)buf[pos];
        if (c > 0) x = (x > 0.f ? x / repeat : x * repeat) - often * (float)c - there;
        if (w.y != 0.f) x += w.x;
        buf[pos] = (T)x;
    };
    // a thread keeps its first token
    int mine_at = 0, mine_count = 0;
    float2 mine_bias = make_float2(0.f, 0.f);
    if (tid < min(nl, kListed)) {
        mine_at = listed[tid];
        mine_count = count[mine_at];
        mine_bias = bias_of(mine_at);
    }
    // the mask's bits of this thread's vectors of a row, read one row ahead
    constexpr int kEach = S::vecs / kRuleThreads;
    uint32_t allowed[kEach], allowed_next[kEach];
    auto mask_bits = [&](int row, uint32_t (&bits)[kEach]) {
        if (row >= row1 || mask_of[row] < 0) return;
        const uint32_t *mask = p.masks + mask_of[row] * p.ld_mask;
        const int shift = span(row).lead - v0 * n;
#pragma unroll
        for (int u = 0; u < kEach; ++u) bits[u] = bits_at(mask, (u * kRuleThreads + tid) * n - shift, mask_words);
    };
    mask_bits(row0, allowed_next);
    int row = row0;
    for (; row < row1; ++row) {
        const Span s = span(row);
        const int stage = (row - row0) % p.stages;
        T *buf = reinterpret_cast<T *>(sm + stage * BYTES);         // token c at c + lead - v0 n
        const int shift = s.lead - v0 * n;
        const bool rules = row < used;
#pragma unroll
        for (int u = 0; u < kEach; ++u) allowed[u] = allowed_next[u];
        mask_bits(row + 1, allowed_next);
        // tokens [c0, c1) that go one by one: of the vector before va and of the one at vb, or all of them
        auto singles = [&](auto f) {
            if (!p.same) {
                const int end = min(p.V, (v0 + S::vecs) * n);
                for (int c = v0 * n + tid; c < end; c += kRuleThreads) f(c);
                return;
            }
            if (tid >= 2 * n) return;
            const int v = tid < n ? v0 : s.vb, c = v * n + tid % n - s.lead;
            const bool mine = tid < n ? s.va > v0 : s.vb >= s.va && s.vb < v0 + S::vecs;
            if (mine && c >= 0 && c < p.V) f(c);
        };
        singles([&](int c) { buf[c + shift] = s.src[c]; });
        bar_wait(&full[stage], (uint32_t)((row - row0) / p.stages) & 1, &abort, p.status, kSpinLimit);
        if (!p.same || s.va != v0 || s.vb != v0 + S::vecs) __syncthreads();         // (those that went one by one)
        if (rules) {
            if (nl <= kListed) {
                if (tid < nl) fix(mine_at, mine_count, mine_bias, shift, row, buf);
                for (int k = tid + kRuleThreads; k < nl; k += kRuleThreads) {
                    const int at = listed[k];
                    fix(at, count[at], bias_of(at), shift, row, buf);
                }
            } else {
                for (int at = tid; at < kTokens; at += kRuleThreads)
                    if (touched[at >> 5] >> (at & 31) & 1) fix(at, count[at], bias_of(at), shift, row, buf);
            }
            if (mask_of[row] >= 0) {
                __syncthreads();
#pragma unroll
                for (int u = 0; u < kEach; ++u) {
                    uint4 *at = reinterpret_cast<uint4 *>(buf) + u * kRuleThreads + tid;
                    const uint4 a = *at;
                    uint32_t w[4] = {a.x, a.y, a.z, a.w};
                    RuleLanes<T>::forbid(w, allowed[u]);
                    *at = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
        fence_stores();
        __syncthreads();
        if (abort) break;
        singles([&](int c) { s.dst[c] = buf[c + shift]; });
        if (tid == 0) {
            if (s.vb > s.va)
                bulk_store(s.dst + (s.va * n - s.lead), smem_addr(buf) + (s.va - v0) * 16, (uint32_t)(s.vb - s.va) * 16);
            // the row before this one has left its stage: the next one may come
            asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 1;" ::: "memory");
            if (row > row0 && fetched < row1) fetch(fetched++);
        }
    }
    if (tid == 0) {
        stores_read();
        // copies in flight write shared memory: none may be left when the CTA ends
        for (; row < fetched; ++row) bar_wait_quiet(&full[(row - row0) % p.stages], (uint32_t)((row - row0) / p.stages) & 1, kSpinLimit);
    }
}

template <typename T, int BYTES>
cudaError_t launch_rules(const RuleParams &p, unsigned ctas, cudaStream_t st)
{
    const size_t smem = Stretch<T, BYTES>::smem(p.stages, p.n_bias, p.nodes.parents ? p.nodes.T : 0);
    if (smem > 40000) {
        static std::atomic<bool> attr_set[64];   // host threads may race to set it: all of them store `true`
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
            e = cudaFuncSetAttribute(rules_kernel<T, BYTES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)Stretch<T, BYTES>::smem(kMaxStages, kRuleMaxBiases, kMaxTreeNodes));
            if (e != cudaSuccess) return e;
            if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
        }
    }
    rules_kernel<T, BYTES><<<ctas, Stretch<T, BYTES>::threads, smem, st>>>(p);
    return cudaGetLastError();
}

// Few rows, and stretches of the vocabulary beyond what is resident at once, go to logits_rules_single.cu: a stretch's tables
// take longer than its rows.  256x1 over 128256 entries 69 -> 33 us (history of 4000: 102 -> 55), 64x3 34 -> 24 us, 24x1
// 10.3 -> 7.7 us; but 256x4 147 -> 149 us, and 64x1 over 32000 entries, 512 stretches, 7.0 -> 7.8 us.
constexpr int kSingleRows = 3, kSingleStretches = 148 * 4;

template <typename T>
cudaError_t pick_rules(RuleParams &p, cudaStream_t st)
{
    constexpr int n = 16 / sizeof(T), kLong = 8192, kShort = 4096;
    const int rows = p.nodes.T;
    auto chunks_of = [&](int bytes) { return (int)(((int64_t)p.V + n - 1 + bytes / sizeof(T) - 1) / (bytes / (int64_t)sizeof(T))); };
    const bool wide = (int64_t)p.B * chunks_of(kLong) >= 148 * 4;
    if (rows <= kSingleRows && (int64_t)p.B * chunks_of(kLong) >= kSingleStretches) return launch_rules_single<T>(p, st);
    p.pieces = chunks_of(wide ? kLong : kShort);
    // few sequences: their rows are dealt out too, to as many CTAs as are resident (8 short stretches an SM rather than 4: 8x9 over
    // 50257 entries 12.6 -> 9.5 us, 116x26x6130 90 -> 54 us; 16: 12.4 and 57)
    int64_t groups = 148 * (wide ? 4 : 8) / ((int64_t)p.B * p.pieces);
    groups = groups < 1 ? 1 : groups > rows ? rows : groups;
    p.rows_per_group = (int)((rows + groups - 1) / groups);
    p.stages = p.rows_per_group < kMaxStages ? p.rows_per_group : kMaxStages;
    p.row_groups = (rows + p.rows_per_group - 1) / p.rows_per_group;
    const int64_t ctas = (int64_t)p.B * p.pieces * p.row_groups;
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    return wide ? launch_rules<T, kLong>(p, (unsigned)ctas, st) : launch_rules<T, kShort>(p, (unsigned)ctas, st);
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
    if (B < 0 || T < 0 || V <= 0 || V > 1 << 30 || ldv < V || ld_out < V || (int64_t)B * T > 0x7fffffff || n_bias < 0 || n_bias > kRuleMaxBiases)
        return SPR_ERR_INVALID_ARG;
    if (T > kMaxTreeNodes) return SPR_ERR_UNSUPPORTED;
    if (B == 0 || T == 0) return SPR_OK;
    const size_t es = elem_size(dt);
    if (!logits || !out || !aligned(logits, es) || !aligned(out, es) || (logits == out && ldv != ld_out)) return SPR_ERR_INVALID_ARG;
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
    p.same = (reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(out)) % 16 == 0 && (ldv - ld_out) * (int64_t)es % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return finish(dt == SPR_F32 ? pick_rules<float>(p, st) : pick_rules<__nv_bfloat16>(p, st));
}
