// logits_rules where the rows are few beside the sequences: a decoding step of many sequences.  logits_rules.cu has the
// formulas.
//
// Bound by memory: a row is read and written once.  A CTA has a piece of the vocabulary of one sequence, for a run of its rows.
// The tokens of the piece that stand in the history, on nodes or among the biases are gathered once, in a hash table in
// shared memory (counts by integer atomics, so that their order does not matter): they are few beside a row, and the piece can be
// as long as balance allows.  A row then goes from registers to registers' places, in vectors, masked on the way, and the
// touched tokens' values, which were read before, are written over it.  A piece with more touched tokens than the table holds is
// taken in shorter stretches.  256 x 1 rows of 128256 bf16 entries: 40 us with 2048 tokens of history each, 22 us (6.1 TB/s) with none.
#include "rules.cuh"

namespace spr {

namespace {

constexpr int kRuleThreads = 256;
constexpr int kRuleCtasPerSm = 4;     // 64 registers a thread
constexpr int kSlots = 2048;          // of the table
constexpr int kListed = 1536;         // touched tokens; each thread may be putting in one more when these are full
static_assert(kListed + kRuleThreads < kSlots, "a search of the table ends at a free slot");

template <typename T>
__global__ void __launch_bounds__(kRuleThreads, kRuleCtasPerSm) rules_single_kernel(const RuleParams p)
{
    constexpr int n = 16 / sizeof(T), es = sizeof(T);
    __shared__ int key[kSlots];             // tokens, or -1
    __shared__ int count[kSlots];           // kRuleOnPath: some node has the token
    __shared__ int bias[kSlots];            // 1 + the bias that counts
    __shared__ uint16_t listed[kListed];    // slots in use, in any order
    __shared__ T value[2][kListed];         // what becomes of the listed tokens, in rows by turns
    __shared__ int near[kMaxTreeNodes];     // nodes whose token is in the table: the node, and its slot above
    __shared__ int tree[kMaxTreeNodes];
    __shared__ int mask_of[kMaxTreeNodes];  // the rows' masks, negative: none
    __shared__ int n_near, n_listed;

    const int tid = threadIdx.x;
    const int piece = blockIdx.x % p.pieces, group = blockIdx.x / p.pieces % p.row_groups, b = blockIdx.x / p.pieces / p.row_groups;
    const int TT = p.nodes.T, used = node_count(p.nodes, b);
    const int row0 = group * p.rows_per_group, row1 = min(row0 + p.rows_per_group, TT);

    const bool counted = p.penalties && p.history, on_nodes = p.penalties && p.tokens;
    const int64_t len = counted ? min((int64_t)max(__ldg(p.history_len + b), 0), p.ld_history) : 0;
    float repeat = 1.f, often = 0.f, there = 0.f;
    if (p.penalties) {
        repeat = __ldg(p.penalties + 3 * b);
        often = __ldg(p.penalties + 3 * b + 1);
        there = __ldg(p.penalties + 3 * b + 2);
    }
    for (int i = tid; i < kSlots / 4; i += kRuleThreads) {
        reinterpret_cast<int4 *>(key)[i] = make_int4(-1, -1, -1, -1);
        reinterpret_cast<int4 *>(count)[i] = make_int4(0, 0, 0, 0);
        reinterpret_cast<int4 *>(bias)[i] = make_int4(0, 0, 0, 0);
    }
    if (p.nodes.parents)
        for (int i = tid; i < used; i += kRuleThreads) tree[i] = checked_parent(__ldg(p.nodes.parents + (int64_t)b * TT + i), i, p.status);
    for (int i = row0 + tid; i < row1; i += kRuleThreads) {
        int m = p.masks && i < used ? __ldg(p.mask_rows + (int64_t)b * TT + i) : -1;
        if (m >= p.num_masks) {
            if (piece == 0) raise_status(p.status, SPR_ERR_BAD_ROW);
            m = -1;
        }
        mask_of[i] = m;
    }
    if (tid == 0) n_near = n_listed = 0;
    __syncthreads();

    // A stretch of the piece: vectors [v0, v1) of each row, counted from the 16-byte boundary at or before the row's first
    // element, so that it begins up to a vector less one token earlier in some rows: tokens [first, last) can be met.
    const int mask_words = (p.V + 31) / 32, vectors = (int)(((int64_t)p.V + 2 * n - 2) / n);
    const int piece1 = min((piece + 1) * p.piece, vectors);
    int v0 = piece * p.piece, step = p.piece;
    while (v0 < piece1) {
        const int v1 = min(v0 + step, piece1);
        const int first = max(v0 * n - (n - 1), 0), last = min(v1 * n, p.V);
        auto slot_of = [&](int t) -> int {
            if (t >= p.V && piece == 0) raise_status(p.status, SPR_ERR_BAD_TOKEN);
            if (t < first || t >= last) return -1;
            int s = (int)((uint32_t)t * 0x9e3779b1u >> 21);
            for (int i = 0; i < kSlots; ++i, s = (s + 1) & (kSlots - 1)) {
                const int there = *const_cast<volatile int *>(key + s);
                if (there == t) return s;
                if (there != -1) continue;
                if (*const_cast<volatile int *>(&n_listed) >= kListed) break;
                const int old = atomicCAS(key + s, -1, t);
                if (old == t) return s;
                if (old != -1) continue;
                const int at = atomicAdd(&n_listed, 1);
                if (at < kListed) listed[at] = (uint16_t)s;
                return s;
            }
            n_listed = kListed + kRuleThreads;          // too many (as it would be with this one)
            return -1;
        };
        // everything is asked for before any of it is looked at
        constexpr int kAhead = 8;
        const int32_t *h = p.history + (int64_t)b * p.ld_history, *tok = p.tokens + (int64_t)b * TT;
        const int32_t *bt = p.bias_tokens + (int64_t)b * p.n_bias;
        const int my_token = on_nodes && tid < used ? __ldg(tok + tid) : -1;        // (T <= 256)
        const int my_bias = tid < p.n_bias ? __ldg(bt + tid) : -1;
        for (int64_t i0 = tid; i0 < len; i0 += kAhead * kRuleThreads) {
            int ahead[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) ahead[u] = i0 + u * kRuleThreads < len ? __ldg(h + i0 + u * kRuleThreads) : -1;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int s = slot_of(ahead[u]);
                if (s >= 0) atomicAdd(count + s, 1);
            }
        }
        if (my_token >= 0) {
            const int s = slot_of(my_token);
            if (s >= 0) {
                near[atomicAdd(&n_near, 1)] = tid | s << 8;
                atomicOr(count + s, kRuleOnPath);
            }
        }
        for (int i = tid; i < p.n_bias; i += kRuleThreads) {
            const int s = slot_of(i == tid ? my_bias : __ldg(bt + i));
            if (s >= 0) atomicMax(bias + s, i + 1);
        }
        __syncthreads();
        const int nn = n_near, nl = n_listed;
        const bool fits = nl <= kListed;

        struct Span {
            const T *src;
            T *dst;
            int lead, va, vb;        // elements before the first boundary; the stretch's vectors [va, vb) that are whole
        };
        auto span = [&](int row) {
            Span s;
            const int64_t r = (int64_t)b * TT + row;
            s.src = static_cast<const T *>(p.logits) + r * p.ldv;
            s.dst = static_cast<T *>(p.out) + r * p.ld_out;
            s.lead = p.same ? (int)(reinterpret_cast<uintptr_t>(s.src) % 16) / es : 0;
            s.va = v0 + (v0 == 0 && s.lead ? 1 : 0);
            s.vb = p.same ? min(v1, (p.V + s.lead) / n) : s.va;
            return s;
        };
        auto mask_row = [&](int row) -> const uint32_t * { return mask_of[row] < 0 ? nullptr : p.masks + mask_of[row] * p.ld_mask; };
        auto may = [&](const uint32_t *mask, int c) { return !mask || (__ldg(mask + (c >> 5)) >> (c & 31) & 1); };
        // whether node j is node i or on its path
        auto on_path = [&](int j, int i) {
            if (!p.nodes.parents) return j <= i;
            while (i > j) i = tree[i];
            return i == j;
        };
        // the rules for the token in a slot
        auto fix = [&](int s, int row, T l) {
            int c = count[s];
            if (c & kRuleOnPath) {
                c &= ~kRuleOnPath;
                for (int m = 0; m < nn; ++m)
                    if (near[m] >> 8 == s && on_path(near[m] & 255, row)) ++c;
            }
            const int w = bias[s];
            if (c == 0 && w == 0) return l;         // on other paths only: its bits stay as they are
            float x = (float)l;
            if (c > 0) x = (x > 0.f ? x / repeat : x * repeat) - often * (float)c - there;
            if (w) x += __ldg(p.bias_values + (int64_t)b * p.n_bias + w - 1);
            return (T)x;
        };
        // the listed tokens of a row: read before any of the row is written
        auto read_listed = [&](int row) {
            if (row >= row1 || row >= used) return;
            const Span s = span(row);
            const uint32_t *mask = mask_row(row);
            constexpr int kTogether = 2;
            for (int i = tid; i < nl; i += kTogether * kRuleThreads) {
                T l[kTogether];
                bool ok[kTogether];
                int slot[kTogether];
#pragma unroll
                for (int u = 0; u < kTogether; ++u) {
                    slot[u] = i + u * kRuleThreads < nl ? listed[i + u * kRuleThreads] : -1;
                    if (slot[u] < 0) continue;
                    const int t = key[slot[u]];
                    l[u] = s.src[t];
                    ok[u] = may(mask, t);
                }
#pragma unroll
                for (int u = 0; u < kTogether; ++u)
                    if (slot[u] >= 0) value[row & 1][i + u * kRuleThreads] = ok[u] ? fix(slot[u], row, l[u]) : (T)neg_inf();
            }
        };
        auto write_listed = [&](int row) {
            if (row >= used) return;
            const Span s = span(row);
            for (int i = tid; i < nl; i += kRuleThreads) {
                const int t = key[listed[i]], v = (t + s.lead) / n;
                if (v >= v0 && v < v1) s.dst[t] = value[row & 1][i];
            }
        };
        if (fits) {
            read_listed(row0);
            __syncthreads();
            for (int row = row0; row < row1; ++row) {
                const Span s = span(row);
                const uint32_t *mask = mask_row(row);
                constexpr int kTogether = 4;
                for (int v = s.va + tid; v < s.vb; v += kTogether * kRuleThreads) {
                    uint4 x[kTogether];
                    uint32_t allowed[kTogether];
#pragma unroll
                    for (int u = 0; u < kTogether; ++u) {
                        const int k = v + u * kRuleThreads;
                        if (k >= s.vb) continue;
                        x[u] = __ldcs(reinterpret_cast<const uint4 *>(s.src + (k * n - s.lead)));
                        if (mask) allowed[u] = s.lead ? bits_at(mask, k * n - s.lead, mask_words) : __ldg(mask + k * n / 32) >> (k * n & 31);
                    }
#pragma unroll
                    for (int u = 0; u < kTogether; ++u) {
                        const int k = v + u * kRuleThreads;
                        if (k >= s.vb) continue;
                        uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
                        if (mask) RuleLanes<T>::forbid(w, allowed[u]);
                        __stcs(reinterpret_cast<uint4 *>(s.dst + (k * n - s.lead)), make_uint4(w[0], w[1], w[2], w[3]));
                    }
                }
                // what is left goes one by one: before va and from vb on, or all of it
                const int c0 = max(v0 * n - s.lead, 0), c1 = min(v1 * n - s.lead, p.V), left = max(s.vb - s.va, 0) * n;
                const int head = left ? s.va * n - s.lead - c0 : 0;
                for (int i = tid; i < c1 - c0 - left; i += kRuleThreads) {
                    const int c = c0 + i + (i >= head ? left : 0);
                    const T x = s.src[c];
                    s.dst[c] = may(mask, c) ? x : (T)neg_inf();
                }
                read_listed(row + 1);
                __syncthreads();
                write_listed(row);
            }
            v0 = v1;
        } else {
            step = max((v1 - v0) / 2, kListed / n - 1);      // (a stretch of that many vectors has no more tokens than the list)
        }
        if (v0 < piece1) {
            __syncthreads();
            for (int i = tid; i < kSlots; i += kRuleThreads) key[i] = -1, count[i] = bias[i] = 0;
            if (tid == 0) n_near = n_listed = 0;
            __syncthreads();
        }
    }
}

}  // namespace

template <typename T>
cudaError_t launch_rules_single(RuleParams &p, cudaStream_t st)
{
    constexpr int n = 16 / sizeof(T);
    constexpr int64_t kCtas = 148 * kRuleCtasPerSm;
    const int rows = p.nodes.T;
    const int64_t vectors = ((int64_t)p.V + 2 * n - 2) / n;
    // pieces of a row: a CTA for every place on the GPU, so many that the table holds an even share of the tokens, and no fewer
    // than a vector for every thread
    int64_t pieces = kCtas / p.B;
    const int64_t by_tokens = (p.ld_history + rows + p.n_bias) / 1024;
    pieces = pieces < by_tokens ? by_tokens : pieces;
    const int64_t most = (vectors + kRuleThreads - 1) / kRuleThreads;
    pieces = pieces > most ? most : pieces < 1 ? 1 : pieces;
    p.piece = (int)((vectors + pieces - 1) / pieces);
    p.pieces = (int)((vectors + p.piece - 1) / p.piece);
    // few sequences: their rows are dealt out too
    int64_t groups = kCtas / ((int64_t)p.B * p.pieces);
    groups = groups < 1 ? 1 : groups > rows ? rows : groups;
    p.rows_per_group = (int)((rows + groups - 1) / groups);
    p.row_groups = (rows + p.rows_per_group - 1) / p.rows_per_group;
    const int64_t ctas = (int64_t)p.B * p.pieces * p.row_groups;
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    rules_single_kernel<T><<<(unsigned)ctas, kRuleThreads, 0, st>>>(p);
    return cudaGetLastError();
}

template cudaError_t launch_rules_single<float>(RuleParams &, cudaStream_t);
template cudaError_t launch_rules_single<__nv_bfloat16>(RuleParams &, cudaStream_t);

}  // namespace spr
