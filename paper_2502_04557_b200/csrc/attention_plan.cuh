// How tree_attention's work is dealt out, and how the parts of an item are joined.
//
// An item is a row block of one cached head of one sequence: up to ROWS of its count * G queries (rows are ordered by
// node, then by query head), over all of the sequence's keys in tiles of 64.  The tiles of all items stand in one line
// (by sequence, head, row block, tile) and each CTA takes an equal stretch of it, whatever the lengths, so that
// the split follows the lengths that the device holds and a captured launch serves all of them.  A stretch begins and
// ends inside items.  Where there is little to do, each CTA gets a piece of one item instead, if there are CTAs enough: a
// stretch of two parts would take two ends of parts.  Parts of an item go to the workspace, and the CTA that takes the last
// ticket of an item joins its parts in their order; nothing waits on another CTA.
#pragma once

#include "attention.h"

namespace spr {

struct AttnSeq {
    int b, len, count, tiles, blocks;    // blocks = row blocks
    __device__ __forceinline__ int total(int Hkv) const { return tiles * blocks * Hkv; }
};

// The maximum of a row that has seen keys, all with scores of -inf.  They have no weight beside any other score (parts are joined as ever),
// but where there is none the row's softmax is 0 / 0, unlike a row's that has seen no key (-inf): that is zeros.
constexpr float kOnlyMinusInf = -3.402823466e38f;
__device__ __forceinline__ float attn_top(float scaled, bool saw) { return scaled == neg_inf() && saw ? kOnlyMinusInf : scaled; }
// what a row's results are multiplied by in the end
__device__ __forceinline__ float attn_inverse(float top, float sum) { return sum == 0.f && top == neg_inf() ? 0.f : 1.f / sum; }

// keys of a sequence: its prefix and its nodes, as far as the page table goes
__device__ __forceinline__ int attn_keys(const AttnParams &p, int len, int count) { return (int)min((int64_t)len + count, p.capacity); }

template <int ROWS>
__device__ __forceinline__ AttnSeq attn_seq(const AttnParams &p, int b)
{
    AttnSeq s;
    s.b = b;
    s.len = __ldg(p.nodes.lens + b);
    s.count = s.len < 0 ? 0 : node_count(p.nodes, b);
    s.tiles = s.count ? (int)((uint32_t)(attn_keys(p, s.len, s.count) + kAttnTile - 1) / kAttnTile) : 0;
    s.blocks = (s.count * p.G + ROWS - 1) / ROWS;
    return s;
}

// Where this CTA's stretch lies, in tiles of the line (fewer than 2^31: the host sees to it).  The first `longer` CTAs have
// one tile more than the others.
struct AttnStretch {
    int pos, end;
    int each, longer;
    int first, pieces;       // (pieces > 0) of one item: the CTA with the first, and how many there are
    AttnSeq seq;             // the sequence that pos lies in
    int at;                  // pos within it

    __device__ __forceinline__ int owner(int x) const
    {
        const int lower = longer * (each + 1);
        return x < lower ? x / (each + 1) : longer + (x - lower) / each;
    }
};

// Part of an item: tiles [t0, t0 + n) of it.
struct AttnPart {
    int head, block, t0, n;
};

template <int ROWS>
__device__ __forceinline__ bool attn_next(const AttnParams &p, AttnStretch &s, AttnPart &part)
{
    if (s.pos >= s.end) return false;
    for (int n; s.at >= (n = s.seq.total(p.Hkv));) {
        s.at -= n;
        s.seq = attn_seq<ROWS>(p, s.seq.b + 1);
    }
    const int item = s.at / s.seq.tiles;
    part.t0 = s.at - item * s.seq.tiles;
    part.head = s.seq.blocks == 1 ? item : item / s.seq.blocks;
    part.block = item - part.head * s.seq.blocks;
    part.n = min(s.seq.tiles - part.t0, s.end - s.pos);
    s.pos += part.n;
    s.at += part.n;
    return true;
}

// Called by all THREADS threads of the CTA.  `scratch`: THREADS / 32 + 2 words.  LEAST: the fewest tiles that
// are worth a CTA of their own: an item's parts have to be joined, which takes as long as some tiles.
template <int ROWS, int THREADS, int LEAST>
__device__ __forceinline__ AttnStretch attn_plan(const AttnParams &p, int *scratch)
{
    constexpr int W = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = blockIdx.x;
    AttnStretch s;
    int least = LEAST;
    constexpr int kFewTiles = 16;    // per CTA
    AttnSeq mine = {0, 0, 0, 0, 0};
    if (tid < p.B) mine = attn_seq<ROWS>(p, tid);
    const int own = mine.total(p.Hkv);
    int before = 0, total = 0;       // tiles of the sequences below b0, and of all
    if (p.B > THREADS) {             // the line's length first
        int sum = own;
        for (int b = tid + THREADS; b < p.B; b += THREADS) sum += attn_seq<ROWS>(p, b).total(p.Hkv);
        sum = __reduce_add_sync(0xffffffffu, sum);
        if (lane == 0) scratch[warp] = sum;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) total += scratch[w];
        __syncthreads();
    }
    // the sequence that holds the stretch's first tile
    for (int b0 = 0;; b0 += THREADS) {
        const int b = b0 + tid;
        const int n = b0 == 0 ? own : b < p.B ? attn_seq<ROWS>(p, b).total(p.Hkv) : 0;
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 31) scratch[warp] = incl;
        __syncthreads();
        int lower = before, sum = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w < warp) lower += scratch[w];
            sum += scratch[w];
        }
        if (b0 == 0) {
            if (p.B <= THREADS) total = sum;
            s.first = s.pieces = 0;
            if (p.B <= THREADS && total <= p.ctas * kFewTiles && total > 0) {
                // pieces of items, none longer than the stretches would be
                const int most = max(LEAST, (total + p.ctas - 1) / p.ctas), per = (mine.tiles + most - 1) / most;
                const int pieces = per * mine.blocks * p.Hkv;
                int upto = pieces;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += up;
                }
                __syncthreads();
                if (lane == 31) scratch[warp] = upto;
                __syncthreads();
                int all = 0;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if (w < warp) upto += scratch[w];
                    all += scratch[w];
                }
                if (all <= p.ctas) {
                    s.pos = s.end = s.at = s.longer = 0;
                    s.each = 1;
                    s.seq = AttnSeq{0, 0, 0, 0, 0};
                    if (c >= all) return s;
                    if (c >= upto - pieces && c < upto) {
                        scratch[W] = b;
                        scratch[W + 1] = c - (upto - pieces);
                    }
                    __syncthreads();
                    s.seq = attn_seq<ROWS>(p, scratch[W]);
                    s.pieces = (s.seq.tiles + most - 1) / most;
                    const int item = scratch[W + 1] / s.pieces, piece = scratch[W + 1] - item * s.pieces;
                    const int t0 = piece * s.seq.tiles / s.pieces;
                    s.first = c - piece;
                    s.end = (piece + 1) * s.seq.tiles / s.pieces - t0;
                    s.at = item * s.seq.tiles + t0;
                    return s;
                }
                // more items than CTAs, of two tiles or three: short stretches cut few of them (32 sequences of 100 and 9 nodes, 12
                // heads of 64: 28.7 -> 16.4 us; of 250, four tiles each: 19.3 -> 21.1, as before)
                if (total < 4 * p.ctas) least = 1;
            }
            const int active = min(p.ctas, (int)((uint32_t)(total + least - 1) / least));
            if (c >= active) {
                s.pos = s.end = s.at = s.longer = 0;
                s.each = 1;
                s.seq = AttnSeq{0, 0, 0, 0, 0};
                return s;
            }
            s.each = total / active;
            s.longer = total - s.each * active;
            s.pos = c * s.each + min(c, s.longer);
            s.end = s.pos + s.each + (c < s.longer ? 1 : 0);
        }
        const int at = s.pos - (lower + incl - n);
        if (at >= 0 && at < n) {
            scratch[W] = b;
            scratch[W + 1] = at;
        }
        before += sum;
        __syncthreads();
        if (before > s.pos) break;
    }
    s.seq = attn_seq<ROWS>(p, scratch[W]);
    s.at = scratch[W + 1];
    return s;
}

// Rows of nodes that are not used: zeros.  Dealt out over all CTAs by sequence.
template <typename T>
__device__ __forceinline__ void attn_clear_unused(const AttnParams &p, int threads)
{
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        const int used = __ldg(p.nodes.lens + b) < 0 ? 0 : node_count(p.nodes, b);
        const int64_t row = (int64_t)p.Hq * p.D;
        uint4 *out = reinterpret_cast<uint4 *>(static_cast<T *>(p.out) + ((int64_t)b * p.nodes.T + used) * row);
        const int64_t n = (p.nodes.T - used) * row * (int64_t)sizeof(T) / 16;
        for (int64_t i = threadIdx.x; i < n; i += threads) out[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

// Bits of the nodes that node i sees: itself and its path.  `tree`: the sequence's parents in shared memory, or null.
__device__ __forceinline__ void attn_path_bits(const int *tree, int i, uint32_t *bits, int words, int *status)
{
    for (int w = 0; w < words; ++w) {
        const int below = i + 1 - 32 * w;
        bits[w] = tree ? 0u : below >= 32 ? 0xffffffffu : below > 0 ? (1u << below) - 1 : 0u;
    }
    if (!tree) return;
    for (int j = i; j >= 0; j = checked_parent(tree[j], j, status)) bits[j >> 5] |= 1u << (j & 31);
}

// four results of one row, as they are written
__device__ __forceinline__ void store_out(float *p, float4 x, int left)
{
    if (left >= 4)
        *reinterpret_cast<float4 *>(p) = x;
}
__device__ __forceinline__ void store_out(__nv_bfloat16 *p, float4 x, int left)
{
    if (left < 4) return;
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

// What becomes of a part: the item's result where the part is all of it, else a record in the workspace.
struct AttnTarget {
    bool whole;
    int slot;            // record of this part
    int first, parts;    // (parts of an item) the CTA that has its first tile, and how many have some
    int row0;            // first row of the block
    int rows;            // rows of the block in use
};
template <int ROWS>
__device__ __forceinline__ AttnTarget attn_target(const AttnParams &p, const AttnStretch &s, const AttnPart &part)
{
    AttnTarget t;
    t.whole = part.n == s.seq.tiles;
    t.slot = 2 * blockIdx.x + (part.t0 == 0 ? 1 : 0);
    t.first = t.parts = 0;
    if (s.pieces) {
        t.first = s.first;
        t.parts = s.pieces;
    } else if (!t.whole) {
        const int begin = s.pos - part.n - part.t0;          // (pos already behind the part)
        t.first = s.owner(begin);
        t.parts = s.owner(begin + s.seq.tiles - 1) - t.first + 1;
    }
    t.row0 = part.block * ROWS;
    t.rows = min(ROWS, s.seq.count * p.G - part.block * ROWS);
    return t;
}
__device__ __forceinline__ int64_t attn_out_at(const AttnParams &p, const AttnStretch &s, const AttnPart &part, int row)
{
    const int i = row / p.G, g = row - i * p.G;
    return (((int64_t)s.seq.b * p.nodes.T + i) * p.Hq + (int64_t)part.head * p.G + g) * p.D;
}

// One ticket of the part's item, taken by one thread behind a barrier of those that wrote the part's record; true for the
// last, whose CTA may then read all records (behind another barrier).  The counter is zero again after the last.
__device__ __forceinline__ bool attn_ticket(const AttnParams &p, const AttnTarget &t)
{
    uint32_t old;
    asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(old) : "l"(p.counters + t.first), "r"((uint32_t)t.parts - 1u) : "memory");
    return old == (uint32_t)t.parts - 1u;
}

// Joins the parts of an item; called by all lanes of `warps` warps of the CTA that took its last ticket.  A warp has N rows at a
// time, a lane four columns of them; K parts are on their way together, and are taken in as a pass over keys takes in keys.
template <int ROWS, typename T>
__device__ __forceinline__ void attn_join(const AttnParams &p, const AttnStretch &s, const AttnPart &part, const AttnTarget &t,
                                          int warp, int warps)
{
    constexpr int N = 4, K = 4;
    const int c = (threadIdx.x & 31) * 4;
    for (int row0 = warp * N; row0 < t.rows; row0 += warps * N) {
        float top[N], sum[N];
        float4 o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            top[i] = neg_inf();
            sum[i] = 0.f;
            o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll 1
        for (int k0 = 0; k0 < t.parts; k0 += K) {
            float2 ml[K][N];
            float4 x[K][N];
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int64_t at = (int64_t)(2 * (t.first + k0 + k) + (k0 + k == 0 ? 1 : 0)) * ROWS + row0 + i;
                    const bool there = k0 + k < t.parts && row0 + i < t.rows;
                    ml[k][i] = there ? __ldcg(p.part_ml + at) : make_float2(neg_inf(), 0.f);
                    x[k][i] = there && c < p.D ? __ldcg(reinterpret_cast<const float4 *>(p.part + at * p.D + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float m = top[i];
#pragma unroll
                for (int k = 0; k < K; ++k) m = fmaxf(m, ml[k][i].x);
                const float ref = m == neg_inf() ? 0.f : m, a = ex2(top[i] - ref);
                top[i] = m;
                sum[i] *= a;
                o[i].x *= a, o[i].y *= a, o[i].z *= a, o[i].w *= a;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const float w = ex2(ml[k][i].x - ref);      // (a part that saw nothing has 0 and zeros)
                    sum[i] = fmaf(w, ml[k][i].y, sum[i]);
                    o[i].x = fmaf(w, x[k][i].x, o[i].x), o[i].y = fmaf(w, x[k][i].y, o[i].y);
                    o[i].z = fmaf(w, x[k][i].z, o[i].z), o[i].w = fmaf(w, x[k][i].w, o[i].w);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (row0 + i < t.rows) {
                const float inv = attn_inverse(top[i], sum[i]);
                store_out(static_cast<T *>(p.out) + attn_out_at(p, s, part, t.row0 + row0 + i) + c,
                          make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv), p.D - c);
            }
    }
}

}  // namespace spr
