// How tree_attention's work is dealt out, and how the parts of an item are joined.
//
// An item is a row block of one cached head of one sequence: up to ROWS of its count * G queries (rows are ordered by
// node, then by query head), over all of the sequence's keys in tiles of 64.  The tiles of all items stand in one line
// (by sequence, head, row block, tile) and each CTA takes an equal stretch of it, whatever the lengths, so that
// the split follows the lengths that the device holds and a captured launch serves all of them.  A stretch begins and
// ends inside items.  Parts of an item go to the workspace, and the CTA that takes the last ticket of an item joins
// its parts in their order; nothing waits on another CTA.
#pragma once

#include "attention.h"

namespace spr {

struct AttnSeq {
    int b, len, count, tiles, blocks;    // blocks = row blocks
    __device__ __forceinline__ int total(int Hkv) const { return tiles * blocks * Hkv; }
};

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
    const int own = tid < p.B ? attn_seq<ROWS>(p, tid).total(p.Hkv) : 0;
    int before = 0, total = 0;       // tiles of the sequences below b0, and of all
    if (p.B > THREADS) {             // the line's length first
        int mine = own;
        for (int b = tid + THREADS; b < p.B; b += THREADS) mine += attn_seq<ROWS>(p, b).total(p.Hkv);
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) scratch[warp] = mine;
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
            const int active = min(p.ctas, (int)((uint32_t)(total + LEAST - 1) / LEAST));
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
    if (!t.whole) {
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
// last, whose CTA may then read all records (behind another barrier).
__device__ __forceinline__ bool attn_ticket(const AttnParams &p, const AttnTarget &t)
{
    __threadfence();
    const bool last = take_ticket(p.counters + t.first, t.parts);
    __threadfence();
    return last;
}

// Joins the parts of an item; called by all lanes of `warps` warps of the CTA that took its last ticket.  A warp has a row at
// a time, a lane one part's maximum and sum and then four columns; ROWS_AT_ONCE rows are on their way together.
template <int ROWS, typename T>
__device__ __forceinline__ void attn_join(const AttnParams &p, const AttnStretch &s, const AttnPart &part, const AttnTarget &t,
                                          int warp, int warps)
{
    constexpr int N = 4;
    const int lane = threadIdx.x & 31, c = lane * 4;
    auto slot_of = [&](int k) { return 2 * (t.first + k) + (k == 0 ? 1 : 0); };
    for (int row0 = warp * N; row0 < t.rows; row0 += warps * N) {
        float top[N], sum[N];
        float4 o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            top[i] = neg_inf();
            sum[i] = 0.f;
            o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        for (int k0 = 0; k0 < t.parts; k0 += 32) {      // 32 parts at a time, as in one pass over keys
            auto fetch = [&](int k, float4 (&x)[N]) {
                const float *from = p.part + ((int64_t)slot_of(k0 + k) * ROWS + row0) * p.D + c;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[i] = c < p.D && row0 + i < t.rows && k0 + k < t.parts ? __ldcg(reinterpret_cast<const float4 *>(from + (int64_t)i * p.D))
                                                                            : make_float4(0.f, 0.f, 0.f, 0.f);
            };
            float4 x[N], y[N];
            fetch(0, x);            // (two parts' results are asked for before their weights are known)
            fetch(1, y);
            float2 ml[N];
            float w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool there = k0 + lane < t.parts && row0 + i < t.rows;
                ml[i] = there ? __ldcg(&p.part_ml[(int64_t)slot_of(k0 + lane) * ROWS + row0 + i]) : make_float2(neg_inf(), 0.f);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float m = fmaxf(top[i], warp_max(ml[i].x)), ref = m == neg_inf() ? 0.f : m, a = ex2(top[i] - ref);
                top[i] = m;
                w[i] = ex2(ml[i].x - ref);          // (a part that saw nothing has 0 and zeros)
                sum[i] = sum[i] * a + warp_sum(w[i] * ml[i].y);
                o[i].x *= a, o[i].y *= a, o[i].z *= a, o[i].w *= a;
            }
            const int n = min(32, t.parts - k0);
            auto add = [&](int k, const float4 (&x)[N]) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float a = __shfl_sync(0xffffffffu, w[i], k);
                    o[i].x = fmaf(a, x[i].x, o[i].x), o[i].y = fmaf(a, x[i].y, o[i].y), o[i].z = fmaf(a, x[i].z, o[i].z), o[i].w = fmaf(a, x[i].w, o[i].w);
                }
            };
            for (int k = 0; k < n; k += 2) {
                add(k, x);
                if (k + 2 < n) fetch(k + 2, x);
                if (k + 1 < n) add(k + 1, y);
                if (k + 3 < n) fetch(k + 3, y);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (row0 + i < t.rows) {
                const float inv = sum[i] == 0.f ? 0.f : 1.f / sum[i];
                store_out(static_cast<T *>(p.out) + attn_out_at(p, s, part, t.row0 + row0 + i) + c,
                          make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv), p.D - c);
            }
    }
}

}  // namespace spr
