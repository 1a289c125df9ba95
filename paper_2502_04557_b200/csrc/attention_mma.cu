// tree_attention on bf16 tensors, few rows per cached head (decoding, chains).
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j in one pass over the keys, with a running maximum and sum.  Bound by the
// read of the caches: a key and its value (4 D bytes) meet ROWS queries.  Each of a CTA's four warps takes 16 keys of every
// tile of 64, which it brings into a ring of its own (cp.async, 16 bytes per lane, three to five steps ahead) and works on
// alone: it has its own maxima, sums and results (mma.sync m16n8k16, the block's rows as M), and warps meet only at the end of
// a part, behind which the SM's other CTA goes on.  Copies by lanes take pages as they come: the copy engine's boxes of a
// page of 16 entries are 2 KB each, and their number, not their bytes, sets the time (64 sequences of 4096 tokens, 8 heads
// of 128: 195 us with such boxes).  mma.sync suffices here: at 16 rows a tile of 32 KB (the time of 1400 clocks at the memory's
// rate) takes 128 products per tensor core, some 300 clocks; tcgen05's smallest tile has 64 rows.
//
// 64 sequences of some 3000 tokens, 32/8 heads of 128: 135 us, 6.0 TB/s; one of 131072: 102 us; one of
// 300: 11 us, the length of the chain from the plan to the join.
//
// Weights are used as two bf16 numbers (their rounding and what is left of it), off by up to 2^-17 of themselves: with one
// it would be 2^-8, and results could be off by as much of sum p |v|, more than by their own rounding where values cancel.  The second product is free where the
// memory is what bounds it.
#include <atomic>

#include "attention_plan.cuh"
#include "host_util.h"
#include "launch.h"
#include "tensor_pair.cuh"

namespace spr {

namespace {

using pairtc::pack_bf16;
using pairtc::smem_addr;

constexpr int kMmaThreads = 128;
constexpr int kMmaWarps = kMmaThreads / 32;
constexpr int kJoinCols = 32;                           // columns that are joined at once
constexpr int kJoinPitch = kJoinCols + 4;               // floats per row of the joining buffer
constexpr int kJoinBytes = kMmaWarps * 16 * kJoinPitch * 4;

template <int PANELS>
struct MmaShape {
    static constexpr int row = 128 * PANELS;                    // bytes of a key in the ring
    static constexpr int step = 2 * 16 * row;                   // a warp's 16 keys, then their values
    static constexpr int stages = PANELS == 2 ? 3 : 5;
    static constexpr size_t smem = (size_t)kMmaWarps * stages * step + kJoinBytes;
};

struct MmaControl {
    int scratch[kMmaWarps + 2];
    int tree[16];
    uint32_t path[16];                      // nodes' paths, a bit for each node
    float2 ml[kMmaWarps][16];
    uint32_t valid[kMmaWarps][5];           // a bit for each key of a warp's step that is there
    int last;
};

__device__ __forceinline__ void ldsm(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there)      // or zeros
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// two values as they are, but the largest finite numbers in place of infinities and NaN
__device__ __forceinline__ uint32_t finite_part(uint32_t w)
{
    uint32_t r;
    asm("min.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0x7f7f7f7fu));
    return r;
}
__device__ __forceinline__ bool finite_bf16x2(uint32_t w) { return (w & 0x7f80u) != 0x7f80u && (w & 0x7f800000u) != 0x7f800000u; }

// PANELS: 64-column halves of the head dimension; WHOLE: which it is made of
template <int PANELS, bool WHOLE>
__global__ void __launch_bounds__(kMmaThreads, 2) attention_mma_kernel(const AttnParams p)
{
    constexpr int ROWS = 16, KSTEPS = 4 * PANELS, NTILES = 8 * PANELS;
    using Shape = MmaShape<PANELS>;
    extern __shared__ __align__(1024) uint8_t raw[];
    __shared__ MmaControl ctl;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t ring = smem_addr(raw) + warp * Shape::stages * Shape::step;
    float *join = reinterpret_cast<float *>(raw + (size_t)kMmaWarps * Shape::stages * Shape::step);
    const int w16 = warp * 16;                              // keys w16 .. + 15 of a tile

    AttnStretch s = attn_plan<ROWS, kMmaThreads, 6>(p, ctl.scratch);
    attn_clear_unused<__nv_bfloat16>(p, kMmaThreads);

    // ---------------------------------------------------------------- copies, some steps ahead of the products
    AttnStretch ahead = s;
    AttnPart next_part = {0, 0, 0, 0};
    bool more = true;
    int next_tile = 0, end_tile = 0, left_rows = 0;     // the next tile; left_rows: steps whose rows are in `rows`
    int next_keys = 0;
    int next_stage = 0;
    int rows = -1, rows_behind = -1;                    // lane 2 j + r: row of the caches where run r (8 keys) of step j begins
    auto find = [&](int tile) {                         // for 16 steps from this tile on
        const int t = tile + (lane >> 1);
        const int slot = t * kAttnTile + w16 + 8 * (lane & 1);
        if (t >= end_tile || slot >= next_keys) return -1;
        const int at = slot / p.page_size;
        const int page = __ldg(p.page_table + (int64_t)ahead.seq.b * p.max_pages + at);
        if (page < 0 || page >= p.num_pages) {
            raise_status(p.status, SPR_ERR_BAD_PAGE);
            return -1;
        }
        return (page * p.Hkv + next_part.head) * p.page_size + (slot - at * p.page_size);
    };
    // lane's 16 bytes of a row
    constexpr int kChunks = 8 * PANELS, kRowsAtOnce = 32 / kChunks;
    const int c_row = lane / kChunks, c_chunk = lane % kChunks;
    const bool c_in = c_chunk * 8 < p.D;
    const uint32_t c_dst = c_row * Shape::row + ((c_chunk ^ c_row) << 4);
    auto issue = [&]() {
        while (more && next_tile >= end_tile) {         // on to the next part
            more = attn_next<ROWS>(p, ahead, next_part);
            if (!more) break;
            next_keys = attn_keys(p, ahead.seq.len, ahead.seq.count);
            if (next_keys < (int64_t)ahead.seq.len + ahead.seq.count) raise_status(p.status, SPR_ERR_BAD_PAGE);
            next_tile = next_part.t0;
            end_tile = next_part.t0 + next_part.n;
            left_rows = 0;
            rows_behind = find(next_tile);
        }
        if (more) {
            if (left_rows == 0) {
                rows = rows_behind;
                left_rows = 16;
                rows_behind = find(next_tile + 16);
            }
            const int from = 2 * (16 - left_rows);
            const uint32_t dst = ring + next_stage * Shape::step + c_dst;
            const int run[2] = {__shfl_sync(0xffffffffu, rows, from), __shfl_sync(0xffffffffu, rows, from + 1)};
            const int keys = next_keys - next_tile * kAttnTile - w16;      // of this step that there are
            const uint32_t valid = ((run[0] >= 0 ? 0xffu : 0u) | (run[1] >= 0 ? 0xff00u : 0u)) & (keys >= 16 ? 0xffffu : keys <= 0 ? 0u : (1u << keys) - 1);
            if (lane == 0) ctl.valid[warp][next_stage] = valid;
            if (WHOLE && valid == 0xffffu) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int64_t at = ((int64_t)run[r] + c_row) * (64 * PANELS) + c_chunk * 8;
                    const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(p.k) + at, *v = static_cast<const __nv_bfloat16 *>(p.v) + at;
#pragma unroll
                    for (int r0 = 0; r0 < 8; r0 += kRowsAtOnce) {
                        const uint32_t to = (dst ^ (r0 << 4)) + (8 * r + r0) * Shape::row;
                        copy16(to, k + r0 * 64 * PANELS);
                        copy16(to + 16 * Shape::row, v + r0 * 64 * PANELS);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
                    const int r0 = i * kRowsAtOnce, r = r0 + c_row;
                    const bool there = c_in && (valid >> r & 1);
                    const int64_t at = there ? ((int64_t)run[r0 >> 3] + (r & 7)) * p.D + c_chunk * 8 : 0;
                    const uint32_t to = (dst ^ ((r0 & 7) << 4)) + r0 * Shape::row;
                    copy16(to, static_cast<const __nv_bfloat16 *>(p.k) + at, there);
                    copy16(to + 16 * Shape::row, static_cast<const __nv_bfloat16 *>(p.v) + at, there);
                }
            }
            ++next_tile;
            --left_rows;
        }
        copies_commit();
        next_stage = next_stage + 1 == Shape::stages ? 0 : next_stage + 1;
    };
    // ---------------------------------------------------------------- products
    // ldmatrix addresses: keys (non-transposed): matrices (keys 0-7 | 8-15) x (columns 0-7 | 8-15); values transposed
    const int k_row = (lane & 7) + ((lane >> 4) << 3), k_chunk = (lane >> 3) & 1;
    const int v_row = (lane & 7) + (((lane >> 3) & 1) << 3), v_chunk = lane >> 4;
    const uint32_t k_off = k_row * Shape::row, v_off = (16 + v_row) * Shape::row;
    const int swz = lane & 7;                               // both rows are lane & 7 modulo 8
    const int quad = lane >> 2, pair = lane & 3;
    // There is one block of rows, all of a sequence's queries of a cached head: which node a row belongs to, and where its row of
    // q and out lies behind the part's first, does not change.
    auto offset = [&](int r) { return (r / p.G * p.Hq + r % p.G) * p.D; };
    const int node[2] = {quad / p.G, (quad + 8) / p.G}, q_at[2] = {offset(quad), offset(quad + 8)}, join_at = offset(tid >> 3);
    auto first_row = [&](const AttnStretch &s, const AttnPart &part) {
        return ((int64_t)s.seq.b * p.nodes.T * p.Hq + (int64_t)part.head * p.G) * p.D;
    };
    // a part's queries as A fragments: rows quad and quad + 8 of each row tile.  They are asked for while what comes before
    // the part is still going on.
    uint32_t qf[KSTEPS][4];
    auto load_queries = [&](const AttnStretch &s, const AttnPart &part) {
        const int rows = s.seq.count * p.G;
        const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.q) + first_row(s, part);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool in = h * 8 + quad < rows;
            const uint32_t *src = reinterpret_cast<const uint32_t *>(q + (in ? q_at[h] : 0));
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int col = k * 16 + c * 8 + pair * 2;
                    qf[k][c * 2 + h] = in && col < p.D ? src[col / 2] : 0u;        // (not __ldg: out may be q)
                }
        }
    };
    AttnPart part;
    int tree_of = -1, stage = 0;
    bool have = attn_next<ROWS>(p, s, part);
    if (have) load_queries(s, part);
#pragma unroll 1
    for (int i = 0; i < Shape::stages; ++i) issue();
    while (have) {
        const AttnTarget t = attn_target<ROWS>(p, s, part);
        if ((part.t0 + part.n) * kAttnTile > s.seq.len) {       // the part holds nodes
            __syncthreads();
            if (p.nodes.parents && tree_of != s.seq.b) {
                if (tid < s.seq.count) ctl.tree[tid] = p.nodes.parents[(int64_t)s.seq.b * p.nodes.T + tid];
                tree_of = s.seq.b;
                __syncthreads();
            }
            if (tid < s.seq.count) attn_path_bits(p.nodes.parents ? ctl.tree : nullptr, tid, ctl.path + tid, 1, p.status);
            __syncthreads();
        }
        if (p.flip) {
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
                for (int c = 0; c < 4; ++c) qf[k][c] ^= p.flip;
        }

        float o[NTILES][4], m[2], l[2];
        m[0] = m[1] = neg_inf();
        l[0] = l[1] = 0.f;
        uint32_t saw = 0;                   // a bit for each of the two rows: one of the lane's keys has been seen
#pragma unroll
        for (int n = 0; n < NTILES; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
        for (int n = 0; n < part.n; ++n) {
            copies_wait<Shape::stages - 1>();
            __syncwarp();
            const uint32_t base = ring + stage * Shape::step;
            const uint32_t valid = ctl.valid[warp][stage];
            const int slot0 = (part.t0 + n) * kAttnTile + w16;
            const bool all = valid == 0xffffu && slot0 + 16 <= s.seq.len;

            float sc[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) sc[h][0] = sc[h][1] = sc[h][2] = sc[h][3] = 0.f;
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k) {
                uint32_t b[4];
                ldsm(base + k_off + (((k * 2 + k_chunk) ^ swz) << 4), b);
                mma(sc[0], qf[k], b[0], b[1]);
                mma(sc[1], qf[k], b[2], b[3]);
            }
            uint32_t odd = 0;               // keys whose values hold infinities or NaN, where not every row sees every key
            if (!all) {
                // they are taken out of the product and added one by one to the rows that see them
                bool bad = false;
#pragma unroll
                for (int c = 0; c < 4 * PANELS; ++c) {
                    uint32_t x[4];
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                                 : "r"(base + (16 + (lane & 15)) * Shape::row + ((lane >> 4) * 4 * PANELS + c) * 16) : "memory");
                    bad = bad || !(finite_bf16x2(x[0]) && finite_bf16x2(x[1]) && finite_bf16x2(x[2]) && finite_bf16x2(x[3]));
                }
                odd = __ballot_sync(0xffffffffu, bad);
                odd = (odd | odd >> 16) & 0xffffu;
            }
            // c registers 0, 1: row quad, keys 2 pair, 2 pair + 1; 2, 3: row quad + 8
            if (!all) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int key = h * 8 + pair * 2 + (c & 1);
                        const int j = slot0 + key - s.seq.len;
                        const bool vis = (valid >> key & 1) && (j < 0 || (ctl.path[node[c >> 1]] >> j & 1));
                        if (vis)
                            saw |= 1u << (c >> 1);
                        else
                            sc[h][c] = neg_inf();
                    }
            } else {
                saw = 3;
            }
            float top[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float x = fmaxf(fmaxf(sc[0][2 * g], sc[0][2 * g + 1]), fmaxf(sc[1][2 * g], sc[1][2 * g + 1]));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                top[g] = fmaxf(x, m[g]);
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const float a = ex2((m[g] - (top[g] == neg_inf() ? 0.f : top[g])) * p.abs_scale_log2);
                    m[g] = top[g];
                    l[g] *= a;
#pragma unroll
                    for (int i = 0; i < NTILES; ++i) {
                        o[i][2 * g] *= a;
                        o[i][2 * g + 1] *= a;
                    }
                }
            }
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const float ref = m[g] == neg_inf() ? 0.f : -m[g] * p.abs_scale_log2;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float w = ex2(fmaf(sc[h][2 * g + c], p.abs_scale_log2, ref));
                        sc[h][2 * g + c] = w;
                        l[g] += w;
                    }
            }
            if (odd) {
                for (int key = 0; key < 16; ++key) {
                    if (!(odd >> key & 1)) continue;
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const int h = key >> 3, c = key & 1, from = (lane & 28) | ((key & 7) >> 1);
                        const float w0 = h ? sc[1][2 * g] : sc[0][2 * g], w1 = h ? sc[1][2 * g + 1] : sc[0][2 * g + 1];
                        const float w = __shfl_sync(0xffffffffu, c ? w1 : w0, from);
                        const int j = slot0 + key - s.seq.len;
                        if (j < 0 || (ctl.path[node[g]] >> j & 1)) {
#pragma unroll
                            for (int i = 0; i < NTILES; ++i) {
                                const uint32_t a = base + (16 + key) * Shape::row + ((i ^ (key & 7)) << 4) + pair * 4;
                                uint32_t x;
                                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(a) : "memory");
                                o[i][2 * g] = fmaf(w, __uint_as_float(x << 16), o[i][2 * g]);
                                o[i][2 * g + 1] = fmaf(w, __uint_as_float(x & 0xffff0000u), o[i][2 * g + 1]);
                            }
                        }
                    }
                }
                __syncwarp();
                if (odd >> (lane & 15) & 1)
                    for (int c = 0; c < 4 * PANELS; ++c)
                        asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(base + (16 + (lane & 15)) * Shape::row + ((lane >> 4) * 4 * PANELS + c) * 16), "r"(0u) : "memory");
                __syncwarp();
            }
            // weights as A fragments, in two parts
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const float a = sc[h][2 * g], b = sc[h][2 * g + 1];
                    const uint32_t w = pack_bf16(a, b);
                    hi[h * 2 + g] = w;
                    lo[h * 2 + g] = pack_bf16(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
                }
#pragma unroll
            for (int i = 0; i < NTILES / 2; ++i) {
                uint32_t b[4];
                ldsm_t(base + v_off + (((i * 2 + v_chunk) ^ swz) << 4), b);
                mma(o[2 * i], hi, b[0], b[1]);
                mma(o[2 * i + 1], hi, b[2], b[3]);
                // (infinities are taken in by the first part of their weight, which is positive: the second may be 0 or below)
                mma(o[2 * i], lo, finite_part(b[0]), finite_part(b[1]));
                mma(o[2 * i + 1], lo, finite_part(b[2]), finite_part(b[3]));
            }
            __syncwarp();
            issue();
            stage = stage + 1 == Shape::stages ? 0 : stage + 1;
        }

        AttnStretch s_next = s;
        AttnPart next;
        have = attn_next<ROWS>(p, s_next, next);
        if (have) load_queries(s_next, next);

        // ------------------------------------------------------------ the warps' results joined
        saw |= __shfl_xor_sync(0xffffffffu, saw, 1);
        saw |= __shfl_xor_sync(0xffffffffu, saw, 2);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float x = l[g];
            x += __shfl_xor_sync(0xffffffffu, x, 1);
            x += __shfl_xor_sync(0xffffffffu, x, 2);
            if (pair == 0) ctl.ml[warp][g * 8 + quad] = make_float2(attn_top(m[g] * p.abs_scale_log2, saw >> g & 1), x);
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float top = neg_inf();
#pragma unroll
            for (int w = 0; w < kMmaWarps; ++w) top = fmaxf(top, ctl.ml[w][g * 8 + quad].x);
            const float a = ex2(m[g] * p.abs_scale_log2 - (top == neg_inf() ? 0.f : top));
#pragma unroll
            for (int i = 0; i < NTILES; ++i) {
                o[i][2 * g] *= a;
                o[i][2 * g + 1] *= a;
            }
        }
        const int row = tid >> 3, c4 = (tid & 7) * 4;       // what this thread adds up
        float tall = neg_inf(), sum = 0.f;
#pragma unroll
        for (int w = 0; w < kMmaWarps; ++w) tall = fmaxf(tall, ctl.ml[w][row].x);
#pragma unroll
        for (int w = 0; w < kMmaWarps; ++w) {
            const float2 x = ctl.ml[w][row];
            sum = fmaf(ex2(x.x - (tall == neg_inf() ? 0.f : tall)), x.y, sum);
        }
        const int r = row;
        const float inv = attn_inverse(tall, sum);
        const int64_t out_at = first_row(s, part) + join_at;
#pragma unroll
        for (int h = 0; h < 2 * PANELS; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    *reinterpret_cast<float2 *>(join + (warp * 16 + g * 8 + quad) * kJoinPitch + i * 8 + pair * 2) =
                        make_float2(o[h * 4 + i][2 * g], o[h * 4 + i][2 * g + 1]);
            __syncthreads();
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kMmaWarps; ++w) {
                const float4 x = *reinterpret_cast<const float4 *>(join + (w * 16 + row) * kJoinPitch + c4);
                y.x += x.x, y.y += x.y, y.z += x.z, y.w += x.w;
            }
            const int c = h * kJoinCols + c4;
            if (r < t.rows && c < p.D) {
                if (t.whole) {
                    store_out(static_cast<__nv_bfloat16 *>(p.out) + out_at + c, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv), 4);
                } else {
                    __stcg(reinterpret_cast<float4 *>(p.part + ((int64_t)t.slot * ROWS + r) * p.D + c), y);
                    if (c == 0) __stcg(&p.part_ml[(int64_t)t.slot * ROWS + r], make_float2(tall, sum));
                }
            }
            __syncthreads();
        }
        if (!t.whole) {
            __syncthreads();
            if (tid == 0) ctl.last = attn_ticket(p, t);
            __syncthreads();
            if (ctl.last) attn_join<ROWS, __nv_bfloat16>(p, s, part, t, warp, kMmaWarps);
        }
        s = s_next;
        part = next;
    }
    copies_wait<0>();
}

template <int PANELS, bool WHOLE>
cudaError_t launch_mma(const AttnParams &p, int dev, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];   // host threads may race to set it: all of them store `true`
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_mma_kernel<PANELS, WHOLE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)MmaShape<PANELS>::smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    attention_mma_kernel<PANELS, WHOLE><<<p.ctas, kMmaThreads, MmaShape<PANELS>::smem, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_mma(const AttnParams &p, int dev, cudaStream_t st)
{
    if (p.D == 128) return launch_mma<2, true>(p, dev, st);
    if (p.D == 64) return launch_mma<1, true>(p, dev, st);
    return p.D < 64 ? launch_mma<1, false>(p, dev, st) : launch_mma<2, false>(p, dev, st);
}

}  // namespace spr
