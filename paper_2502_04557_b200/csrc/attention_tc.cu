// tree_attention on bf16 tensors, many rows per cached head (long chains, trees): tcgen05.
//
//   S = Q K^T   128 rows by a tile of 64 keys, into TMEM;   P = exp2(c (S - m)), back into TMEM;   O += P V, in TMEM
//
// One CTA per SM walks its stretch of tiles; tiles go to two groups by turns.  Four softmax warps of a group have a row
// per thread, and one warp issues the group's products: S of the next tile goes ahead of P V of this one (S is
// double-buffered, P takes the place of the S it comes from).  The groups have maxima, sums and an O of their own and wait for
// nothing of one another until the end of a part: a tile takes a softmax warp some 2000 clocks, most of it latency.
// All 512 columns of TMEM are in use: 2 x 2 S, 2 O.
//
// One loader warp brings keys, one values and queries, into a ring of six tiles (cp.async, 16 bytes per lane, into the
// 128-byte swizzle that the matrix descriptors name: pages of 16 entries would be 2 KB boxes for the copy engine, whose
// number sets its time; a warp takes some 800 clocks per 16 KB).  Copies report to the barriers themselves.
// Loaders run ahead into the next part while this one ends.  Every warp that waits on a barrier sees all of its phases.
//
// Exponents are taken against a maximum that stands until a tile's weights add up to more than 2^13 (sums and products in
// fp32 keep their relative precision whatever the common factor): only then are its scores looked through for
// a new one and O, which lives in TMEM, rescaled.  Most tiles need no maximum at all.
// Weights are rounded to bf16 for the second product, each by up to 2^-8 of itself, and a result is off by up to as much of
// sum p |v|: more than its own rounding where values cancel.  (Values that are independent of one another: 0.0023 of the results, root
// mean square, where their own rounding is 0.0017.)  A second bf16 number for what the rounding leaves, as with few rows, would
// cost a fifth of the time (199 us against 164 us when both were measured, at an earlier state of the loaders).
//
// 128 sequences of 17 nodes, 32/8 heads of 128, some 1500 tokens: 175 us, 130 of loads; 16 trees of 64 nodes over 8192: 160 us.  Beside its
// tiles a part takes some 9000 clocks, the latency of its start, its tail (which is masked and looked through) and its results: 128
// sequences of 17 nodes over 100 tokens take 54 us, 13 of loads.
//
// Every wait is bounded: when one runs out the status word becomes SPR_ERR_TIMEOUT, loaders and issuing threads stop and
// wait (again bounded) for what is in flight, and the softmax warps go on without waiting and give NaN.
#include <atomic>

#include "attention_plan.cuh"
#include "host_util.h"
#include "launch.h"
#include "tensor_pair.cuh"
#include "vocab_common.cuh"

namespace spr {

namespace {

using namespace pairtc;

constexpr int kTcThreads = 384;
constexpr int kGroupThreads = 128, kSoftmaxThreads = 2 * kGroupThreads;
constexpr int kMmaWarp = 8, kFirstLoader = 10;                  // (keys, values)
constexpr int kTcRows = 128;
constexpr int kPanel = kAttnTile * 128;                         // 64 keys by 64 columns
constexpr float kMostWeight = 8192.f;                           // of a row in a tile, before its maximum is raised
// TMEM columns: two buffers of S for each group, 64 each, of which P takes 32; each group's O
constexpr int kColS = 0, kColO = 256, kTmemCols = 512;

template <int PANELS>
struct TcShape {
    static constexpr int unit = PANELS * kPanel;                 // a tile's keys, or its values
    static constexpr int units = 12;                             // of the ring: keys and values by turns.  A multiple of four:
                                                                 // a unit's place then always is the same group's
    static constexpr int q_bytes = PANELS * 128 * 128;
    static constexpr size_t smem = (size_t)q_bytes + (size_t)units * unit;
};

struct TcControl {
    uint64_t full[12], empty[12];
    uint64_t s_full[2][2], p_ready[2][2], pv_done[2][2];         // [group][buffer]
    uint64_t q_full, q_empty, drain[2];
    uint64_t valid[12];                      // a bit for each key of a tile that is there, of two rounds of the ring: keys leave it
                                             // before the softmax warps have seen to their scores
    unsigned long long odd[2];
    int o_live[2];
    uint32_t tmem;
    int abort, last;
    int16_t tree[kMaxTreeNodes];             // parents, checked
    union {
        int scratch[kTcThreads / 32 + 2];
        float2 ml[2][kGroupThreads];
    };
};
static_assert(TcShape<2>::smem + sizeof(TcControl) <= 232448, "shared memory of one CTA");

__device__ __forceinline__ void softmax_meet() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void group_meet(int group)
{
    if (group)
        asm volatile("bar.sync 3, 128;" ::: "memory");
    else
        asm volatile("bar.sync 2, 128;" ::: "memory");
}
// the same, and whether any thread has something
__device__ __forceinline__ bool group_any(int group, bool x)
{
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\tbarrier.cta.red.or.pred q, %1, 128, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(any)
                 : "r"(group ? 3 : 2), "r"((int)x)
                 : "memory");
    return any != 0;
}
__device__ __forceinline__ void arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there)      // or zeros
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
// this lane arrives when its copies so far have come
__device__ __forceinline__ void copies_arrive(uint64_t *bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tmem_write32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ bool finite_bf16x2(uint32_t w) { return (w & 0x7f80u) != 0x7f80u && (w & 0x7f800000u) != 0x7f800000u; }
// Four lanes' four vectors each, the other way round: lane j of them has vector j of all.  Rows lie one to a lane, and stores of 16
// bytes in 32 rows take the memory system 32 requests, however near they lie.
__device__ __forceinline__ void exchange4(uint4 (&x)[4], int lane)
{
#pragma unroll
    for (int by = 1; by <= 2; by *= 2) {
        const bool upper = lane & by;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = by == 1 ? 2 * k : k, j = i + by;
            uint4 give = upper ? x[i] : x[j];
            give.x = __shfl_xor_sync(0xffffffffu, give.x, by);
            give.y = __shfl_xor_sync(0xffffffffu, give.y, by);
            give.z = __shfl_xor_sync(0xffffffffu, give.z, by);
            give.w = __shfl_xor_sync(0xffffffffu, give.w, by);
            (upper ? x[i] : x[j]) = give;
        }
    }
}
// which of the nodes first .. first + 63 node i sees: itself and its path
__device__ __forceinline__ uint64_t seen_nodes(const int16_t *tree, int i, int first)
{
    if (!tree) {
        const int n = i + 1 - first;
        return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
    }
    uint64_t bits = 0;
    for (; i >= first && i >= 0; i = tree[i])        // (parents come first)
        if (i - first < 64) bits |= 1ull << (i - first);
    return bits;
}

// WHOLE: heads are whole panels, so that the distances between rows are known
template <int PANELS, bool WHOLE>
__global__ void __launch_bounds__(kTcThreads, 1) attention_tc_kernel(const AttnParams p)
{
    constexpr int ROWS = kTcRows, COLS = 64 * PANELS;
    using Shape = TcShape<PANELS>;
    extern __shared__ __align__(1024) uint8_t raw[];
    __shared__ TcControl ctl;
    const uint32_t q_tile = smem_addr(raw), ring = q_tile + Shape::q_bytes;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t limit = p.spin_limit;

    if (tid == 0) {
        for (int i = 0; i < Shape::units; ++i) {
            bar_init(&ctl.full[i], 32);          // each lane of the warp that brings it
            bar_init(&ctl.empty[i], 1);
        }
        for (int i = 0; i < 4; ++i) {
            bar_init(&ctl.s_full[i >> 1][i & 1], 1);
            bar_init(&ctl.p_ready[i >> 1][i & 1], 4);
            bar_init(&ctl.pv_done[i >> 1][i & 1], 1);
        }
        bar_init(&ctl.q_full, 32);
        bar_init(&ctl.q_empty, 2);
        for (int i = 0; i < 2; ++i) {
            bar_init(&ctl.drain[i], 1);
            ctl.odd[i] = 0;
            ctl.o_live[i] = -1;
        }
        ctl.abort = 0;
        if (q_tile & 1023u) {                    // the swizzle goes by address (the array's alignment sees to it)
            ctl.abort = 1;
            raise_timeout(p.status);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)), "r"((uint32_t)kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    AttnStretch s = attn_plan<ROWS, kTcThreads, 6>(p, ctl.scratch);
    attn_clear_unused<__nv_bfloat16>(p, kTcThreads);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = ctl.tmem;
    // lane's 16 bytes of a row of keys, values or queries
    constexpr int kChunks = 8 * PANELS, kRowsAtOnce = 32 / kChunks;
    const int c_row = lane / kChunks, c_chunk = lane % kChunks;
    const bool c_in = c_chunk * 8 < p.D;

    // a wait that is most often over
    auto quick_wait = [&](uint64_t *bar, uint32_t parity) {
        return bar_poll(bar, parity & 1) || bar_wait(bar, parity & 1, &ctl.abort, p.status, limit);
    };
    if (warp >= kFirstLoader) {
        // ------------------------------------------------------------ keys; values and queries
        const int kv = warp - kFirstLoader;
        // rows 8 r + r0 + c_row of a unit lie at (c_dst + 128 (8 r + r0)) ^ (r0 << 4): r0 is a multiple of kRowsAtOnce
        const uint32_t c_dst = (c_chunk >> 3) * kPanel + c_row * 128 + (((c_chunk & 7) ^ c_row) << 4);
        const int D = WHOLE ? COLS : p.D;
        AttnPart part = {0, 0, 0, 0};
        int unit = kv;                              // place in the ring
        uint32_t round = 0, parts = 0;
        bool alive = !(p.test_flags & ATTN_TEST_NO_LOADS);
        while (alive && attn_next<ROWS>(p, s, part)) {
            if (kv) {
                // the part's queries (rows behind the block's last are whatever was there: nobody looks at what becomes of them)
                if (parts > 0 && !__all_sync(0xffffffffu, quick_wait(&ctl.q_empty, parts - 1))) break;
                ++parts;
                const int row0 = part.block * ROWS, rows = min(ROWS, s.seq.count * p.G - row0);
                const int i0 = row0 / p.G, g0 = row0 - i0 * p.G;
                const float per_node = 1.f / (float)p.G;
                const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.q) +
                                         (((int64_t)s.seq.b * p.nodes.T + i0) * p.Hq + part.head * p.G + g0) * D + c_chunk * 8;
                const int hop = (p.Hq - p.G) * D;           // from a node's last row to the next one's first, in elements
                const uint32_t dst = q_tile + (c_chunk >> 3) * ROWS * 128 + c_row * 128 + (((c_chunk & 7) ^ c_row) << 4);
#pragma unroll 4
                for (int r0 = 0; r0 < rows; r0 += kRowsAtOnce) {
                    const int r = r0 + c_row;
                    const int i = (int)(((float)(g0 + r) + 0.5f) * per_node);       // (g0 + r) / G: both are small
                    const bool there = c_in && r < rows;
                    copy16((dst ^ ((r0 & 7) << 4)) + r0 * 128, q + (there ? r * D + (int64_t)i * hop : 0), there);
                }
                copies_arrive(&ctl.q_full);
            }
            const int keys = attn_keys(p, s.seq.len, s.seq.count);
            if (keys < (int64_t)s.seq.len + s.seq.count) raise_status(p.status, SPR_ERR_BAD_PAGE);
            const int end = part.t0 + part.n;
            auto find = [&](int tile) {             // lane 8 j + r: where run r (8 keys) of tile + j begins in the caches
                const int t = tile + (lane >> 3);
                const int slot = t * kAttnTile + 8 * (lane & 7);
                if (t >= end || slot >= keys) return -1;
                const int at = slot / p.page_size;
                const int page = __ldg(p.page_table + (int64_t)s.seq.b * p.max_pages + at);
                if (page < 0 || page >= p.num_pages) {
                    raise_status(p.status, SPR_ERR_BAD_PAGE);
                    return -1;
                }
                return (page * p.Hkv + part.head) * p.page_size + (slot - at * p.page_size);
            };
            int tile = part.t0, next = find(tile);
            while (alive && tile < end) {
                const int rows = next;
                next = find(tile + 4);
                for (int u = 0; alive && u < 4 && tile < end; ++u, ++tile) {
                    const int left = keys - tile * kAttnTile;
                    uint64_t valid = left >= 64 ? ~0ull : (1ull << left) - 1;
                    const uint32_t runs = __ballot_sync(0xffffffffu, rows >= 0) >> (8 * u) & 0xffu;
                    if (runs != 0xffu)
                        for (int r = 0; r < 8; ++r)
                            if (!(runs >> r & 1)) valid &= ~(0xffull << (8 * r));
                    if (round > 0 && !__all_sync(0xffffffffu, quick_wait(&ctl.empty[unit], round - 1))) {
                        alive = false;
                        break;
                    }
                    if (kv == 0 && lane == 0) {
                        ctl.valid[(unit >> 1) + (round & 1) * (Shape::units / 2)] = valid;
                        __threadfence_block();
                    }
                    const __nv_bfloat16 *cache = static_cast<const __nv_bfloat16 *>(kv ? p.v : p.k) + c_row * D + c_chunk * 8;
                    const uint32_t dst = ring + unit * Shape::unit + c_dst;
                    if (WHOLE && valid == ~0ull) {
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            const __nv_bfloat16 *from = cache + (int64_t)__shfl_sync(0xffffffffu, rows, 8 * u + r) * COLS;
#pragma unroll
                            for (int r0 = 0; r0 < 8; r0 += kRowsAtOnce) copy16((dst ^ (r0 << 4)) + (8 * r + r0) * 128, from + r0 * COLS);
                        }
                    } else {
#pragma unroll 1
                        for (int r = 0; r < 8; ++r) {
                            const int run = __shfl_sync(0xffffffffu, rows, 8 * u + r);
                            for (int r0 = 0; r0 < 8; r0 += kRowsAtOnce) {
                                const bool there = c_in && (valid >> (8 * r + r0 + c_row) & 1);
                                copy16((dst ^ (r0 << 4)) + (8 * r + r0) * 128, there ? cache + ((int64_t)run + r0) * D : p.k, there);
                            }
                        }
                    }
                    copies_arrive(&ctl.full[unit]);
                    unit += 2;
                    if (unit >= Shape::units) {
                        unit -= Shape::units;
                        ++round;
                    }
                }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");       // none is left when the CTA ends
    } else if (warp >= kMmaWarp) {
        if (lane == 0) {
            // -------------------------------------------------------- products of a group
            const int group = warp - kMmaWarp;
            constexpr uint32_t kQk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kAttnTile >> 3) << 17) | (8u << 24);
            constexpr uint32_t kPv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(COLS >> 3) << 17) | (8u << 24);
            const uint32_t col_s = tmem + kColS + 128 * group, col_o = tmem + kColO + 128 * group;
            AttnPart part;
            int at = 0;                     // tiles of the stretch before the part
            uint32_t parts = 0;
            int v_unit = 2 * group + 1;     // place of the values of this group's next tile
            uint32_t v_round = 0;
            bool alive = true;
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                if (alive && !quick_wait(bar, parity)) alive = false;
                return alive;
            };
            // where S of tile i goes P of tile i - 4, this group's last but one, was: the product with it has to be complete
            int k_unit = 2 * group;             // place of the keys of this group's next tile
            uint32_t k_round = 0;
            auto scores = [&](int i) {
                const int unit = k_unit, b = i >> 1 & 1;
                if (!wait(&ctl.full[unit], k_round) || (i >= 4 && !wait(&ctl.pv_done[group][b], (uint32_t)(i >> 2) - 1))) return;
                k_unit += 4;
                if (k_unit >= Shape::units) {
                    k_unit -= Shape::units;
                    ++k_round;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // the lanes' copies, for the tensor core
                fence_after();
                const uint32_t k = ring + unit * Shape::unit;
#pragma unroll
                for (int q = 0; q < 4 * PANELS; ++q)
                    mma_smem(col_s + 64 * b, tile_desc(q_tile + (q >> 2) * ROWS * 128 + (q & 3) * 32, false),
                             tile_desc(k + (q >> 2) * kPanel + (q & 3) * 32, false), kQk, q != 0);
                commit(&ctl.s_full[group][b]);
                commit(&ctl.empty[unit]);
            };
            while (alive && attn_next<ROWS>(p, s, part)) {
                const int end = at + part.n;
                int mine = at + ((at ^ group) & 1);
                at = end;
                if (!wait(&ctl.q_full, parts++)) break;
                if (mine < end) scores(mine);
                if (mine + 2 < end) scores(mine + 2);
                if (mine + 4 >= end) {          // no more scores of this part from this group
                    if (mine < end)
                        commit(&ctl.q_empty);
                    else
                        arrive(&ctl.q_empty);
                }
                for (bool begun = false; alive && mine < end; mine += 2, begun = true) {
                    const int unit = v_unit, b = mine >> 1 & 1;
                    const uint32_t phase = (uint32_t)(mine >> 2);
                    if (!wait(&ctl.full[unit], v_round) || !wait(&ctl.p_ready[group][b], phase)) break;
                    v_unit += 4;
                    if (v_unit >= Shape::units) {
                        v_unit -= Shape::units;
                        ++v_round;
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    fence_after();
                    const uint32_t v = ring + unit * Shape::unit, w = col_s + 64 * b;
                    const bool live = begun || *reinterpret_cast<volatile int *>(&ctl.o_live[group]) == mine;
#pragma unroll
                    for (int q = 0; q < 4; ++q) mma_tmem(col_o, w + 8 * q, tile_desc(v + q * 2048, true), kPv, live || q != 0);
                    commit(&ctl.pv_done[group][b]);
                    commit(&ctl.empty[unit]);
                    if (mine + 4 < end) {
                        scores(mine + 4);
                        if (mine + 6 >= end) commit(&ctl.q_empty);
                    }
                }
            }
            commit(&ctl.drain[group]);      // nothing of this thread's products is left when TMEM is given back
            bar_wait_quiet(&ctl.drain[group], 0, limit);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ softmax: a row per thread
        const int group = warp >> 2, row = tid & (kGroupThreads - 1);
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t col_o = lanes + kColO + 128 * group;
        const float c = p.abs_scale_log2;
        AttnPart part;
        int at = 0;
        int tree_of = -1;
        bool dead = false;
        auto wait = [&](uint64_t *bar, uint32_t parity) {
            if (!dead) dead = !quick_wait(bar, parity);
        };
        auto warp_arrive = [&](uint64_t *bar) {
            __syncwarp();
            if (lane == 0) arrive(bar);
        };
        while (attn_next<ROWS>(p, s, part)) {
            const AttnTarget t = attn_target<ROWS>(p, s, part);
            const bool in = row < t.rows, warp_in = (warp & 3) * 32 < t.rows;
            const int node = in ? (t.row0 + row) / p.G : 0;
            softmax_meet();                                 // (both groups have read both O, and the tree)
            if (p.nodes.parents && tree_of != s.seq.b && (part.t0 + part.n) * kAttnTile > s.seq.len) {
                for (int j = tid; j < s.seq.count; j += kSoftmaxThreads)
                    ctl.tree[j] = (int16_t)checked_parent(p.nodes.parents[(int64_t)s.seq.b * p.nodes.T + j], j, p.status);
                tree_of = s.seq.b;
                softmax_meet();
            }
            float m = neg_inf(), l = 0.f;
            bool saw = false;                               // a key of this group's tiles
            int mine = at + ((at ^ group) & 1);             // this group's next tile
            const int begin = at, end = at + part.n;
            at = end;
            const bool any = mine < end;
            int slot0 = (part.t0 + (mine - begin)) * kAttnTile;
            int place = mine % Shape::units;         // of the tile in two rounds of the ring
            for (bool begun = false; mine < end; mine += 2, begun = true, slot0 += 2 * kAttnTile, place = place < Shape::units - 2 ? place + 2 : place + 2 - Shape::units) {
                const int b = mine >> 1 & 1;
                const uint32_t phase = (uint32_t)(mine >> 2), col_s = lanes + kColS + 128 * group + 64 * b;
                wait(&ctl.s_full[group][b], phase);
                const bool tail = slot0 + kAttnTile > s.seq.len;      // (alike in all threads, whatever went wrong: they meet)
                unsigned long long odd = 0;
                uint64_t vis = ctl.valid[place];
                if (tail) {
                    const int d = s.seq.len - slot0;         // keys of the prefix
                    const int16_t *tree = p.nodes.parents ? ctl.tree : nullptr;
                    vis &= d <= 0 ? seen_nodes(tree, node, -d) : seen_nodes(tree, node, 0) << d | ((1ull << d) - 1);
                    // values that are not finite, where not every row sees every key: each thread looks at half a key
                    wait(&ctl.full[(2 * place + 1) % Shape::units], (uint32_t)(mine / (Shape::units / 2)));
                    const uint32_t v = ring + (2 * place + 1) % Shape::units * Shape::unit + (row >> 1) * 128 + (row & 1) * 64;
                    bool bad = false;
#pragma unroll
                    for (int k = 0; k < 4 * PANELS; ++k) {
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(v + (k >> 2) * kPanel + ((k ^ (row >> 1)) & 3) * 16) : "memory");      // (banks)
                        bad = bad || !(finite_bf16x2(w[0]) && finite_bf16x2(w[1]) && finite_bf16x2(w[2]) && finite_bf16x2(w[3]));
                    }
                    if (group_any(group, bad)) {
                        if (bad) atomicOr(&ctl.odd[group], 1ull << (row >> 1));
                        group_meet(group);
                        odd = *reinterpret_cast<volatile unsigned long long *>(&ctl.odd[group]);
                    }
                }
                saw = saw || vis != 0;
                if (!warp_in && !odd) {                      // no row of this warp is in use: its part of P is not looked at
                    warp_arrive(&ctl.p_ready[group][b]);
                    continue;
                }
                fence_after();
                float x[64], sum;
#pragma unroll 1
                for (bool looked = !begun;; looked = true) {
                    tmem_read32(col_s, *reinterpret_cast<float (*)[32]>(x));
                    tmem_read32(col_s + 32, *reinterpret_cast<float (*)[32]>(x + 32));
                    tmem_wait();
                    if (p.flip) {
#pragma unroll
                        for (int i = 0; i < 64; ++i) x[i] = -x[i];
                    }
                    if (vis != ~0ull) {
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            if (!((i < 32 ? (uint32_t)vis : (uint32_t)(vis >> 32)) >> (i & 31) & 1)) x[i] = neg_inf();
                    }
                    if (looked) {
                        float t4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                        for (int i = 4; i < 64; i += 2) t4[(i >> 1) & 3] = fmaxf(fmaxf(t4[(i >> 1) & 3], x[i]), x[i + 1]);
                        const float top = fmaxf(fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])), m);
                        // (m = -inf: nothing seen so far, and O holds nothing of this row)
                        const float a = m != neg_inf() && top > m ? ex2((m - top) * c) : 1.f;
                        m = top;
                        l *= a;
                        if (begun) {
                            wait(&ctl.pv_done[group][b ^ 1], (uint32_t)((mine - 2) >> 2));
                            fence_after();
#pragma unroll 1
                            for (int k = 0; k < 2 * PANELS; ++k) {
                                float o[32];
                                uint32_t w[32];
                                tmem_read32(col_o + 32 * k, o);
                                tmem_wait();
#pragma unroll
                                for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(o[i] * a);
                                tmem_write32(col_o + 32 * k, w);
                            }
                            tmem_wait_st();        // (O may be read again below, and stores are not in order with reads)
                        }
                    }
                    const float ref = m == neg_inf() ? 0.f : -m * c;
                    const uint64_t c2 = pack2(c, c), ref2 = pack2(ref, ref);
                    uint64_t s2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        unpack2(fma2(pack2(x[2 * i], x[2 * i + 1]), c2, ref2), x[2 * i], x[2 * i + 1]);
                        x[2 * i] = ex2(x[2 * i]);
                        x[2 * i + 1] = ex2(x[2 * i + 1]);
                        s2[i & 1] = add2(s2[i & 1], pack2(x[2 * i], x[2 * i + 1]));
                    }
                    float sum1;
                    unpack2(add2(s2[0], s2[1]), sum, sum1);
                    sum += sum1;
                    if (looked || !__any_sync(0xffffffffu, in && (m == neg_inf() || !(sum <= kMostWeight)))) break;
                }
                l += sum;
                if (odd) {
                    // taken out of the product, and added one by one to the rows that see them
                    if (begun) wait(&ctl.pv_done[group][b ^ 1], (uint32_t)((mine - 2) >> 2));
                    const uint32_t v_unit = ring + (2 * place + 1) % Shape::units * Shape::unit;
                    fence_after();
#pragma unroll 1
                    for (int k = 0; k < 2 * PANELS; ++k) {
                        float o[32];
                        uint32_t w[32];
                        tmem_read32(col_o + 32 * k, o);
                        tmem_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!begun) o[i] = 0.f;
                        for (unsigned long long rest = odd & vis; rest; rest &= rest - 1) {
                            const int key = __ffsll((long long)rest) - 1;
                            float weight = 0.f;
#pragma unroll
                            for (int i = 0; i < 64; ++i) weight = i == key ? x[i] : weight;
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                uint32_t y;
                                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(y)
                                             : "r"(v_unit + (k >> 1) * kPanel + key * 128 + ((((k & 1) * 4 + (i >> 2)) ^ (key & 7)) << 4) + (i & 3) * 4) : "memory");
                                o[2 * i] = fmaf(weight, __uint_as_float(y << 16), o[2 * i]);
                                o[2 * i + 1] = fmaf(weight, __uint_as_float(y & 0xffff0000u), o[2 * i + 1]);
                            }
                        }
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(o[i]);
                        tmem_write32(col_o + 32 * k, w);
                    }
                    group_meet(group);
                    if (odd >> (row >> 1) & 1)
                        for (int k = 0; k < 4 * PANELS; ++k)
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v_unit + (row >> 1) * 128 + (row & 1) * 64 + (k >> 2) * kPanel + (k & 3) * 16), "r"(0u) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    if (row == 0) {
                        ctl.odd[group] = 0;
                        if (!begun) ctl.o_live[group] = mine;
                    }
                    group_meet(group);
                }
                uint32_t w[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
                tmem_write32(col_s, w);
                tmem_wait_st();
                fence_before();
                warp_arrive(&ctl.p_ready[group][b]);
            }

            // -------------------------------------------------------- the part's results: each group has half of the columns
            if (any) wait(&ctl.pv_done[group][(mine - 2) >> 1 & 1], (uint32_t)((mine - 2) >> 2));
            if (dead) l = __int_as_float(0x7fc00000);       // what a wait that ran out leaves is no result
            m = attn_top(m, saw);
            ctl.ml[group][row] = make_float2(m, l);
            softmax_meet();
            fence_after();
            const float2 other = ctl.ml[group ^ 1][row];
            const float top = fmaxf(m, other.x), shift = top == neg_inf() ? 0.f : top;
            float by[2] = {ex2((m - shift) * c), ex2((other.x - shift) * c)};
            l = l * by[0] + other.y * by[1];
            const bool all = part.n > 1;                    // else the other group's O is not of this part, or this group's
            const float inv = attn_inverse(top, l);
            if (warp_in) {
                // the rows that this lane writes vectors of, and where they begin
                const int64_t out_at = in ? attn_out_at(p, s, part, t.row0 + row) : 0;
                const int first = row & ~3;
                int64_t to[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) to[i] = __shfl_sync(0xffffffffu, out_at, (lane & ~3) + i);
#pragma unroll 1
                for (int k = group * PANELS; k < (group + 1) * PANELS; ++k) {
                    float o[32], y[32];
                    tmem_read32(lanes + kColO + 128 * (any ? group : group ^ 1) + 32 * k, o);
                    tmem_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] *= any ? by[0] : by[1];
                    if (all) {
                        tmem_read32(lanes + kColO + 128 * (group ^ 1) + 32 * k, y);
                        tmem_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = fmaf(y[i], by[1], o[i]);
                    }
                    uint4 v[4];
                    if (t.whole) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[i] = make_uint4(pack_bf16(o[8 * i] * inv, o[8 * i + 1] * inv), pack_bf16(o[8 * i + 2] * inv, o[8 * i + 3] * inv),
                                              pack_bf16(o[8 * i + 4] * inv, o[8 * i + 5] * inv), pack_bf16(o[8 * i + 6] * inv, o[8 * i + 7] * inv));
                        exchange4(v, lane);
                        const int col = 32 * k + 8 * (lane & 3);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (first + i < t.rows && col < p.D) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) + to[i] + col) = v[i];
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                v[i] = make_uint4(__float_as_uint(o[16 * h + 4 * i]), __float_as_uint(o[16 * h + 4 * i + 1]),
                                                  __float_as_uint(o[16 * h + 4 * i + 2]), __float_as_uint(o[16 * h + 4 * i + 3]));
                            exchange4(v, lane);
                            const int col = 32 * k + 16 * h + 4 * (lane & 3);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (first + i < t.rows && col < p.D)
                                    __stcg(reinterpret_cast<uint4 *>(p.part + ((int64_t)t.slot * ROWS + first + i) * p.D + col), v[i]);
                        }
                    }
                }
            }
            if (!t.whole && group == 0 && in) __stcg(&p.part_ml[(int64_t)t.slot * ROWS + row], make_float2(attn_top(top * c, top != neg_inf()), l));
            fence_before();
            if (!t.whole) {
                softmax_meet();
                if (tid == 0) ctl.last = attn_ticket(p, t);
                softmax_meet();
                if (ctl.last) attn_join<ROWS, __nv_bfloat16>(p, s, part, t, warp, kSoftmaxThreads / 32);
            }
        }
    }
    fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kTmemCols) : "memory");
    }
}

template <int PANELS, bool WHOLE>
cudaError_t launch_tc(const AttnParams &p, int dev, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];   // host threads may race to set it: all of them store `true`
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_tc_kernel<PANELS, WHOLE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)TcShape<PANELS>::smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    attention_tc_kernel<PANELS, WHOLE><<<p.ctas, kTcThreads, TcShape<PANELS>::smem, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_tc(const AttnParams &p, int dev, cudaStream_t st)
{
    if (p.D == 128) return launch_tc<2, true>(p, dev, st);
    if (p.D == 64) return launch_tc<1, true>(p, dev, st);
    return p.D < 64 ? launch_tc<1, false>(p, dev, st) : launch_tc<2, false>(p, dev, st);
}

}  // namespace spr
