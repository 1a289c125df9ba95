// tree_attention on bf16 tensors, many rows per cached head (long chains, trees): tcgen05.
//
//   S = Q K^T   128 rows by a tile of 64 keys, into TMEM;   P = exp2(c (S - m)), back into TMEM;   O += P V, in TMEM
//
// Two CTAs per SM walk a stretch of tiles each, so that one's waits, beginnings and ends of parts hide behind the other's
// work.  One loader warp brings keys and one values into a ring of units (cp.async, 16 bytes per lane, into the 128-byte
// swizzle that the matrix descriptors name; a warp takes 1500 clocks to ask for 16 KB, so that one would not do for both,
// and pages of 16 entries would be 2 KB boxes for the copy engine, whose number sets its time).  Copies report to the ring's
// barriers themselves.  One thread issues the products: S of the next tile goes ahead of P V of this one.  Four softmax
// warps have a row per thread, and the registers that the others do without.  S is double-buffered, and P takes the place
// of the S it comes from.  The maximum that exponents are taken against is only raised when a score passes it by 2^8
// (weights then stay below 2^8, and sums and products in fp32 keep their relative precision), so that O, which lives in
// TMEM, is hardly ever rescaled.
//
// Weights are used as two bf16 numbers, their rounding and what is left of it: one would put an error of 2^-9 on the
// result, as much as its own rounding.  Up to 64 rows (DUP) the tile's other half holds the same queries again and
// takes the second number, so that the one product does both; above, there is a second product.
//
// Every wait is bounded: when one runs out the status word becomes SPR_ERR_TIMEOUT, loader and issuing thread stop and
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

constexpr int kTcThreads = 256;
constexpr int kSoftmaxThreads = 128;
constexpr int kMmaWarp = 4, kFirstLoader = 5;    // one for keys, one for values (warp 7 idles)
constexpr int kPanel = kAttnTile * 128;                         // 64 keys by 64 columns
constexpr float kRaise = 8.f;                                   // by how much scores may pass the maximum in use
// TMEM columns: two buffers of S, 64 each, where P's two numbers take 32 and 32; O
constexpr int kColS = 0, kColO = 128, kTmemCols = 256;

template <int PANELS>
struct TcShape {
    static constexpr int unit = PANELS * kPanel;                 // a tile's keys, or its values
    static constexpr int units = 8 / PANELS;                     // of the ring: keys and values by turns
    static constexpr int q_bytes = PANELS * 128 * 128;
    static constexpr size_t smem = (size_t)q_bytes + (size_t)units * unit + 1024;
};

struct TcControl {
    uint64_t full[8], empty[8];
    uint64_t s_full[2], p_ready[2], pv_done[2];   // by turns: a softmax warp may be a tile ahead of another, and of P V
    uint64_t q_ready, drain;
    uint64_t valid[8];                       // a bit for each key of a tile that is there
    int64_t scratch[2 * (kTcThreads / 32) + 4];
    unsigned long long odd;
    int64_t o_live;
    uint32_t tmem;
    int abort, last;
    int tree[kMaxTreeNodes];
    uint32_t path[128][kMaxTreeNodes / 32];
};

__device__ __forceinline__ void softmax_meet() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
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
// 64 bits of a path from node `at` on
__device__ __forceinline__ uint64_t path_bits64(const uint32_t *path, int at)
{
    constexpr int n = kMaxTreeNodes / 32;
    const int w = at >> 5;
    const uint32_t a = w < n ? path[w] : 0u, b = w + 1 < n ? path[w + 1] : 0u, c = w + 2 < n ? path[w + 2] : 0u;
    return (uint64_t)__funnelshift_r(a, b, at & 31) | (uint64_t)__funnelshift_r(b, c, at & 31) << 32;
}

template <int PANELS, bool DUP>
__global__ void __launch_bounds__(kTcThreads, 2) attention_tc_kernel(const AttnParams p)
{
    constexpr int ROWS = DUP ? 64 : 128, COLS = 64 * PANELS;
    using Shape = TcShape<PANELS>;
    extern __shared__ uint8_t raw[];
    __shared__ TcControl ctl;
    const uint32_t q_tile = (smem_addr(raw) + 1023u) & ~1023u, ring = q_tile + Shape::q_bytes;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t limit = p.spin_limit;

    if (tid == 0) {
        for (int i = 0; i < Shape::units; ++i) {
            bar_init(&ctl.full[i], 32);          // each lane of the warp that brings it
            bar_init(&ctl.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&ctl.s_full[i], 1);
            bar_init(&ctl.p_ready[i], 4);
            bar_init(&ctl.pv_done[i], 1);
        }
        bar_init(&ctl.q_ready, 4);
        bar_init(&ctl.drain, 1);
        ctl.abort = 0;
        ctl.odd = 0;
        ctl.o_live = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)), "r"((uint32_t)kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    AttnStretch s = attn_plan<ROWS, kTcThreads>(p, ctl.scratch);
    attn_clear_unused<__nv_bfloat16>(p, kTcThreads);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = ctl.tmem;

    // (256 threads start with 128 registers each: 168 and 88 make the same sum)
    if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
      if (warp >= kFirstLoader) {
        // ------------------------------------------------------------ loaders (the ring holds an even number of units: each
        // has stages of its own, and sees every phase of their barriers)
        constexpr int kChunks = 8 * PANELS, kRowsAtOnce = 32 / kChunks;
        const int c_row = lane / kChunks, c_chunk = lane % kChunks;
        const bool c_in = c_chunk * 8 < p.D;
        // rows 8 r + r0 + c_row of a unit lie at (c_dst + 128 (8 r + r0)) ^ (r0 << 4): r0 is a multiple of kRowsAtOnce
        const uint32_t c_dst = (c_chunk >> 3) * kPanel + c_row * 128 + (((c_chunk & 7) ^ c_row) << 4);
        AttnPart part = {0, 0, 0, 0};
        const int kv = warp - kFirstLoader;
        int64_t unit = kv;
        bool alive = !(p.test_flags & ATTN_TEST_NO_LOADS);
        while (kv < 2 && alive && attn_next<ROWS>(p, s, part)) {
            int64_t keys = (int64_t)s.seq.len + s.seq.count;
            if (keys > (int64_t)p.max_pages * p.page_size) {
                raise_status(p.status, SPR_ERR_BAD_PAGE);
                keys = (int64_t)p.max_pages * p.page_size;
            }
            const int end = part.t0 + part.n;
            auto find = [&](int tile) {             // lane 8 j + r: where run r (8 keys) of tile + j begins in the caches
                const int t = tile + (lane >> 3);
                const int64_t slot = (int64_t)t * kAttnTile + 8 * (lane & 7);
                if (t >= end || slot >= keys) return -1;
                const uint32_t at = (uint32_t)((uint64_t)slot >> 3) / (uint32_t)(p.page_size >> 3);       // pages are whole runs
                const int page = __ldg(p.page_table + (int64_t)s.seq.b * p.max_pages + at);
                if (page < 0 || page >= p.num_pages) {
                    raise_status(p.status, SPR_ERR_BAD_PAGE);
                    return -1;
                }
                return (page * p.Hkv + part.head) * p.page_size + (int)(slot - (int64_t)at * p.page_size);
            };
            int next = find(part.t0);
            for (int n = 0; alive && n < part.n; n += 4) {
                const int rows = next;
                next = find(part.t0 + n + 4);
                for (int u = 0; alive && u < 4 && n + u < part.n; ++u) {
                    const int64_t left = keys - ((int64_t)part.t0 + n + u) * kAttnTile;
                    uint64_t valid = left >= 64 ? ~0ull : (1ull << left) - 1;
                    const uint32_t runs = __ballot_sync(0xffffffffu, rows >= 0) >> (8 * u) & 0xffu;
                    if (runs != 0xffu)
                        for (int r = 0; r < 8; ++r)
                            if (!(runs >> r & 1)) valid &= ~(0xffull << (8 * r));
                    const bool all = valid == ~0ull;
                    const int slot = (int)(unit % Shape::units);
                    const uint32_t round = (uint32_t)(unit / Shape::units);
                    if (round > 0 && !__all_sync(0xffffffffu, bar_wait(&ctl.empty[slot], (round - 1) & 1, &ctl.abort, p.status, limit))) {
                        alive = false;
                        break;
                    }
                    if (kv == 0 && lane == 0) {
                        ctl.valid[(unit >> 1) & 7] = valid;
                        __threadfence_block();
                    }
                    const __nv_bfloat16 *cache = static_cast<const __nv_bfloat16 *>(kv ? p.v : p.k);
                    const uint32_t dst = ring + slot * Shape::unit + c_dst;
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const int run = __shfl_sync(0xffffffffu, rows, 8 * u + r);
                        const __nv_bfloat16 *from = cache + (run < 0 ? 0 : ((int64_t)run + c_row) * p.D + c_chunk * 8);
#pragma unroll
                        for (int i = 0; i < 8 / kRowsAtOnce; ++i) {
                            const int r0 = i * kRowsAtOnce;
                            const bool there = c_in && (all || (valid >> (8 * r + r0 + c_row) & 1));
                            copy16((dst + (8 * r + r0) * 128) ^ (r0 << 4), there ? from : cache, there);
                            from += kRowsAtOnce * p.D;
                        }
                    }
                    // this lane arrives when its copies have
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_addr(&ctl.full[slot])) : "memory");
                    unit += 2;
                }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");       // none is left when the CTA ends
      } else {
        // ------------------------------------------------------------ products
        if (lane == 0) {
            constexpr uint32_t kQk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kAttnTile >> 3) << 17) | (8u << 24);
            constexpr uint32_t kPv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(COLS >> 3) << 17) | (8u << 24);
            AttnPart part;
            int64_t at = 0;                 // tiles of the stretch
            uint32_t parts = 0;
            bool alive = true;
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                if (alive && !bar_wait(bar, parity & 1, &ctl.abort, p.status, limit)) alive = false;
                return alive;
            };
            // (where S of tile i goes P of tile i - 2 was: the product with it is complete when this is called)
            auto scores = [&](int64_t i) {
                const int slot = (int)((2 * i) % Shape::units), b = (int)(i & 1);
                if (!wait(&ctl.full[slot], (uint32_t)((2 * i) / Shape::units))) return;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // the lanes' copies, for the tensor core
                fence_after();
                const uint32_t k = ring + slot * Shape::unit;
#pragma unroll
                for (int q = 0; q < 4 * PANELS; ++q)
                    mma_smem(tmem + kColS + 64 * b, tile_desc(q_tile + (q >> 2) * 128 * 128 + (q & 3) * 32, false),
                             tile_desc(k + (q >> 2) * kPanel + (q & 3) * 32, false), kQk, q != 0);
                commit(&ctl.s_full[b]);
                commit(&ctl.empty[slot]);
            };
            while (alive && attn_next<ROWS>(p, s, part)) {
                if (!wait(&ctl.q_ready, parts++)) break;
                scores(at);
                if (part.n > 1) scores(at + 1);
                for (int n = 0; alive && n < part.n; ++n, ++at) {
                    const int slot = (int)((2 * at + 1) % Shape::units);
                    if (!wait(&ctl.full[slot], (uint32_t)((2 * at + 1) / Shape::units)) || !wait(&ctl.p_ready[at & 1], (uint32_t)(at >> 1))) break;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    fence_after();
                    const uint32_t v = ring + slot * Shape::unit, w = tmem + kColS + 64 * (int)(at & 1);
                    const bool live = n > 0 || *reinterpret_cast<volatile int64_t *>(&ctl.o_live) == at;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        mma_tmem(tmem + kColO, w + 8 * q, tile_desc(v + q * 2048, true), kPv, live || q != 0);
                        if (!DUP) mma_tmem(tmem + kColO, w + 32 + 8 * q, tile_desc(v + q * 2048, true), kPv, 1u);
                    }
                    commit(&ctl.pv_done[at & 1]);
                    commit(&ctl.empty[slot]);
                    if (n + 2 < part.n) {
                        if (!wait(&ctl.pv_done[at & 1], (uint32_t)(at >> 1))) break;
                        scores(at + 2);
                    }
                }
            }
            commit(&ctl.drain);             // nothing of this CTA's products is left when its TMEM is given back
            bar_wait_quiet(&ctl.drain, 0, limit);
        }
        __syncwarp();
      }
    } else {
        // ------------------------------------------------------------ softmax: a row per thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16), col_o = lanes + kColO;
        const int row = DUP ? tid & 63 : tid;               // in the block
        const bool second = DUP && tid >= 64;               // this thread's weights are what rounding left
        const float c = p.abs_scale_log2;
        AttnPart part;
        int64_t at = 0;
        int tree_of = -1;
        bool dead = false;
        auto wait = [&](uint64_t *bar, uint32_t parity) {
            if (!dead) dead = !__all_sync(0xffffffffu, bar_wait(bar, parity & 1, &ctl.abort, p.status, limit));
        };
        auto warp_arrive = [&](uint64_t *bar) {
            __syncwarp();
            if (lane == 0) arrive(bar);
        };
        while (attn_next<ROWS>(p, s, part)) {
            const AttnTarget t = attn_target<ROWS>(p, s, part);
            // this row's query (zeros where there is none; all products of the part before have been formed)
            const bool in = row < t.rows;
            const int64_t out_at = in ? attn_out_at(p, s, part, t.row0 + row) : 0;
            softmax_meet();
            {
                const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) + out_at);
#pragma unroll
                for (int k = 0; k < 8 * PANELS; ++k) {
                    uint4 x = in && k * 8 < p.D ? __ldg(src + k) : make_uint4(0u, 0u, 0u, 0u);
                    x.x ^= p.flip, x.y ^= p.flip, x.z ^= p.flip, x.w ^= p.flip;
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};"
                                 ::"r"(q_tile + (k >> 3) * 128 * 128 + tid * 128 + (((k & 7) ^ (tid & 7)) << 4)), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            warp_arrive(&ctl.q_ready);
            const uint32_t *path = ctl.path[0];
            if ((int64_t)(part.t0 + part.n) * kAttnTile > s.seq.len) {       // some tile holds nodes
                const int i0 = (int)(t.row0 / p.G);
                const int nodes = (int)((t.row0 + t.rows - 1) / p.G) - i0 + 1;
                if (p.nodes.parents && tree_of != s.seq.b) {
                    for (int j = tid; j < s.seq.count; j += kSoftmaxThreads) ctl.tree[j] = p.nodes.parents[(int64_t)s.seq.b * p.nodes.T + j];
                    tree_of = s.seq.b;
                    softmax_meet();
                }
                if (tid < nodes) {
                    for (int w = (s.seq.count + 31) / 32; w < kMaxTreeNodes / 32; ++w) ctl.path[tid][w] = 0u;
                    attn_path_bits(p.nodes.parents ? ctl.tree : nullptr, i0 + tid, ctl.path[tid], (s.seq.count + 31) / 32, p.status);
                }
                if (in) path = ctl.path[(int)((t.row0 + row) / p.G) - i0];
                softmax_meet();
            }

            float m = neg_inf(), l = 0.f;
            for (int n = 0; n < part.n; ++n, ++at) {
                const uint32_t col_s = lanes + kColS + 64 * (uint32_t)(at & 1);
                const bool begun = n > 0;
                float x[64];
                wait(&ctl.s_full[at & 1], (uint32_t)(at >> 1));
                fence_after();
                tmem_read32(col_s, *reinterpret_cast<float (*)[32]>(x));
                tmem_read32(col_s + 32, *reinterpret_cast<float (*)[32]>(x + 32));
                tmem_wait();
                const int64_t slot0 = ((int64_t)part.t0 + n) * kAttnTile;
                const uint64_t valid = ctl.valid[at & 7];
                const uint32_t v_unit = ring + (int)((2 * at + 1) % Shape::units) * Shape::unit;
                const bool tail = slot0 + kAttnTile > s.seq.len;      // (alike in all threads, whatever went wrong: they meet)
                unsigned long long odd = 0;
                uint64_t vis = valid;
                if (tail) {
                    const int64_t d = s.seq.len - slot0;     // keys of the prefix
                    vis &= d <= 0 ? path_bits64(path, (int)-d) : path_bits64(path, 0) << d | ((1ull << d) - 1);
                }
                if (vis != ~0ull) {
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        if (!((i < 32 ? (uint32_t)vis : (uint32_t)(vis >> 32)) >> (i & 31) & 1)) x[i] = neg_inf();
                }
                if (tail) {
                    // values that are not finite, where not every row sees every key: each thread looks at half a key
                    wait(&ctl.full[(2 * at + 1) % Shape::units], (uint32_t)((2 * at + 1) / Shape::units));
                    const uint32_t v = v_unit + (tid >> 1) * 128 + (tid & 1) * 64;
                    bool bad = false;
#pragma unroll
                    for (int k = 0; k < 4 * PANELS; ++k) {
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(v + (k >> 2) * kPanel + (k & 3) * 16) : "memory");
                        bad = bad || !(finite_bf16x2(w[0]) && finite_bf16x2(w[1]) && finite_bf16x2(w[2]) && finite_bf16x2(w[3]));
                    }
                    softmax_meet();
                    if (bad) atomicOr(&ctl.odd, 1ull << (tid >> 1));
                    softmax_meet();
                    odd = *reinterpret_cast<volatile unsigned long long *>(&ctl.odd);
                }
                float t4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                for (int i = 4; i < 64; i += 2) t4[(i >> 1) & 3] = fmaxf(fmaxf(t4[(i >> 1) & 3], x[i]), x[i + 1]);
                const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
                // (m = -inf: nothing seen so far, and O holds nothing of this row)
                const bool raise = top > m && (m == neg_inf() || (top - m) * c > kRaise);
                if (begun && (__any_sync(0xffffffffu, raise) || odd)) wait(&ctl.pv_done[(at - 1) & 1], (uint32_t)((at - 1) >> 1));
                if (__any_sync(0xffffffffu, raise)) {
                    const float a = raise && m != neg_inf() ? ex2((m - top) * c) : 1.f;
                    if (raise) m = top;
                    l *= a;
                    if (begun && __any_sync(0xffffffffu, a != 1.f)) {
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
                float sum0, sum1;
                unpack2(add2(s2[0], s2[1]), sum0, sum1);
                l += sum0 + sum1;
                if (odd) {
                    // taken out of the product, and added one by one to the rows that see them
                    fence_after();
                    const uint32_t v = v_unit;
#pragma unroll 1
                    for (int k = 0; k < 2 * PANELS; ++k) {
                        float o[32];
                        uint32_t w[32];
                        tmem_read32(col_o + 32 * k, o);
                        tmem_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!begun) o[i] = 0.f;
                        for (unsigned long long rest = odd & vis; rest && !second; rest &= rest - 1) {
                            const int key = __ffsll((long long)rest) - 1;
                            float weight = 0.f;
#pragma unroll
                            for (int i = 0; i < 64; ++i) weight = i == key ? x[i] : weight;
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                uint32_t y;
                                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(y)
                                             : "r"(v + (k >> 1) * kPanel + key * 128 + ((((k & 1) * 4 + (i >> 2)) ^ (key & 7)) << 4) + (i & 3) * 4) : "memory");
                                o[2 * i] = fmaf(weight, __uint_as_float(y << 16), o[2 * i]);
                                o[2 * i + 1] = fmaf(weight, __uint_as_float(y & 0xffff0000u), o[2 * i + 1]);
                            }
                        }
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(o[i]);
                        tmem_write32(col_o + 32 * k, w);
                    }
                    softmax_meet();
                    if (odd >> (tid >> 1) & 1)
                        for (int k = 0; k < 4 * PANELS; ++k)
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v + (tid >> 1) * 128 + (tid & 1) * 64 + (k >> 2) * kPanel + (k & 3) * 16), "r"(0u) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    if (tid == 0) {
                        ctl.odd = 0;
                        if (!begun) ctl.o_live = at;
                    }
                    softmax_meet();
                }
                uint32_t w[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
                if (!DUP || !second) tmem_write32(col_s, w);
                if (!DUP || second) {
                    const uint64_t minus = pack2(-1.f, -1.f);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float a, b;
                        unpack2(fma2(pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), minus, pack2(x[2 * i], x[2 * i + 1])), a, b);
                        w[i] = pack_bf16(a, b);
                    }
                    tmem_write32(col_s + (DUP ? 0 : 32), w);
                }
                tmem_wait_st();
                fence_before();
                warp_arrive(&ctl.p_ready[at & 1]);
            }

            // -------------------------------------------------------- the part's results
            wait(&ctl.pv_done[(at - 1) & 1], (uint32_t)((at - 1) >> 1));
            fence_after();
            if (dead) l = __int_as_float(0x7fc00000);       // what a wait that ran out leaves is no result
            const float inv = l == 0.f ? 0.f : 1.f / l;
            if (DUP) {      // the second numbers' results, by way of the query tile
                if (second) {
#pragma unroll 1
                    for (int k = 0; k < 2 * PANELS; ++k) {
                        float o[32];
                        tmem_read32(col_o + 32 * k, o);
                        tmem_wait();
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};"
                                         ::"r"(q_tile + row * COLS * 4 + (((8 * k + i) ^ (row & 7)) << 4)), "f"(o[4 * i]), "f"(o[4 * i + 1]), "f"(o[4 * i + 2]), "f"(o[4 * i + 3]) : "memory");
                    }
                }
                softmax_meet();
            }
            if (!second) {
#pragma unroll 1
                for (int k = 0; k < 2 * PANELS; ++k) {
                    float o[32];
                    tmem_read32(col_o + 32 * k, o);
                    tmem_wait();
                    if (DUP) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float y[4];
                            asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(y[0]), "=f"(y[1]), "=f"(y[2]), "=f"(y[3])
                                         : "r"(q_tile + row * COLS * 4 + (((8 * k + i) ^ (row & 7)) << 4)) : "memory");
                            o[4 * i] += y[0], o[4 * i + 1] += y[1], o[4 * i + 2] += y[2], o[4 * i + 3] += y[3];
                        }
                    }
                    if (in) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int col = 32 * k + 8 * i;
                            if (col >= p.D) continue;
                            if (t.whole) {
                                *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) + out_at + col) =
                                    make_uint4(pack_bf16(o[8 * i] * inv, o[8 * i + 1] * inv), pack_bf16(o[8 * i + 2] * inv, o[8 * i + 3] * inv),
                                               pack_bf16(o[8 * i + 4] * inv, o[8 * i + 5] * inv), pack_bf16(o[8 * i + 6] * inv, o[8 * i + 7] * inv));
                            } else {
                                float4 *to = reinterpret_cast<float4 *>(p.part + ((int64_t)t.slot * ROWS + row) * p.D + col);
                                __stcg(to, make_float4(o[8 * i], o[8 * i + 1], o[8 * i + 2], o[8 * i + 3]));
                                __stcg(to + 1, make_float4(o[8 * i + 4], o[8 * i + 5], o[8 * i + 6], o[8 * i + 7]));
                            }
                        }
                    }
                    __syncwarp();
                }
                if (!t.whole && in) __stcg(&p.part_ml[(int64_t)t.slot * ROWS + row], make_float2(m * c, l));
            }
            fence_before();
            if (!t.whole) {
                __threadfence();
                softmax_meet();
                if (tid == 0) ctl.last = take_ticket(p.counters + t.first, t.parts);
                softmax_meet();
                if (ctl.last) {
                    __threadfence();
                    attn_join<ROWS, __nv_bfloat16>(p, s, part, t, warp, kSoftmaxThreads / 32);
                }
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

template <int PANELS, bool DUP>
cudaError_t launch_tc(const AttnParams &p, int dev, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];   // host threads may race to set it: all of them store `true`
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_tc_kernel<PANELS, DUP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)TcShape<PANELS>::smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    attention_tc_kernel<PANELS, DUP><<<p.ctas, kTcThreads, TcShape<PANELS>::smem, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_tc(const AttnParams &p, int rows, int dev, cudaStream_t st)
{
    if (rows == 64) return p.D <= 64 ? launch_tc<1, true>(p, dev, st) : launch_tc<2, true>(p, dev, st);
    return p.D <= 64 ? launch_tc<1, false>(p, dev, st) : launch_tc<2, false>(p, dev, st);
}

}  // namespace spr
