// tree_attention on bf16 tensors, few rows per cached head (decoding, chains).
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j in one pass over the keys, with a running maximum and sum.  Bound by the
// read of the caches: a key and its value (4 D bytes) meet ROWS queries.  One producer warp brings tiles of 64 keys into
// a ring by TMA, one lane per box of a page (128-byte swizzle); page numbers are read a batch ahead.  Eight consumer
// warps form two teams that take tiles in turn, each warp 16 of a tile's keys: it has its own maxima, sums
// and results (mma.sync m16n8k16, the block's rows as M), so that warps wait for nothing but their tiles, and
// they are joined through shared memory at the end of a part.  mma.sync suffices here: at 16 rows a tile
// of 32 KB (the time of 1400 clocks at the memory's rate) takes 128 products per tensor core, some 300 clocks; tcgen05's
// smallest tile has 64 rows.
//
// Weights are used as two bf16 numbers (their rounding and what is left of it): with one, results would be off by 2^-9
// of themselves for that alone, as much as by their own rounding.  The second product is free where the
// memory is what bounds it.
#include <atomic>

#include "attention_plan.cuh"
#include "host_util.h"
#include "launch.h"
#include "tensor_pair.cuh"

namespace spr {

namespace {

using namespace pairtc;

constexpr int kMmaConsumers = 256;
constexpr int kMmaThreads = kMmaConsumers + 32;
constexpr int kMmaWarps = kMmaConsumers / 32;
constexpr int kTeams = 2;
constexpr int kPanelBytes = kAttnTile * 128;            // 64 keys by 64 columns
constexpr int kJoinPitch = 68;                          // floats per row of the joining buffer
constexpr int kJoinBytes = kMmaWarps * 16 * kJoinPitch * 4;

template <int PANELS>
struct MmaShape {
    static constexpr int stage = 2 * PANELS * kPanelBytes;      // keys, then values
    static constexpr int stages = PANELS == 2 ? 5 : 10;
    static constexpr size_t smem = (size_t)stages * stage + kJoinBytes + 1024;
};

struct MmaControl {
    uint64_t full[10], empty[10];
    uint64_t valid[10];              // a bit for each key of the stage's tile that is there
    int64_t scratch[2 * (kMmaThreads / 32) + 4];
    int tree[kMaxTreeNodes];
    uint32_t path[32][kMaxTreeNodes / 32];
    float2 ml[kMmaWarps][32];
    int last, abort;
};

__device__ __forceinline__ void consumers_meet() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

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
__device__ __forceinline__ void load_tile_box(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(smem_addr(bar))
        : "memory");
}
__device__ __forceinline__ void arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// all lanes of a warp wait; false when any of them gave up
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, int *abort, int *status, uint32_t limit)
{
    return __all_sync(0xffffffffu, bar_wait(bar, parity, abort, status, limit));
}
__device__ __forceinline__ bool finite_bf16x2(uint32_t w) { return (w & 0x7f80u) != 0x7f80u && (w & 0x7f800000u) != 0x7f800000u; }

// MT: row tiles of 16; PANELS: 64-column halves of the head dimension
template <int MT, int PANELS>
__global__ void __launch_bounds__(kMmaThreads, 1)
attention_mma_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const AttnParams p)
{
    constexpr int ROWS = 16 * MT, KSTEPS = 4 * PANELS, NTILES = 8 * PANELS;
    using Shape = MmaShape<PANELS>;
    extern __shared__ uint8_t raw[];
    __shared__ MmaControl ctl;
    const uint32_t ring = (smem_addr(raw) + 1023u) & ~1023u;
    float *join = reinterpret_cast<float *>(raw + (ring - smem_addr(raw)) + (size_t)Shape::stages * Shape::stage);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < Shape::stages; ++i) {
            bar_init(&ctl.full[i], 1);
            bar_init(&ctl.empty[i], kMmaWarps / kTeams);
        }
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    AttnStretch s = attn_plan<ROWS, kMmaThreads>(p, ctl.scratch);
    __syncthreads();
    attn_clear_unused<__nv_bfloat16>(p, kMmaThreads);

    if (warp == kMmaWarps) {
        // ------------------------------------------------------------ producer
        const int boxes = kAttnTile / p.box;               // per tile
        AttnPart part;
        int64_t issued = 0;
        bool alive = !(p.test_flags & ATTN_TEST_NO_LOADS);
        while (alive && attn_next<ROWS>(p, s, part)) {
            const int64_t keys = min((int64_t)s.seq.len + s.seq.count, (int64_t)p.max_pages * p.page_size);
            if (keys < (int64_t)s.seq.len + s.seq.count && lane == 0) raise_status(p.status, SPR_ERR_BAD_PAGE);
            const int32_t *table = p.page_table + (int64_t)s.seq.b * p.max_pages;
            const int per_batch = 32 / boxes;               // tiles whose boxes a warp's lanes hold
            const int my_tile = lane / boxes, my_box = lane - my_tile * boxes;
            // row of the caches where this lane's box of a batch begins; -1 where there is none
            auto find = [&](int tile0) -> int64_t {
                const int64_t slot = ((int64_t)tile0 + my_tile) * kAttnTile + my_box * p.box;
                if (my_tile >= per_batch || tile0 + my_tile >= part.t0 + part.n || slot >= keys) return -1;
                const int64_t at = slot / p.page_size;
                const int page = __ldg(table + at);
                if (page < 0 || page >= p.num_pages) {
                    raise_status(p.status, SPR_ERR_BAD_PAGE);
                    return -1;
                }
                return ((int64_t)page * p.Hkv + part.head) * p.page_size + (slot - at * p.page_size);
            };
            int64_t next = find(part.t0);
            for (int n = 0; alive && n < part.n; n += per_batch) {
                const int64_t row = next;
                if (n + per_batch < part.n) next = find(part.t0 + n + per_batch);
                const uint32_t there = __ballot_sync(0xffffffffu, row >= 0);
                for (int u = 0; u < per_batch && n + u < part.n; ++u, ++issued) {
                    const int stage = (int)(issued % Shape::stages);
                    const uint32_t round = (uint32_t)(issued / Shape::stages);
                    if (round > 0 && !warp_wait(&ctl.empty[stage], (round - 1) & 1, &ctl.abort, p.status, p.spin_limit)) {
                        alive = false;
                        break;
                    }
                    const uint32_t mine = there >> (u * boxes) & ((1u << boxes) - 1);
                    if (lane == 0) {
                        // keys of this tile that are there: whole boxes, up to the last key
                        const int64_t left = keys - ((int64_t)part.t0 + n + u) * kAttnTile;
                        uint64_t bits = 0;
                        for (int i = 0; i < boxes; ++i)
                            if (mine >> i & 1) bits |= (p.box == 64 ? ~0ull : ((1ull << p.box) - 1)) << (i * p.box);
                        if (left < 64) bits &= (1ull << left) - 1;
                        ctl.valid[stage] = bits;
                        bar_expect(&ctl.full[stage], (uint32_t)(__popc(mine) * p.box * 128 * 2 * PANELS));
                    }
                    __syncwarp();
                    if (my_tile == u && row >= 0) {
                        const uint32_t dst = ring + stage * Shape::stage + my_box * p.box * 128;
#pragma unroll
                        for (int h = 0; h < PANELS; ++h) {
                            load_tile_box(dst + h * kPanelBytes, &k_map, 64 * h, (int)row, &ctl.full[stage]);
                            load_tile_box(dst + (PANELS + h) * kPanelBytes, &v_map, 64 * h, (int)row, &ctl.full[stage]);
                        }
                    }
                    __syncwarp();
                }
            }
        }
        // copies in flight write shared memory: none may be left when the CTA ends
        for (int64_t i = issued > Shape::stages ? issued - Shape::stages : 0; i < issued; ++i)
            bar_wait_quiet(&ctl.full[i % Shape::stages], (uint32_t)(i / Shape::stages) & 1, p.spin_limit);
        return;
    }

    // ---------------------------------------------------------------- consumers
    const int team = warp / (kMmaWarps / kTeams), w16 = (warp % (kMmaWarps / kTeams)) * 16;     // keys w16 .. + 15 of the tile
    // ldmatrix addresses within a panel: keys (non-transposed): matrices (keys 0-7 | 8-15) x (columns 0-7 | 8-15)
    const int k_row = w16 + (lane & 7) + ((lane >> 4) << 3), k_chunk = (lane >> 3) & 1;
    const int v_row = w16 + (lane & 7) + (((lane >> 3) & 1) << 3), v_chunk = lane >> 4;
    const uint32_t k_off = k_row * 128, v_off = v_row * 128;
    const int swz = lane & 7;                               // both rows are lane & 7 modulo 8
    const int quad = lane >> 2, pair = lane & 3;
    AttnPart part;
    int64_t taken = 0;                                      // tiles of this CTA's stretch before the part
    int tree_of = -1;
    bool alive = true;
    while (attn_next<ROWS>(p, s, part)) {
        const AttnTarget t = attn_target<ROWS>(p, s, part);
        const int i0 = (int)(t.row0 / p.G);
        const int nodes = (int)((t.row0 + t.rows - 1) / p.G) - i0 + 1;
        consumers_meet();
        if (p.nodes.parents && tree_of != s.seq.b) {
            for (int j = tid; j < s.seq.count; j += kMmaConsumers) ctl.tree[j] = p.nodes.parents[(int64_t)s.seq.b * p.nodes.T + j];
            tree_of = s.seq.b;
            consumers_meet();
        }
        if (tid < nodes)
            attn_path_bits(p.nodes.parents ? ctl.tree : nullptr, i0 + tid, ctl.path[tid], (s.seq.count + 31) / 32, p.status);

        // queries as A fragments: rows quad and quad + 8 of each row tile
        uint32_t qf[MT][KSTEPS][4];
        int node[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = mt * 16 + h * 8 + quad;
                const bool in = r < t.rows;
                node[mt][h] = in ? (int)((t.row0 + r) / p.G) - i0 : 0;
                const uint32_t *src = reinterpret_cast<const uint32_t *>(static_cast<const __nv_bfloat16 *>(p.q) + (in ? attn_out_at(p, s, part, t.row0 + r) : 0));
#pragma unroll
                for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int col = k * 16 + c * 8 + pair * 2;
                        qf[mt][k][c * 2 + h] = in && col < p.D ? __ldg(src + col / 2) : 0u;
                    }
            }
        consumers_meet();

        float o[MT][NTILES][4], m[MT][2], l[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt][0] = m[mt][1] = neg_inf();
            l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
            for (int n = 0; n < NTILES; ++n) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
        }
        for (int n = 0; n < part.n; ++n) {
            const int64_t at = taken + n;
            if ((int)(at % kTeams) != team) continue;
            const int stage = (int)(at % Shape::stages);
            if (!alive || !warp_wait(&ctl.full[stage], (uint32_t)(at / Shape::stages) & 1, &ctl.abort, p.status, p.spin_limit)) {
                alive = false;
                break;
            }
            const uint32_t ks = ring + stage * Shape::stage, vs = ks + PANELS * kPanelBytes;
            const uint32_t valid = (uint32_t)(ctl.valid[stage] >> w16) & 0xffffu;
            const int64_t slot0 = ((int64_t)part.t0 + n) * kAttnTile + w16;
            const bool all = valid == 0xffffu && slot0 + 16 <= s.seq.len;

            float sc[MT][2][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h) sc[mt][h][0] = sc[mt][h][1] = sc[mt][h][2] = sc[mt][h][3] = 0.f;
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k) {
                uint32_t b[4];
                ldsm(ks + (k >> 2) * kPanelBytes + k_off + ((((k & 3) * 2 + k_chunk) ^ swz) << 4), b);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mma(sc[mt][0], qf[mt][k], b[0], b[1]);
                    mma(sc[mt][1], qf[mt][k], b[2], b[3]);
                }
            }
            uint32_t odd = 0;               // keys whose values hold infinities or NaN, where not every row sees every key
            if (!all) {
                // values of keys that are not there are whatever the page or the ring held: zeros.  Values that are
                // not finite are taken out of the product and added one by one to the rows that see them.
                const int row = lane & 15, half = lane >> 4;
                const bool there = valid >> row & 1;
                bool bad = false;
                for (int h = 0; h < PANELS; ++h)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t a = vs + h * kPanelBytes + (w16 + row) * 128 + (half * 4 + c) * 16;
                        uint32_t x[4];
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(a) : "memory");
                        bad = bad || !(finite_bf16x2(x[0]) && finite_bf16x2(x[1]) && finite_bf16x2(x[2]) && finite_bf16x2(x[3]));
                        if (!there) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(a), "r"(0u) : "memory");
                    }
                odd = __ballot_sync(0xffffffffu, bad && there);
                odd = (odd | odd >> 16) & 0xffffu;
                __syncwarp();
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                // c registers 0, 1: row quad, keys 2 pair, 2 pair + 1; 2, 3: row quad + 8
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float x = sc[mt][h][c] * p.scale_log2;
                        if (!all) {
                            const int key = h * 8 + pair * 2 + (c & 1);
                            const int64_t j = slot0 + key - s.seq.len;
                            const bool vis = (valid >> key & 1) && (j < 0 || (ctl.path[node[mt][c >> 1]][j >> 5] >> (j & 31) & 1));
                            if (!vis) x = neg_inf();
                        }
                        sc[mt][h][c] = x;
                    }
                float top[2];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float x = fmaxf(fmaxf(sc[mt][0][2 * g], sc[mt][0][2 * g + 1]), fmaxf(sc[mt][1][2 * g], sc[mt][1][2 * g + 1]));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                    top[g] = fmaxf(x, m[mt][g]);
                }
                if (__any_sync(0xffffffffu, top[0] > m[mt][0] || top[1] > m[mt][1])) {
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const float a = ex2(m[mt][g] - (top[g] == neg_inf() ? 0.f : top[g]));
                        m[mt][g] = top[g];
                        l[mt][g] *= a;
#pragma unroll
                        for (int i = 0; i < NTILES; ++i) {
                            o[mt][i][2 * g] *= a;
                            o[mt][i][2 * g + 1] *= a;
                        }
                    }
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const float ref = m[mt][g] == neg_inf() ? 0.f : m[mt][g];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float w = ex2(sc[mt][h][2 * g + c] - ref);
                            sc[mt][h][2 * g + c] = w;
                            l[mt][g] += w;
                        }
                }
            }
            if (odd) {
                for (int key = 0; key < 16; ++key) {
                    if (!(odd >> key & 1)) continue;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const int h = key >> 3, c = key & 1, from = (lane & 28) | ((key & 7) >> 1);
                            const float w0 = h ? sc[mt][1][2 * g] : sc[mt][0][2 * g], w1 = h ? sc[mt][1][2 * g + 1] : sc[mt][0][2 * g + 1];
                            const float w = __shfl_sync(0xffffffffu, c ? w1 : w0, from);
                            const int64_t j = slot0 + key - s.seq.len;
                            if (j < 0 || (ctl.path[node[mt][g]][j >> 5] >> (j & 31) & 1)) {
#pragma unroll
                                for (int i = 0; i < NTILES; ++i) {
                                    const uint32_t a = vs + (i >> 3) * kPanelBytes + (w16 + key) * 128 + (((i & 7) ^ ((w16 + key) & 7)) << 4) + pair * 4;
                                    uint32_t x;
                                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(a) : "memory");
                                    o[mt][i][2 * g] = fmaf(w, __uint_as_float(x << 16), o[mt][i][2 * g]);
                                    o[mt][i][2 * g + 1] = fmaf(w, __uint_as_float(x & 0xffff0000u), o[mt][i][2 * g + 1]);
                                }
                            }
                        }
                }
                __syncwarp();
                if (odd >> (lane & 15) & 1)
                    for (int h = 0; h < PANELS; ++h)
                        for (int c = 0; c < 4; ++c)
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(vs + h * kPanelBytes + (w16 + (lane & 15)) * 128 + ((lane >> 4) * 4 + c) * 16), "r"(0u) : "memory");
                __syncwarp();
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            // weights as A fragments, in two parts
            uint32_t hi[MT][4], lo[MT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const float a = sc[mt][h][2 * g], b = sc[mt][h][2 * g + 1];
                        const uint32_t w = pack_bf16(a, b);
                        hi[mt][h * 2 + g] = w;
                        lo[mt][h * 2 + g] = pack_bf16(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
                    }
#pragma unroll
            for (int i = 0; i < NTILES / 2; ++i) {
                uint32_t b[4];
                ldsm_t(vs + (i >> 2) * kPanelBytes + v_off + ((((i & 3) * 2 + v_chunk) ^ swz) << 4), b);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mma(o[mt][2 * i], hi[mt], b[0], b[1]);
                    mma(o[mt][2 * i + 1], hi[mt], b[2], b[3]);
                    mma(o[mt][2 * i], lo[mt], b[0], b[1]);
                    mma(o[mt][2 * i + 1], lo[mt], b[2], b[3]);
                }
            }
            __syncwarp();
            if (lane == 0) arrive(&ctl.empty[stage]);
        }
        taken += part.n;

        // ------------------------------------------------------------ the warps' results joined
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float x = l[mt][g];
                x += __shfl_xor_sync(0xffffffffu, x, 1);
                x += __shfl_xor_sync(0xffffffffu, x, 2);
                if (!alive) x = __int_as_float(0x7fc00000);        // what a wait that ran out leaves is no result
                if (pair == 0) ctl.ml[warp][mt * 16 + g * 8 + quad] = make_float2(m[mt][g], x);
            }
        consumers_meet();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float top[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                top[g] = neg_inf();
#pragma unroll
                for (int w = 0; w < kMmaWarps; ++w) top[g] = fmaxf(top[g], ctl.ml[w][mt * 16 + g * 8 + quad].x);
                const float a = ex2(m[mt][g] - (top[g] == neg_inf() ? 0.f : top[g]));
#pragma unroll
                for (int i = 0; i < NTILES; ++i) {
                    o[mt][i][2 * g] *= a;
                    o[mt][i][2 * g + 1] *= a;
                }
            }
            const int row = tid >> 4, c4 = (tid & 15) * 4;      // what this thread adds up
            float tall = neg_inf(), sum = 0.f;
#pragma unroll
            for (int w = 0; w < kMmaWarps; ++w) tall = fmaxf(tall, ctl.ml[w][mt * 16 + row].x);
#pragma unroll
            for (int w = 0; w < kMmaWarps; ++w) {
                const float2 x = ctl.ml[w][mt * 16 + row];
                sum = fmaf(ex2(x.x - (tall == neg_inf() ? 0.f : tall)), x.y, sum);
            }
#pragma unroll
            for (int h = 0; h < PANELS; ++h) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int g = 0; g < 2; ++g)
                        *reinterpret_cast<float2 *>(join + (warp * 16 + g * 8 + quad) * kJoinPitch + i * 8 + pair * 2) =
                            make_float2(o[mt][h * 8 + i][2 * g], o[mt][h * 8 + i][2 * g + 1]);
                consumers_meet();
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kMmaWarps; ++w) {
                    const float4 x = *reinterpret_cast<const float4 *>(join + (w * 16 + row) * kJoinPitch + c4);
                    y.x += x.x, y.y += x.y, y.z += x.z, y.w += x.w;
                }
                const int r = mt * 16 + row, c = h * 64 + c4;
                if (r < t.rows && c < p.D) {
                    if (t.whole) {
                        const float inv = sum == 0.f ? 0.f : 1.f / sum;
                        store_out(static_cast<__nv_bfloat16 *>(p.out) + attn_out_at(p, s, part, t.row0 + r) + c,
                                  make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv), 4);
                    } else {
                        __stcg(reinterpret_cast<float4 *>(p.part + ((int64_t)t.slot * ROWS + r) * p.D + c), y);
                        if (c == 0) __stcg(&p.part_ml[(int64_t)t.slot * ROWS + r], make_float2(tall, sum));
                    }
                }
                consumers_meet();
            }
        }
        if (!t.whole) {
            __threadfence();
            consumers_meet();
            if (tid == 0) ctl.last = take_ticket(p.counters + t.first, t.parts);
            consumers_meet();
            if (ctl.last) {
                __threadfence();
                attn_join<ROWS, __nv_bfloat16>(p, s, part, t, tid, kMmaConsumers);
            }
        }
    }
}

template <int MT, int PANELS>
cudaError_t launch_mma(const AttnParams &p, const CUtensorMap &k, const CUtensorMap &v, int dev, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];   // host threads may race to set it: all of them store `true`
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_mma_kernel<MT, PANELS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)MmaShape<PANELS>::smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    attention_mma_kernel<MT, PANELS><<<p.ctas, kMmaThreads, MmaShape<PANELS>::smem, st>>>(k, v, p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_mma(const AttnParams &p, int rows, const CUtensorMap &k, const CUtensorMap &v, int dev, cudaStream_t st)
{
    if (rows == 16) return p.D <= 64 ? launch_mma<1, 1>(p, k, v, dev, st) : launch_mma<1, 2>(p, k, v, dev, st);
    return p.D <= 64 ? launch_mma<2, 1>(p, k, v, dev, st) : launch_mma<2, 2>(p, k, v, dev, st);
}

}  // namespace spr
