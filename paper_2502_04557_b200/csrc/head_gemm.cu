// Matrix products of the vocabulary head (softmax cross entropy and its gradient) on CTA pairs.
//
//   logits = H W^T        kept nowhere: the epilogue turns a tile into row statistics, or into
//                         the tile of the softmax gradient D
//   dH = D W, dW = D^T H  D comes from the workspace
//
// Bound by the tensor pipe for batches of a few hundred tokens and more, by the sweep over W
// below that.  A pair of CTAs (cluster of 2) owns a 256 x 256 tile: each CTA stages 128 rows of A
// and 128 of B per 64-deep stage (32 KB by TMA, 128-byte swizzle, no multicast), one thread of the
// even CTA issues tcgen05.mma.cta_group::2 for both, and the accumulator (256 fp32 columns in each
// CTA's TMEM) is double-buffered: while the eight epilogue warps work on one the other is filled.
// The grid is persistent, one CTA per SM.  An operand tile is loaded as 64 x 64 boxes
// whether its contiguous axis runs along the contraction or across it, so that D and D^T, W and
// W^T are read from one copy of each; the matrix descriptors say which.
//
// The tensor pipe truncates when it adds to the accumulator: every 16 elements of the contraction
// cost up to one unit in the last place, always towards zero (measured: a log-sum-exp of products
// 2048 deep came out 2.3e-6 low, a ratio of two such probabilities 1.2e-5 off).  Where the result is
// wanted to fp32 - row statistics, and everything with fp32 operands - an accumulator therefore
// takes only `kc` blocks of 64, and the epilogue warps add such chunks up in registers, rounding
// to nearest.  They have the time: a chunk is read in about a quarter of the time it takes to form.
// Results that are rounded to bf16 do so, too, where a contraction is long enough to show (head_loss.cu).
//
// fp32 operands: x = x0 + x1 + x2 with bf16 parts (8 significant bits each: the remainder is
// below 2^-24 |x|).  The six products of parts with i + j <= 2 make the result exact to about
// 2^-23; in each chunk they are accumulated smallest first, so that the truncations that count
// are those of the last product alone.
//
// Warp roles (320 threads): warp 0 = TMA producer, warp 1 = TMEM owner and MMA issuer, warps
// 2..9 = epilogue (warp w reads TMEM lanes 32 (w % 4) .. + 31, one row per thread, and half of the
// tile's 256 columns: all 128 in registers where chunks are added up, else 32 at a time).  Results go
// out through 4 KB of shared memory per warp: bf16 as TMA boxes of 64 columns by 32 rows (against stores from
// registers: gradient of 256x768x50257 86 -> 84 us, 128x4096x32000 241 -> 229 us), the rest in store instructions that
// write whole 128-byte lines (a thread per row would touch 32 lines with each).  Every wait is bounded: when one
// runs out the status word becomes SPR_ERR_TIMEOUT, all roles leave their loops, the even CTA
// waits (again bounded) for the copies and products in flight, and both CTAs meet before they exit.
//
// What bounds it.  An SM takes in some 41 bytes a clock from L2 whatever the tiles, so that a step of 64 KB per pair
// takes 0.42 us (1424 TFLOP/s over 74 pairs; measured 4096x2048x128256: loss 1510 - 1770 us, 1.22 - 1.43 PFLOP/s as the
// power cap allows, the library's plain bf16 product 1.39 sustained).  With a few hundred tokens: one sweep over W in
// waves of 74 tiles (256x768x50257: 197 tiles, three waves where 2.66 are work), and for the gradient the write
// of dW beside it (77 MB there; a fill of as much takes 12 us).
#include <atomic>

#include "head_gemm.h"
#include "launch.h"
#include "tensor_pair.cuh"
#include "vocab_common.cuh"

namespace spr {

namespace {

using namespace pairtc;

constexpr int kPairThreads = 320;
constexpr int kFirstEpilogueWarp = 2;
constexpr int kHalfBytes = 128 * kPairBlockK * 2;       // this CTA's half of an operand tile: two 64 x 64 boxes
constexpr int kBoxBytes = 64 * 64 * 2;
constexpr int kStageBytes = 2 * kHalfBytes;
constexpr int kStages = 6;
constexpr int kTmemCols = 512;                          // two accumulators of 256 columns

struct PairControl {
    uint64_t full[kStages];
    uint64_t empty[kStages];
    uint64_t acc_full[2];
    uint64_t acc_empty[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
    long long consumed;      // stages whose operands the MMA issuer saw arrive
};
constexpr int kOutBytes = 32 * 32 * 4;                  // staging of one epilogue warp: 32 rows of 32 fp32 columns
constexpr int kOutOffset = kStages * kStageBytes;
constexpr int kCtlOffset = kOutOffset + 8 * kOutBytes;
constexpr size_t kPairSmem = (size_t)kCtlOffset + 1024 + sizeof(PairControl);
static_assert(kPairSmem <= 232448, "shared memory of one CTA");

// what a pair does, in order: its items of job 0, then its run of job 1
struct Item {
    int job, m, n, split;
};
__device__ __forceinline__ int items_of_pair(const PairParams &prm, int pair, int pairs)
{
    const int n0 = pair < prm.items[0] ? (prm.items[0] - pair + pairs - 1) / pairs : 0;
    return n0 + (prm.items[1] ? prm.count1[pair] : 0);
}
__device__ __forceinline__ Item get_item(const PairParams &prm, int pair, int pairs, int i)
{
    const int n0 = pair < prm.items[0] ? (prm.items[0] - pair + pairs - 1) / pairs : 0;
    Item it;
    it.job = i < n0 ? 0 : 1;
    const PairJob &j = prm.job[it.job];
    int x = i < n0 ? pair + i * pairs : prm.begin1[pair] + (i - n0);
    // rows run fastest where there are few row tiles (the tokens of a head product): concurrent
    // tiles then share the columns' operand
    const int tiles = j.tiles_m * j.tiles_n;
    it.split = x / tiles;
    x -= it.split * tiles;
    if (j.tiles_m <= j.tiles_n) {
        it.n = x / j.tiles_m;
        it.m = x - it.n * j.tiles_m;
    } else {
        it.m = x / j.tiles_n;
        it.n = x - it.m * j.tiles_n;
    }
    return it;
}
__device__ __forceinline__ int item_blocks(const PairJob &j, int split) { return min(j.kb_per, j.kb - split * j.kb_per); }

// parts of A and B in product p of 6: (0,2) (2,0) (1,1) (0,1) (1,0) (0,0); of 2: (1,0) (0,0)
__device__ __forceinline__ int part_a(int nprod, int p) { return nprod == 6 ? (0x021010 >> (4 * (5 - p))) & 15 : nprod - 1 - p; }
__device__ __forceinline__ int part_b(int nprod, int p) { return nprod == 6 ? (0x201100 >> (4 * (5 - p))) & 15 : 0; }

// ---------------------------------------------------------------- epilogues (one thread = one row)
struct Stats {
    float m, s;
};
// (max, sum of exp) of `v` of the row's 128 logits in this thread's registers
__device__ __forceinline__ Stats row_stats(float (&x)[4][32], int v)
{
    if (v < 128) {
#pragma unroll
        for (int j = 0; j < 128; ++j)
            if (j >= v) x[j >> 5][j & 31] = neg_inf();
    }
    float t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = x[0][j];
#pragma unroll
    for (int j = 8; j < 128; ++j) t[j & 7] = fmaxf(t[j & 7], x[j >> 5][j & 31]);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
#pragma unroll
        for (int j = 0; j < o; ++j) t[j] = fmaxf(t[j], t[j + o]);
    Stats a;
    a.m = t[0];
    const float ref = a.m == neg_inf() ? 0.f : a.m;
    // x - ref first: the largest term is then exactly 1 whatever the size of the logits
    const uint64_t neg2 = pack2(-ref, -ref), log2 = pack2(kLog2e, kLog2e);
    uint64_t s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = pack2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 128; j += 2) {
        float t0, t1;
        unpack2(mul2(add2(pack2(x[j >> 5][j & 31], x[j >> 5][(j & 31) + 1]), neg2), log2), t0, t1);
        s[(j >> 1) & 3] = add2(s[(j >> 1) & 3], pack2(ex2(t0), ex2(t1)));
    }
    float t0, t1;
    unpack2(add2(add2(s[0], s[1]), add2(s[2], s[3])), t0, t1);
    a.s = t0 + t1;
    return a;
}

// A warp's block of 32 rows x 32 columns, a row per thread, into its buffer, to be read so that eight lanes hold a row:
// staged(i) is columns 4 (lane % 8) .. + 3 of row 4 i + lane / 8.
__device__ __forceinline__ void to_stage(const float (&x)[32], float4 *stage, int lane)
{
#pragma unroll
    for (int c = 0; c < 8; ++c)
        stage[lane * 8 + (c ^ (lane & 7))] = make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
    __syncwarp();
}
__device__ __forceinline__ float4 &staged(float4 *stage, int i, int lane)
{
    const int r = 4 * i + (lane >> 3);
    return stage[r * 8 + ((lane & 7) ^ (r & 7))];
}
// four elements of a row
__device__ __forceinline__ void store4(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 x)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}
// The staged block where rows start anywhere or columns are missing: out[r * pitch] of the first `rows` rows, a lane per
// column (a store instruction is then one run of a row), lanes below `width`.
template <typename T>
__device__ __forceinline__ void store_any(T *out, int64_t pitch, const float4 *stage, int lane, int rows, int width)
{
    const float *s = reinterpret_cast<const float *>(stage);
#pragma unroll 4
    for (int r = 0; r < 32; ++r, out += pitch)
        if (r < rows && lane < width) out[0] = (T)s[r * 32 + (((lane >> 2) ^ (r & 7)) << 2) + (lane & 3)];
}
__device__ __forceinline__ float minus_bf16(float x) { return x - __bfloat162float(__float2bfloat16(x)); }

// CHUNKED: the whole row's columns in registers, added up over chunks of the contraction; else 32 columns at a time, straight
// from the one accumulator
template <int EPI, typename T, bool CHUNKED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
pair_kernel(const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_b0,
            const __grid_constant__ CUtensorMap map_a1, const __grid_constant__ CUtensorMap map_b1,
            const __grid_constant__ CUtensorMap map_out0, const __grid_constant__ CUtensorMap map_out1,
            const __grid_constant__ PairParams prm)
{
    extern __shared__ unsigned char smem_raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    PairControl *ctl = reinterpret_cast<PairControl *>(ring + kCtlOffset);
    pdl_trigger();   // a kernel launched behind this one may set itself up
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)cluster_rank();
    const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
    const int n_items = items_of_pair(prm, pair, pairs);
    const uint32_t limit = prm.spin_limit;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            bar_init(&ctl->full[s], 1);
            bar_init(&ctl->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(&ctl->acc_full[b], 1);
            bar_init(&ctl->acc_empty[b], 16);      // eight epilogue warps of each CTA
        }
        bar_init(&ctl->drain, 1);
        ctl->abort = 0;
        ctl->consumed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl->tmem_base)),
                     "r"((uint32_t)kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = ctl->tmem_base;
    // both CTAs have set up their barriers: copies and commits of one count on the other's
    cluster_arrive();
    cluster_wait();
    pdl_wait();      // launched behind a kernel of the same call: nothing of its results is touched before this

    long long issued = 0;
    if (warp == 0) {
        // ---------------- producer: lanes 0, 1 load the boxes of A, lanes 2, 3 those of B
        if (lane < 4 && !(prm.test_flags & PAIR_TEST_NO_LOADS)) {
            const bool is_b = lane >> 1;
            int s = 0;
            uint32_t par = 1;
            for (int i = 0; i < n_items; ++i) {
                const Item it = get_item(prm, pair, pairs, i);
                const PairJob &j = prm.job[it.job];
                const CUtensorMap *map = it.job ? (is_b ? &map_b1 : &map_a1) : (is_b ? &map_b0 : &map_a0);
                const bool across = is_b ? j.b_across : j.a_across;
                const int seg = is_b ? j.b_seg : j.a_seg;
                const int mn = (is_b ? it.n : it.m) * kPairTile + rank * 128 + (lane & 1) * 64;
                const int kb0 = it.split * j.kb_per, kbs = item_blocks(j, it.split);
                bool ok = true;
                for (int kc = 0, p = 0; kc < kbs && ok;) {        // chunk by chunk, product by product
                    const int off = seg * (is_b ? part_b(j.nprod, p) : part_a(j.nprod, p));
                    const int k_end = min(kc + j.kc, kbs);
                    for (int k = kc; k < k_end; ++k) {
                        ok = bar_wait(&ctl->empty[s], par, &ctl->abort, prm.status, limit);
                        if (!ok) break;
                        if (lane == 0 && rank == 0) bar_expect(&ctl->full[s], 2 * kStageBytes);
                        const int at = (kb0 + k) * kPairBlockK;
                        load_box(smem_addr(ring + s * kStageBytes) + lane * kBoxBytes, map, across ? mn + off : at + off,
                                 across ? at : mn, &ctl->full[s]);
                        ++issued;
                        if (++s == kStages) {
                            s = 0;
                            par ^= 1u;
                        }
                    }
                    if (++p == j.nprod) {
                        p = 0;
                        kc = k_end;
                    }
                }
                if (!ok) break;
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer: one thread of the even CTA, for both
        if (lane == 0 && rank == 0) {
            int s = 0;
            uint32_t par = 0;
            long long used = 0;
            uint32_t chunk = 0;
            bool ok = true;
            for (int i = 0; i < n_items && ok; ++i) {
                const Item it = get_item(prm, pair, pairs, i);
                const PairJob &j = prm.job[it.job];
                const bool aa = j.a_across, ba = j.b_across;
                // bf16 x bf16 -> fp32, M = N = 256
                const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)aa << 15) | ((uint32_t)ba << 16) |
                                       ((uint32_t)(kPairTile >> 3) << 17) | ((uint32_t)(kPairTile >> 4) << 24);
                // 16 further along K: 32 bytes inside the swizzle row, or two 8-deep groups
                const uint64_t a_step = (aa ? 2048 : 32) >> 4, b_step = (ba ? 2048 : 32) >> 4;
                const int kbs = item_blocks(j, it.split);
                for (int kc = 0; kc < kbs && ok; kc += j.kc, ++chunk) {
                    const int steps = j.nprod * min(j.kc, kbs - kc);
                    const int buf = (int)(chunk & 1u);
                    const uint32_t acc = tmem + (uint32_t)(buf * kPairTile);
                    ok = bar_wait(&ctl->acc_empty[buf], ((chunk >> 1) & 1u) ^ 1u, &ctl->abort, prm.status, limit);
                    if (!ok) break;
                    fence_after();
                    for (int k = 0; k < steps; ++k) {
                        ok = bar_wait(&ctl->full[s], par, &ctl->abort, prm.status, limit);
                        if (!ok) break;
                        fence_after();
                        const uint32_t a_addr = smem_addr(ring + s * kStageBytes);
                        const uint64_t da = tile_desc(a_addr, aa), db = tile_desc(a_addr + kHalfBytes, ba);
#pragma unroll
                        for (int q = 0; q < kPairBlockK / 16; ++q)
                            mma_pair(acc, da + q * a_step, db + q * b_step, idesc, (k | q) != 0 ? 1u : 0u);
                        commit_pair(&ctl->empty[s]);
                        ++used;
                        if (++s == kStages) {
                            s = 0;
                            par ^= 1u;
                        }
                    }
                    if (ok) commit_pair(&ctl->acc_full[buf]);
                }
            }
            ctl->consumed = used;
            if (!ok) commit_pair(&ctl->drain);
        }
    } else {
        // ---------------- epilogue: a row and 128 columns of the tile per thread
        const int quarter = warp & 3, half = (warp - kFirstEpilogueWarp) >> 2;
        float4 *stage = reinterpret_cast<float4 *>(ring + kOutOffset + (warp - kFirstEpilogueWarp) * kOutBytes);
        const int r_in = rank * 128 + quarter * 32 + lane;
        const uint32_t lane_base = tmem + (uint32_t)(half * 128) + ((uint32_t)(quarter * 32) << 16);
        uint32_t chunk = 0;
        bool ok = true;
        for (int i = 0; i < n_items && ok; ++i) {
            const Item it = get_item(prm, pair, pairs, i);
            const PairJob &j = prm.job[it.job];
            constexpr int kGroups = CHUNKED ? 4 : 1;
            float x[kGroups][32];
            const int kbs = item_blocks(j, it.split);
            uint32_t acc = 0;
            for (int kc = 0; kc < kbs; kc += j.kc, ++chunk) {
                const int buf = (int)(chunk & 1u);
                ok = bar_wait(&ctl->acc_full[buf], (chunk >> 1) & 1u, &ctl->abort, prm.status, limit);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                fence_after();
                acc = lane_base + (uint32_t)(buf * kPairTile);
                if constexpr (CHUNKED) {
                    if (kc == 0) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) tmem_read32(acc + 32 * q, x[q]);
                        tmem_wait();
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            float y[16];
                            tmem_read16(acc + 16 * q, y);
                            tmem_wait();
                            float *z = &x[q >> 1][16 * (q & 1)];
#pragma unroll
                            for (int e = 0; e < 16; e += 2)
                                unpack2(add2(pack2(z[e], z[e + 1]), pack2(y[e], y[e + 1])), z[e], z[e + 1]);
                        }
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_even(&ctl->acc_empty[buf]);
                }
            }
            if (!ok) break;
            auto columns = [&](int q) -> float(&)[32] {      // columns 32 q .. of the row
                if constexpr (CHUNKED) {
                    return x[q];
                } else {
                    tmem_read32(acc + 32 * q, x[0]);
                    tmem_wait();
                    return x[0];
                }
            };
            // 64 columns of bf16 (16 of two each), h = 0 or 1, as a box of 32 rows: written swizzled, so that no bank is met
            // twice, and on their way while the next ones are formed
            const CUtensorMap *map_out = it.job ? &map_out1 : &map_out0;
            auto put_box = [&](int h, const float(&line)[32], int c, int64_t r, int64_t cols) {
                if (lane == 0) stores_read();
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    stage[lane * 8 + (e ^ (lane & 7))] = make_float4(line[4 * e], line[4 * e + 1], line[4 * e + 2], line[4 * e + 3]);
                fence_stores();
                __syncwarp();
                if (lane == 0 && c + 64 * h < cols && r < j.rows) store_box(map_out, c + 64 * h, (int)r, stage);
            };
            const int64_t row = (int64_t)it.m * kPairTile + r_in;
            const bool live = row < j.rows;
            const int c0 = it.n * kPairTile + half * 128;
            const int width = min(128, j.cols - c0);              // columns that exist (not positive: none)
            if (EPI == PAIR_STATS) {
                Stats st = {0.f, 0.f};
                if constexpr (CHUNKED) st = row_stats(x, width);
                if (live) j.part[row * (2 * j.tiles_n) + 2 * it.n + half] = make_float2(st.m, st.s);
            } else if (EPI == PAIR_DLOGITS) {
                // D = g (exp(l - lse) - [v = target]); rows without a target are zero whatever they hold, and so are the
                // columns behind the last: a part of D is whole tiles wide
                const int t = live ? j.targets[row] : -1;
                const bool keep = t >= 0 && t < j.V;
                const float lse = keep ? j.lse[row] : 0.f, g = keep ? j.grad_loss[row] : 0.f;
                const int hot = keep ? t - j.v0 - c0 : -1;
                const int rows = (int)min((int64_t)32, j.rows - (row - lane)) - (lane >> 3);
                const int64_t step = 4 * j.dl_pitch;
                const int seg = j.dl_seg;
                __nv_bfloat16 *dst = j.dlogits + (row - lane + (lane >> 3)) * j.dl_pitch + c0 + (sizeof(T) == 2 ? 8 : 4) * (lane & 7);
                float line[32], rest[32];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float(&y)[32] = columns(q);
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float p = sizeof(T) == 4 ? expf(y[e] - lse) : ex2((y[e] - lse) * kLog2e);
                        y[e] = keep && 32 * q + e < width ? g * p : 0.f;
                    }
                    if (hot >= 32 * q && hot < 32 * q + 32) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (hot == 32 * q + e) y[e] -= g;
                    }
                    __syncwarp();
                    if constexpr (sizeof(T) == 2) {
                        // 64 columns of bf16 are a line of 128 bytes: two groups go out as one
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            line[16 * (q & 1) + e / 2] = __uint_as_float(pack_bf16(y[e], y[e + 1]));
                            rest[16 * (q & 1) + e / 2] = __uint_as_float(pack_bf16(minus_bf16(y[e]), minus_bf16(y[e + 1])));
                        }
                        if (q & 1) {
                            put_box(q >> 1, line, c0, row - lane, seg);
                            if (j.dl_parts == 2) put_box(q >> 1, rest, seg + c0, row - lane, 2 * (int64_t)seg);
                        }
                        continue;
                    }
                    to_stage(y, stage, lane);
                    __nv_bfloat16 *o = dst + 32 * q;
#pragma unroll 2
                    for (int i = 0; i < 8; ++i, o += step) {
                        if (4 * i < rows) {
                            float4 v = staged(stage, i, lane);
                            store4(o, v);
                            v = make_float4(minus_bf16(v.x), minus_bf16(v.y), minus_bf16(v.z), minus_bf16(v.w));
                            store4(o + seg, v);
                            v = make_float4(minus_bf16(v.x), minus_bf16(v.y), minus_bf16(v.z), minus_bf16(v.w));
                            store4(o + 2 * (int64_t)seg, v);
                        }
                    }
                    __syncwarp();
                }
            } else {
                // this lane's part of a block: columns 4 (lane % 8) .. + 3 of rows lane / 8, + 4, ...
                const int rows = (int)min((int64_t)32, j.rows - (row - lane)) - (lane >> 3);
                const int64_t r0 = row - lane + (lane >> 3);
                const int cl = c0 + 4 * (lane & 7);
                const bool to_out = j.out != nullptr, add = j.add_acc != 0;
                const int64_t acc_step = 4 * j.acc_pitch, out_step = 4 * j.out_pitch;
                float *a = j.acc + (int64_t)it.split * j.acc_stride + r0 * j.acc_pitch + cl;    // used where there is an acc
                T *o = static_cast<T *>(j.out) + r0 * j.out_pitch + cl;                         // used where there is an out
                // four elements of the caller's type are stored at once where every row allows it
                const uintptr_t where = reinterpret_cast<uintptr_t>(j.out) | (uintptr_t)(j.out_pitch * (int64_t)sizeof(T));
                const bool vec = (where & (4 * sizeof(T) - 1)) == 0;
                if (sizeof(T) == 2 && j.boxes) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float line[32];
#pragma unroll
                        for (int q = 2 * h; q < 2 * h + 2; ++q) {
                            const float(&y)[32] = columns(q);
#pragma unroll
                            for (int e = 0; e < 32; e += 2) line[16 * (q & 1) + e / 2] = __uint_as_float(pack_bf16(y[e], y[e + 1]));
                        }
                        put_box(h, line, c0, row - lane, j.cols);
                    }
                } else
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (32 * q >= width) break;
                    to_stage(columns(q), stage, lane);
                    if (add) {                   // acc's pitch covers whole groups of 32
                        const float *p = a + 32 * q;
#pragma unroll 4
                        for (int i = 0; i < 8; ++i, p += acc_step) {
                            if (4 * i < rows) {
                                const float4 y = *reinterpret_cast<const float4 *>(p);
                                float4 &v = staged(stage, i, lane);
                                v = make_float4(v.x + y.x, v.y + y.y, v.z + y.z, v.w + y.w);
                            }
                        }
                        __syncwarp();
                    }
                    if (!to_out) {
                        float *p = a + 32 * q;
#pragma unroll 4
                        for (int i = 0; i < 8; ++i, p += acc_step)
                            if (4 * i < rows) store4(p, staged(stage, i, lane));
                    } else if (vec && width - 32 * q >= 32) {
                        T *p = o + 32 * q;
#pragma unroll 4
                        for (int i = 0; i < 8; ++i, p += out_step)
                            if (4 * i < rows) store4(p, staged(stage, i, lane));
                    } else {
                        store_any(static_cast<T *>(j.out) + (row - lane) * j.out_pitch + c0 + 32 * q + lane, j.out_pitch, stage, lane,
                                  rows + (lane >> 3), width - 32 * q);
                    }
                    __syncwarp();
                }
            }
            if constexpr (!CHUNKED) {
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_even(&ctl->acc_empty[(chunk - 1u) & 1u]);
            }
            __syncwarp();
        }
        if (sizeof(T) == 2 && lane == 0) stores_done();
    }

    // ---------------- way out
    __syncwarp();
    fence_before();
    __syncthreads();
    if (*reinterpret_cast<volatile int *>(&ctl->abort)) {
        // copies and products in flight get a bounded time to end
        if (warp == 0 && lane == 0 && rank == 0) {
            const long long used = *reinterpret_cast<volatile long long *>(&ctl->consumed);
            for (long long st = used; st < issued; ++st)
                bar_wait_quiet(&ctl->full[st % kStages], (uint32_t)(st / kStages) & 1u, 1u << 20);
        }
        if (warp == 1 && lane == 0 && rank == 0) bar_wait_quiet(&ctl->drain, 0, 1u << 20);
        __syncthreads();
    }
    cluster_arrive();
    cluster_wait();
    if (warp == 1) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kTmemCols)
                     : "memory");
    }
}

// ---------------------------------------------------------------- host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn()
{
    static const EncodeTiledFn fn = [] {   // initialised once, thread-safe
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            return reinterpret_cast<EncodeTiledFn>(p);
        return static_cast<EncodeTiledFn>(nullptr);
    }();
    return fn;
}

// boxes of 64 x `rows` elements, 128-byte swizzle, zeros outside
bool make_map(CUtensorMap *map, const PairOperand &t, int rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)t.cols, (cuuint64_t)t.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)t.pitch * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)rows};
    const cuuint32_t elem[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(t.base), dims, strides, box, elem,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int EPI, typename T, bool CHUNKED>
cudaError_t launch(const CUtensorMap (&maps)[6], const PairParams &prm, int ctas, int dev, bool behind, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];   // host threads may race to set it: all of them store `true`
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(pair_kernel<EPI, T, CHUNKED>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)kPairSmem);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = behind ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, pair_kernel<EPI, T, CHUNKED>, maps[0], maps[1], maps[2], maps[3], maps[4], maps[5], prm);
}

}  // namespace

// set for the calling host thread by the test hook spr_test_pair_kernels
static thread_local int t_test_flags = 0;
static thread_local unsigned t_spin_limit = 0;

cudaError_t launch_pair(PairEpilogue epi, bool f32, PairParams &prm, int njobs, const PairOperand *a,
                        const PairOperand *b, bool behind, cudaStream_t st)
{
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    CUtensorMap maps[6];
    for (int i = 0; i < njobs; ++i) {
        if (!make_map(&maps[2 * i], a[i], 64) || !make_map(&maps[2 * i + 1], b[i], 64)) return cudaErrorInvalidValue;
        // bf16 results go out as boxes where nothing is added to them and their rows are whole 16-byte vectors
        PairJob &j = prm.job[i];
        PairOperand out = {nullptr, j.rows, 0, 0};
        if (!f32 && epi == PAIR_DLOGITS) out = PairOperand{j.dlogits, j.rows, (int64_t)j.dl_parts * j.dl_seg, j.dl_pitch};
        if (!f32 && epi == PAIR_OUT && !j.add_acc && j.out_pitch % 8 == 0) out = PairOperand{j.out, j.rows, j.cols, j.out_pitch};
        j.boxes = out.base != nullptr;
        maps[4 + i] = maps[0];
        if (j.boxes && !make_map(&maps[4 + i], out, 32)) return cudaErrorInvalidValue;
    }
    if (njobs == 1) {       // not used
        maps[2] = maps[0];
        maps[3] = maps[1];
        maps[5] = maps[0];
    }
    int pairs = sms / 2 < kMaxPairs ? sms / 2 : kMaxPairs;
    int64_t total = 0;
    double work = 0.0, len[2] = {0.0, 0.0};
    bool chunked = epi == PAIR_STATS || f32;
    for (int i = 0; i < 2; ++i) {
        prm.items[i] = 0;
        if (i >= njobs) continue;
        const PairJob &j = prm.job[i];
        const int64_t n = (int64_t)j.tiles_m * j.tiles_n * j.splits;
        if (n > 0x3fffffff) return cudaErrorInvalidValue;
        prm.items[i] = (int)n;
        total += n;
        chunked = chunked || j.kc < j.kb_per;
        len[i] = (double)j.nprod * j.kb_per + 2.0;      // in blocks, with about two blocks' time of turn-around
        work += len[i] * (double)n;
    }
    if (total < pairs) pairs = (int)total;
    if (prm.items[1]) {
        // job 1 fills every pair up to the same share of the work
        const double share = work / pairs;
        double owed = 0.0;
        int next = 0;
        for (int p = 0; p < pairs; ++p) {
            const int n0 = p < prm.items[0] ? (prm.items[0] - p + pairs - 1) / pairs : 0;
            owed += share - n0 * len[0];
            int n1 = owed > 0.0 ? (int)(owed / len[1] + 0.5) : 0;
            if (p == pairs - 1 || n1 > prm.items[1] - next) n1 = prm.items[1] - next;
            prm.begin1[p] = next;
            prm.count1[p] = n1;
            next += n1;
            owed -= n1 * len[1];
        }
    }
    prm.spin_limit = t_spin_limit ? t_spin_limit : kSpinLimit;
    prm.test_flags = t_test_flags;
    switch (epi) {
    case PAIR_STATS: return launch<PAIR_STATS, float, true>(maps, prm, 2 * pairs, dev, behind, st);      // the same for both types
    case PAIR_DLOGITS:
        return f32       ? launch<PAIR_DLOGITS, float, true>(maps, prm, 2 * pairs, dev, behind, st)
               : chunked ? launch<PAIR_DLOGITS, __nv_bfloat16, true>(maps, prm, 2 * pairs, dev, behind, st)
                         : launch<PAIR_DLOGITS, __nv_bfloat16, false>(maps, prm, 2 * pairs, dev, behind, st);
    default:
        return f32       ? launch<PAIR_OUT, float, true>(maps, prm, 2 * pairs, dev, behind, st)
               : chunked ? launch<PAIR_OUT, __nv_bfloat16, true>(maps, prm, 2 * pairs, dev, behind, st)
                         : launch<PAIR_OUT, __nv_bfloat16, false>(maps, prm, 2 * pairs, dev, behind, st);
    }
}

}  // namespace spr

extern "C" void spr_test_pair_kernels(int flags, unsigned spin_limit)
{
    spr::t_test_flags = flags & spr::PAIR_TEST_NO_LOADS;
    spr::t_spin_limit = spin_limit;
}
