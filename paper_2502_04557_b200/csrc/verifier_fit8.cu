// One Adam step of the linear verifier on hidden states kept in 8 bits (hidden_pack.cu):
//   z_i = b + sum_j w_j q_ij 2^e_ij,  r = sigma(z) - y,  grad_j = sum_i r_i 2^e_ij q_ij
// Floor: the packed rows once, 1.03 d bytes a sample (2^18 rows of 2048: 554 MB, 86 us; measured 113 us).  At that
// rate an SM takes in some 24 elements a clock, and on the CUDA cores it is instructions that bound the pass: a byte
// turned into a float costs as much as the two products it goes into (measured: 244 us that way, 180 us with the
// dot products in dp4a).  So both sums are integer products on the tensor cores (mma.m16n8k32, s8 x s8 -> s32):
//   - a block of 32 columns shares its exponent within a row, so a block is one step of the contraction of
//     the dot products.  A weight is written relative to the largest of its block, in six balanced signed digits
//     (six_digits(): 46 bits), six of the eight columns of the second operand.  What is left per block and row is one
//     conversion and the row's scale.
//   - for the gradient the contraction runs over the rows of a tile: r_i 2^e_ij of the block, written relative to the
//     largest of the tile in six digits, too, times the bytes, which ldmatrix transposes.  The integer sums are
//     exact; per tile and column one conversion for every two digits, and an fp32 sum over tiles.
// Six digits, because the largest of a group need not have a part in a sum beside it: a state whose one huge column sets the
// exponent of its block has bytes of zero in the other 31, and a large weight may meet a zero.  What is left out is 2^-46 of
// the largest, so the other terms keep their 24 bits up to 2^22 below it (with three digits they lost a bit for every factor of
// two).  The products work on eight columns whatever these hold; the digits themselves cost 110 -> 113 us at 2^18 x 2048, 67 ->
// 69 us at 2^19 x 512 and 157 -> 172 us at 2^17 x 4096.
// A CTA takes tiles of consecutive rows through a ring in shared memory.  A warp has 128 columns (256 above 2048) of
// every tile: it fetches them itself, by TMA in boxes of 128 bytes by all rows with the 128-byte swizzle, which keeps
// ldmatrix free of bank conflicts; it forms its part of the tile's dot products, then the sums of its columns of
// the tile before, and asks for the next columns at once.  One more warp turns dot products into residuals in the
// meantime and fetches the exponent bytes, which all warps read.  Nothing but these residuals joins the warps: with a
// barrier per tile and the tile fetched as one the step took 158 us at 2^18 x 2048, with the residuals by a warp of
// their own 132 us, with every warp its own fetches 111 us, now 113 us (4.9 TB/s).  What is left to the floor is the
// latency of a tile: two of the three that fit are in use, and the third arrives while they are worked on.  Up to 1024
// columns shared memory holds several CTAs, which fill each other's gaps (2^18 x 1024: 113 us with one, 65 us; 2^19 x 512:
// 198, 69 us).  Above 2048 columns a tile has 16 rows, and what is done once per tile is done twice as often: 2^17 x 4096, the
// same bytes but for the exponents, takes 172 us (3.2 TB/s).  Below some 10^4 rows the step is two launches and one trip to memory, 8.5 us.
// Tiles are dealt in a fixed pattern and all sums have a fixed order: a step is reproducible bit for bit.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "host_util.h"
#include "launch.h"
#include "vocab_common.cuh"

namespace spr {

namespace {

constexpr int kMaxTiles = 8;             // tiles of the ring, and twice as many of their exponent bytes
constexpr int kAhead = 2;                // tiles on their way into L2 behind those of the ring

__device__ __forceinline__ uint32_t fit_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool fit_wait(uint64_t *bar, uint32_t parity, uint32_t limit)
{
    for (uint32_t n = 0; n < limit; ++n) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(fit_addr(bar)), "r"(parity)
            : "memory");
        if (done) return true;
    }
    return false;
}

__device__ __forceinline__ void fit_init(uint64_t *bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(fit_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void fit_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
// what the warp's lanes did before is there for whom the barrier lets through
__device__ __forceinline__ void fit_arrive(uint64_t *bar, int lane)
{
    __syncwarp();
    if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(fit_addr(bar)) : "memory");
}

__device__ __forceinline__ void fit_expect(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(fit_addr(bar)), "r"(bytes) : "memory");
}

__device__ __forceinline__ void fetch_box(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
        "r"(c0), "r"(c1), "r"(fit_addr(bar))
        : "memory");
}

// the same box on its way into L2 only
__device__ __forceinline__ void prefetch_box(const CUtensorMap *map, int c0, int c1)
{
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(c0), "r"(c1) : "memory");
}

// 2^e of an exponent byte.  -128 marks a block that held an infinity or NaN, with bytes of zero: the same shift
// makes that minus infinity, and its product with a zero sum NaN.
__device__ __forceinline__ float block_scale(uint32_t word, int k)      // byte k of the word
{
    return __int_as_float(((int)(word << (24 - 8 * k)) >> 24) * (1 << 23) + 127 * (1 << 23));
}
// N exponent bytes, 4 or 8, from a shared address that is a multiple of N
template <int N>
__device__ __forceinline__ void load_exponents(uint32_t (&x)[N / 4], uint32_t addr)
{
    static_assert(N == 4 || N == 8, "exponent bytes");
    if constexpr (N == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x[0]) : "r"(addr));
    else asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(addr));
}
// A number in units of its group as six balanced digits of a byte: x = 256^2 d0 + 256 d1 + d2 + 2^-23 (256^2 d3 + 256 d4 + d5),
// |x| <= 8355711.  hi is x rounded to the unit, lo the rest of it in units of 2^-23, so |lo| <= 2^22; both are exact, and so is
// every number of fp32 down to 2^-22 of the largest that the group can hold.  The digits stand in the order d0 .. d5, 0, 0.
__device__ __forceinline__ uint32_t digits(int v) { return ((uint32_t)v + 0x808080u) ^ 0x808080u; }      // bytes 2, 1, 0
__device__ __forceinline__ uint2 six_digits(int hi, int lo)
{
    const uint32_t h = digits(hi), l = digits(lo);
    return make_uint2(__byte_perm(h, l, 0x6012), __byte_perm(l, 0u, 0x4401));
}
// An operand of the products is put together in shared memory: a row of 16 bytes for each number of the contraction, the digits
// of two groups side by side.  Read transposed, eight of the columns are then a product's second operand: column n is digit n,
// the seventh and eighth are zero.
__device__ __forceinline__ void put_digits(uint32_t row, uint2 a, uint2 b)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(row), "r"(a.x), "r"(a.y), "r"(b.x), "r"(b.y) : "memory");
}
__device__ __forceinline__ void put_digits(uint32_t half_row, uint2 a)
{
    asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(half_row), "r"(a.x), "r"(a.y) : "memory");
}
// 32 numbers of two groups; row: that of number `lane`
__device__ __forceinline__ void get_digits(uint32_t row, uint2 &a, uint2 &b)
{
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];"
                 : "=r"(a.x), "=r"(b.x), "=r"(a.y), "=r"(b.y)
                 : "r"(row)
                 : "memory");
}
// 16 numbers of two groups; row: that of number `lane` % 16
__device__ __forceinline__ void get_digits_k16(uint32_t row, uint32_t &a, uint32_t &b)
{
    asm volatile("ldmatrix.sync.aligned.m16n16.x1.trans.shared.b8 {%0,%1}, [%2];" : "=r"(a), "=r"(b) : "r"(row) : "memory");
}

__device__ __forceinline__ void mma_s8(int (&c)[4], const uint32_t (&a)[4], uint2 b)      // c = A (16 x 32) B (32 x 8)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y), "r"(0));
}
__device__ __forceinline__ void mma_s8_k16(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t b)   // c = A (16 x 16) B (16 x 8)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%7,%7,%7,%7};"
                 : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3])
                 : "r"(a0), "r"(a1), "r"(b), "r"(0));
}

// Scaled residuals of a tile relative to the largest of them (its bits): less than 2^22 units of 2^E
__device__ __forceinline__ int residual_exponent(uint32_t top) { return max((int)(top >> 23), 27) - 148; }
// v 2^-E + 1.5 2^23 rounds to the unit, and the integer stands in the low bits of the sum; the rest is exact
__device__ __forceinline__ uint2 residual_digits(float v, int E)
{
    const float scale = __int_as_float((127 - E) << 23), t = fmaf(v, scale, 12582912.f);
    const float rest = fmaf(v, scale, 12582912.f - t);
    return six_digits((int)(__float_as_uint(t) - 0x4b400000u), (int)(__float_as_uint(fmaf(rest, 8388608.f, 12582912.f)) - 0x4b400000u));
}

// A tile in shared memory: boxes of 128 bytes x T rows, one after the other; inside, 16-byte units are swizzled.
// Byte c of row r:
template <int T>
__device__ __forceinline__ uint32_t tile_at(int r, int c)
{
    return (uint32_t)((c >> 7) * (T * 128) + r * 128 + (((c >> 4) ^ r) & 7) * 16 + (c & 15));
}
// Unit k past a unit whose own index is a multiple of the units asked for: the swizzle's exclusive or is linear in it.
__device__ __forceinline__ uint32_t unit_at(uint32_t base, int k) { return base ^ (uint32_t)(k << 4); }
// Behind the boxes of the d bytes a box of the rows' exponent bytes: 16, 32, 64 or 128 bytes x T rows, swizzled in as many bytes.
__host__ __device__ constexpr int tile_boxes(int d) { return (d + 127) / 128; }
__host__ __device__ constexpr int exponent_width(int d) { return d <= 512 ? 16 : d <= 1024 ? 32 : d <= 2048 ? 64 : 128; }
// a tile's share of the ring
__host__ __device__ constexpr int tile_share(int d, int rows) { return rows * (tile_boxes(d) * 128 + 2 * exponent_width(d)); }
__device__ __forceinline__ uint32_t exponent_at(int width, int r, int b)
{
    return (uint32_t)(r * width + (((b >> 4) ^ ((r * width) >> 7)) & (width / 16 - 1)) * 16 + (b & 15));
}

// NB: blocks of 32 columns per warp; T: rows per tile (16 or 32); W: warps that have columns; C: CTAs on an SM
template <int NB, int T, int W>
struct Fit8 {
    static constexpr int kThreads = (W + 1) * 32;
    // shared memory behind the ring: digits of numbers that a warp puts into operands, two blocks' at a time; units of the
    // weights, parts of the dot products, residuals, barriers (a warp's columns of a tile there, exponents there, exponents
    // done with, dot products there, residuals there)
    static constexpr int kDigits = 0, kDigitBytes = 32 * 16, kUnit = kDigits + W * kDigitBytes, kZpart = kUnit + W * NB * 4;
    static constexpr int kResidual = kZpart + 2 * W * T * 4, kBars = kResidual + 2 * 32 * 4;
    static constexpr int kBytes = kBars + (kMaxTiles * W + 4 * kMaxTiles + 4) * 8;
    static constexpr int kBoxes = NB / 4;      // a warp's columns are as many boxes
    static_assert(NB % 4 == 0 && kDigits % 16 == 0 && kUnit % 4 == 0 && kBars % 8 == 0, "alignment");
};

template <int NB, int T, int W, int C>
__global__ void __launch_bounds__((W + 1) * 32, C) train8_kernel(const TrainParams prm, const __grid_constant__ CUtensorMap map,
                                                                     const __grid_constant__ CUtensorMap emap, int ring_tiles)
{
    using F = Fit8<NB, T, W>;
    constexpr int kRowGroups = T / 16, kWords = NB / 4;
    extern __shared__ __align__(1024) unsigned char smem[];        // the ring comes first: swizzled boxes repeat every 1024 bytes
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int d = prm.d, blocks = (d + 31) / 32, workers = (blocks + NB - 1) / NB;
    const int boxes = tile_boxes(d), ewidth = exponent_width(d), tile_bytes = boxes * T * 128, exp_bytes = T * ewidth;
    const int ring_exps = 2 * ring_tiles;
    const uint32_t ring = fit_addr(smem), exps = ring + (uint32_t)(ring_tiles * tile_bytes);
    unsigned char *tables = smem + ring_tiles * tile_bytes + ring_exps * exp_bytes;
    float *unit = reinterpret_cast<float *>(tables + F::kUnit);
    float(*zpart)[W][T] = reinterpret_cast<float(*)[W][T]>(tables + F::kZpart);
    float(*residual)[32] = reinterpret_cast<float(*)[32]>(tables + F::kResidual);
    uint64_t *there = reinterpret_cast<uint64_t *>(tables + F::kBars), *ethere = there + kMaxTiles * W, *edone = ethere + 2 * kMaxTiles;
    uint64_t *dots = edone + 2 * kMaxTiles, *resid = dots + 2;
    pdl_trigger();

    // this CTA's tiles: blockIdx.x, + gridDim.x, ...; only the last tile of the data can be short
    const int N = (int)prm.N;
    const int all = (N + T - 1) / T;
    const int n = (int)blockIdx.x < all ? (all - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
    const int row_step = (int)gridDim.x * T;
    float *out = prm.part + (int64_t)blockIdx.x * (d + 2);
    bool ok = true;
    const bool feed = !(prm.test_flags & TRAIN_TEST_NO_FETCH);
    int row0 = (int)blockIdx.x * T, asked = 0;             // first row of the tile at hand; tiles asked for
    if (warp == W) {
        // ---- the warp that fetches exponent bytes and turns dot products into residuals, a row per lane
        auto fetch = [&](int slot, int row) {              // rows and bytes that do not exist arrive as zeros
            if (lane == 0) {
                fit_expect(&ethere[slot], (uint32_t)exp_bytes);
                fetch_box(exps + (uint32_t)(slot * exp_bytes), &emap, d, row, &ethere[slot]);
            }
        };
        if (lane == 0) {                                   // (the other barriers: below)
            for (int s = 0; s < ring_exps; ++s) {
                fit_init(&ethere[s], 1);
                fit_init(&edone[s], workers);
            }
            for (int s = 0; s < 2; ++s) {
                fit_init(&dots[s], workers);
                fit_init(&resid[s], 1);
            }
            fit_init_fence();
        }
        const float bias = prm.theta[d];
        for (; feed && asked < ring_exps && asked < n; ++asked) fetch(asked, row0 + asked * row_step);
        // labels two tiles ahead and as the bytes they are: a label fetched when it is wanted would cost a trip to memory
        auto tile_label = [&](int64_t row) -> uint32_t { return prm.labels[lane < T && row + lane < prm.N ? row + lane : 0]; };
        uint32_t y_raw[2] = {tile_label(row0), tile_label((int64_t)row0 + row_step)};
        double acc_b = 0.0, acc_loss = 0.0;
        int slot = 0;                              // of tile k - 1
        uint32_t parity = 0;
        __syncthreads();                           // the barriers are set up, and the weights' digits there
        for (int k = 0; k < n; ++k) {
            const float y = (float)y_raw[0];
            y_raw[0] = y_raw[1];
            y_raw[1] = tile_label((int64_t)row0 + 2 * (int64_t)row_step);
            ok = __all_sync(0xffffffffu, fit_wait(&dots[k & 1], (uint32_t)(k >> 1) & 1u, prm.spin_limit));
            if (!ok) break;
            float z = bias;
#pragma unroll
            for (int s = 0; s < W; ++s) z += s < workers ? zpart[k & 1][s][lane & (T - 1)] : 0.f;
            const bool live = lane < T && row0 + lane < N;
            const float r = live ? 1.f / (1.f + expf(-z)) - y : 0.f;
            residual[k & 1][lane] = r;
            fit_arrive(&resid[k & 1], lane);
            if (live) {
                acc_b += (double)r;
                acc_loss += (double)(fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))) - y * z);
            }
            if (k > 0) {
                if (asked < n) {
                    ok = __all_sync(0xffffffffu, fit_wait(&edone[slot], parity, prm.spin_limit));
                    if (!ok) break;
                    if (feed) fetch(slot, row0 + (ring_exps - 1) * row_step);
                    ++asked;
                }
                if (++slot == ring_exps) {
                    slot = 0;
                    parity ^= 1u;
                }
            }
            row0 += row_step;
        }
        if (!ok) {
            // A wait ran out: report it, then give the copies still on their way the same bounded time to land
            // before the CTA's shared memory goes away.
            if (lane == 0) raise_timeout(prm.status);
            for (int i = max(0, asked - ring_exps); feed && i < asked; ++i)
                fit_wait(&ethere[i % ring_exps], (uint32_t)(i / ring_exps) & 1u, prm.spin_limit);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            acc_b += __shfl_xor_sync(0xffffffffu, acc_b, o);
            acc_loss += __shfl_xor_sync(0xffffffffu, acc_loss, o);
        }
        if (lane == 0) {
            out[d] = (float)acc_b;
            out[d + 1] = (float)acc_loss;
        }
        __syncthreads();                           // no warp is at the tiles any more
        return;
    }

    // ---- the warps that have columns: each fetches its own, and asks for the next as soon as it is done with a tile
    const int b0 = warp * NB, nb = min(NB, blocks - b0), box0 = warp * F::kBoxes, nbox = min(F::kBoxes, boxes - box0);
    uint64_t *mine = there + warp * kMaxTiles;
    auto fetch = [&](int slot, int row) {                  // rows and bytes that do not exist arrive as zeros
        fit_expect(&mine[slot], (uint32_t)(nbox * T * 128));
        for (int b = 0; b < nbox; ++b)
            fetch_box(ring + (uint32_t)(slot * tile_bytes + (box0 + b) * T * 128), &map, (box0 + b) * 128, row, &mine[slot]);
    };
    // Three tiles of 2048 columns are all that shared memory holds, and two of them are in use: what comes after the
    // next tile is asked for as far as L2, so that memory always has kAhead tiles to bring.
    auto prefetch = [&](int row) {
        for (int b = 0; b < nbox; ++b) prefetch_box(&map, (box0 + b) * 128, row);
    };
    if (nb > 0 && lane == 0) {
        for (int s = 0; s < ring_tiles; ++s) fit_init(&mine[s], 1);
        fit_init_fence();
        for (int k = 0; feed && k < ring_tiles && k < n; ++k) fetch(k, row0 + k * row_step);
        for (int k = ring_tiles; feed && k < ring_tiles + kAhead && k < n; ++k) prefetch(row0 + k * row_step);
    }
    asked = min(ring_tiles, n);

    // This warp's weights, block by block, as operands in registers.
    const uint32_t dig = fit_addr(tables + F::kDigits) + (uint32_t)(warp * F::kDigitBytes), dig_row = dig + (uint32_t)(lane * 16);
    uint2 wdig[NB];
#pragma unroll
    for (int i = 0; i < NB; i += 2) {
        uint2 two[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int b = b0 + i + k, c = b * 32 + lane;
            const float w = c < d ? prm.theta[c] : 0.f;
            const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(w) & 0x7fffffffu);
            // unit 2^E with |w| <= 8355711 units (three digits reach that), at least 2^-122
            int E = max((int)(top >> 23) - 127, -100) - 22;
            if (rintf(ldexpf(__uint_as_float(top), -E)) > 8355711.f) ++E;
            const bool finite = top < 0x7f800000u;         // a weight that is not finite shows in every sum
            const float x = finite ? ldexpf(w, -E) : 0.f, hi = rintf(x);
            two[k] = six_digits(__float2int_rn(hi), __float2int_rn((x - hi) * 8388608.f));
            if (lane == 0) unit[b] = finite ? ldexpf(1.f, E) : __int_as_float(0x7fc00000);
        }
        __syncwarp();                          // what stood there is read
        put_digits(dig_row, two[0], two[1]);
        __syncwarp();
        get_digits(dig_row, wdig[i], wdig[i + 1]);
    }

    // A lane's part of a product's result: columns 2 (lane % 4) and + 1, hence d0 and d1, d2 and d3, d4 and d5, or nothing.
    // The integers 256 d0 + d1, 128 d2 + d3 and 256 d4 + d5 are added up apart and weighted at the very end.
    const int m0 = (lane & 3) == 1 ? 128 : 256;
    const float weight = (lane & 3) == 0 ? 256.f : (lane & 3) == 1 ? 1.f / 128.f : (lane & 3) == 2 ? 1.f / 8388608.f : 0.f;
    // blocks b0 .. b0 + NB - 1 are this warp's: dot products by 16 rows at a time, columns with a row per lane
    const uint32_t a1 = tile_at<T>((lane & 7) + ((lane >> 3) & 1) * 8, b0 * 32 + (lane >> 4) * 16);      // ldmatrix of 16 x 32
    const uint32_t e1 = exponent_at(ewidth, lane >> 2, b0);         // rows lane / 4 and, 8 * ewidth on, + 8
    const int my_row = lane & (T - 1);
    const uint32_t a2 = tile_at<T>(my_row, b0 * 32), e2 = exponent_at(ewidth, my_row, b0);
    float grad[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) grad[i][e] = 0.f;
    __syncthreads();                           // the barriers are set up, and the weights' digits there

    // Dot products of tile k, then columns of tile k - 1, whose residuals came in the meantime.  zpart and residual have two
    // halves: a warp is at tile k + 2 only once it has the residuals of tile k, hence when zpart's half is read; and
    // residual's half is written when every warp has handed in tile k + 2, behind the columns of tile k.
    int slot = 0, before = 0;                  // of tile k, of tile k - 1
    uint32_t parity = 0, xnow = exps, xbefore = exps;          // exponent bytes of tile k, of tile k - 1
    int eslot = 0, ebefore = 0;
    uint32_t eparity = 0;
    for (int k = 0; k <= n && nb > 0; ++k) {
        const uint32_t now = ring + (uint32_t)(slot * tile_bytes);
        if (k < n) {
            ok = fit_wait(&ethere[eslot], eparity, prm.spin_limit);
            ok = __all_sync(0xffffffffu, ok && fit_wait(&mine[slot], parity, prm.spin_limit));
            if (!ok) break;
            float z[2 * kRowGroups];
            uint32_t x1[2 * kRowGroups][kWords];
#pragma unroll
            for (int g = 0; g < 2 * kRowGroups; ++g) {
                z[g] = 0.f;
                load_exponents<NB>(x1[g], xnow + e1 + (uint32_t)(g * 8 * ewidth));
            }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                if (i < nb) {
                    const float u = unit[b0 + i];
#pragma unroll
                    for (int g = 0; g < kRowGroups; ++g) {
                        uint32_t a[4];
                        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                                     : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
                                     : "r"(unit_at(now + a1 + (uint32_t)(g * 2048 + (i / 4) * (T * 128)), 2 * (i & 3))));
                        int c[4];
                        mma_s8(c, a, wdig[i]);
                        z[2 * g] = fmaf((float)(c[0] * m0 + c[1]) * u, block_scale(x1[2 * g][i / 4], i & 3), z[2 * g]);
                        z[2 * g + 1] = fmaf((float)(c[2] * m0 + c[3]) * u, block_scale(x1[2 * g + 1][i / 4], i & 3), z[2 * g + 1]);
                    }
                }
            }
#pragma unroll
            for (int g = 0; g < 2 * kRowGroups; ++g) {
                z[g] *= weight;
                z[g] += __shfl_xor_sync(0xffffffffu, z[g], 1);
                z[g] += __shfl_xor_sync(0xffffffffu, z[g], 2);
                if ((lane & 3) == 0) zpart[k & 1][warp][g * 8 + (lane >> 2)] = z[g];
            }
            fit_arrive(&dots[k & 1], lane);
        }
        if (k > 0) {
            // ---- columns of this warp's blocks in tile k - 1
            const uint32_t tile = ring + (uint32_t)(before * tile_bytes);
            ok = __all_sync(0xffffffffu, fit_wait(&resid[(k - 1) & 1], (uint32_t)((k - 1) >> 1) & 1u, prm.spin_limit));
            if (!ok) break;
            const float r = residual[(k - 1) & 1][my_row];
            const float show = __any_sync(0xffffffffu, r != r) ? __int_as_float(0x7fc00000) : 1.f;    // NaN has no digits
            uint32_t x[kWords];
            load_exponents<NB>(x, xbefore + e2);
            if (T == 16)
#pragma unroll
                for (int w = 0; w < kWords; ++w) x[w] >>= (lane >> 4) * 8;
#pragma unroll
            for (int i0 = 0; i0 < NB; i0 += 2) {
                float scale[2];
                uint2 bd[2];
                __syncwarp();                      // the digits that stood there are read
                // a row that does not exist has r = 0, a block that does not exist is not read below
                if constexpr (T == 32) {
                    uint2 two[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float v = r != 0.f ? r * block_scale(x[(i0 + i) / 4], (i0 + i) & 3) : 0.f;
                        const int E = residual_exponent(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
                        two[i] = residual_digits(v, E);
                        scale[i] = __int_as_float((E + 127) << 23) * show;
                    }
                    put_digits(dig_row, two[0], two[1]);
                    __syncwarp();
                    get_digits(dig_row, bd[0], bd[1]);
                } else {
                    // 16 rows: two blocks at a time, one by each half of the warp
                    const float v = r != 0.f ? r * block_scale(x[i0 / 4], i0 & 3) : 0.f;
                    const uint32_t size = __float_as_uint(v) & 0x7fffffffu;
                    const int Ea = residual_exponent(__reduce_max_sync(0xffffffffu, lane < 16 ? size : 0u));
                    const int Eb = residual_exponent(__reduce_max_sync(0xffffffffu, lane < 16 ? 0u : size));
                    scale[0] = __int_as_float((Ea + 127) << 23) * show;
                    scale[1] = __int_as_float((Eb + 127) << 23) * show;
                    put_digits(dig + (uint32_t)((lane & 15) * 16 + (lane >> 4) * 8), residual_digits(v, lane < 16 ? Ea : Eb));
                    __syncwarp();
                    get_digits_k16(dig + (uint32_t)((lane & 15) * 16), bd[0].x, bd[1].x);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (i0 + i < nb) {
                        float *g = grad[i0 + i];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // a last block of 16 reads on, into what follows in the row
                            const uint32_t at = unit_at(tile + a2 + (uint32_t)((i0 + i) / 4 * (T * 128)), 2 * ((i0 + i) & 3) + h);
                            int c[4];
                            if constexpr (T == 32) {
                                uint32_t a[4];
                                asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];"
                                             : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
                                             : "r"(at));
                                mma_s8(c, a, bd[i]);
                            } else {
                                uint32_t a0, a4;
                                asm volatile("ldmatrix.sync.aligned.m16n16.x1.trans.shared.b8 {%0,%1}, [%2];"
                                             : "=r"(a0), "=r"(a4)
                                             : "r"(at));
                                mma_s8_k16(c, a0, a4, bd[i].x);
                            }
                            g[2 * h] = fmaf((float)(c[0] * m0 + c[1]), scale[i], g[2 * h]);
                            g[2 * h + 1] = fmaf((float)(c[2] * m0 + c[3]), scale[i], g[2 * h + 1]);
                        }
                    }
                }
            }
            fit_arrive(&edone[ebefore], lane);
            if (asked < n) {                           // row0: the first row of tile k
                if (feed && lane == 0) {
                    fetch(before, row0 + (ring_tiles - 1) * row_step);
                    if (asked + kAhead < n) prefetch(row0 + (ring_tiles - 1 + kAhead) * row_step);
                }
                ++asked;
            }
        }
        row0 += row_step;
        before = slot;
        if (++slot == ring_tiles) {
            slot = 0;
            parity ^= 1u;
        }
        xbefore = xnow;
        ebefore = eslot;
        xnow += (uint32_t)exp_bytes;
        if (++eslot == ring_exps) {
            eslot = 0;
            eparity ^= 1u;
            xnow = exps;
        }
    }
    if (!ok) {                                 // as above
        if (lane == 0) raise_timeout(prm.status);
        for (int i = max(0, asked - ring_tiles); feed && i < asked; ++i)
            fit_wait(&mine[i % ring_tiles], (uint32_t)(i / ring_tiles) & 1u, prm.spin_limit);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float s = grad[i][e] * weight;
            s += __shfl_xor_sync(0xffffffffu, s, 1);
            s += __shfl_xor_sync(0xffffffffu, s, 2);
            const int c = (warp * NB + i) * 32 + (e >> 1) * 16 + (e & 1) * 8 + (lane >> 2);
            if ((lane & 3) == 0 && c < d) out[c] = s;
        }
    }
    __syncthreads();
}

// The CTAs' partial sums, and the Adam step: 32 parameters per CTA, eight warps that each add up every
// eighth partial (their loads all in flight), then the eight sums in order.  c1 = 1 - beta1^t, c2 = 1 - beta2^t.
__global__ void __launch_bounds__(256) train8_adam_kernel(const TrainParams prm, double c1, double c2)
{
    __shared__ double sums[8][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int d = prm.d, j = blockIdx.x * 32 + lane;
    pdl_wait();
    const float *p = prm.part + min(j, d + 1);
    double sum = 0.0;
    for (int c0 = warp; c0 < prm.ctas; c0 += 8 * 20) {
        float x[20];
#pragma unroll
        for (int k = 0; k < 20; ++k) x[k] = p[(int64_t)min(c0 + 8 * k, prm.ctas - 1) * (d + 2)];
#pragma unroll
        for (int k = 0; k < 20; ++k)
            if (c0 + 8 * k < prm.ctas) sum += (double)x[k];
    }
    sums[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || j > d + 1) return;
    if (*reinterpret_cast<volatile int *>(prm.status) == SPR_ERR_TIMEOUT) {
        // the gradient pass gave up: no step is taken, the loss reads NaN
        if (j == d + 1 && prm.loss) *prm.loss = __int_as_float(0x7fc00000);
        return;
    }
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += sums[w][lane];
    sum /= (double)prm.N;
    if (j == d + 1) {
        if (prm.loss) *prm.loss = (float)sum;
        return;
    }
    const double m = prm.beta1 * (double)prm.m[j] + (1.0 - prm.beta1) * sum;
    const double v = prm.beta2 * (double)prm.v[j] + (1.0 - prm.beta2) * sum * sum;
    prm.m[j] = (float)m;
    prm.v[j] = (float)v;
    prm.theta[j] = (float)((double)prm.theta[j] - prm.lr * (m / c1) / (sqrt(v / c2) + prm.eps));
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

// [N, pack8_pitch(d)] bytes in boxes of `width` bytes x `rows` rows, swizzled in `width` bytes
bool packed_map(CUtensorMap *map, const void *base, int64_t N, int d, int width, int rows)
{
    static const EncodeTiledFn fn = [] {   // initialised once, thread-safe
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            return reinterpret_cast<EncodeTiledFn>(p);
        return static_cast<EncodeTiledFn>(nullptr);
    }();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)pack8_pitch(d), (cuuint64_t)N};
    const cuuint64_t strides[1] = {(cuuint64_t)pack8_pitch(d)};
    const cuuint32_t box[2] = {(cuuint32_t)width, (cuuint32_t)rows}, elem[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, elem,
              CU_TENSOR_MAP_INTERLEAVE_NONE,
              width == 16   ? CU_TENSOR_MAP_SWIZZLE_NONE
              : width == 32 ? CU_TENSOR_MAP_SWIZZLE_32B
              : width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                            : CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NB, int T, int W, int C>
cudaError_t launch_train8(const TrainParams &tp, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];
    constexpr size_t room = (size_t)(228 / C - 1) * 1024;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(train8_kernel<NB, T, W, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)room);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    TrainParams p = tp;
    const int64_t all = (tp.N + T - 1) / T, most_ctas = (int64_t)sms * C;
    p.ctas = (int)(all < most_ctas ? all : most_ctas);
    if (p.ctas > kTrainMaxCtas) p.ctas = kTrainMaxCtas;
    const size_t tile = (size_t)tile_share(tp.d, T);
    int64_t ring = (int64_t)((room - Fit8<NB, T, W>::kBytes) / tile);
    if (ring > kMaxTiles) ring = kMaxTiles;
    const int64_t most = (all + p.ctas - 1) / p.ctas;       // tiles of one CTA
    if (ring < 3 && most >= 3) return cudaErrorInvalidConfiguration;      // two tiles are in use while the next arrives
    if (ring > most) ring = most;
    CUtensorMap map, emap;
    if (!packed_map(&map, tp.hidden, tp.N, tp.d, 128, T) || !packed_map(&emap, tp.hidden, tp.N, tp.d, exponent_width(tp.d), T))
        return cudaErrorInvalidValue;
    const size_t smem = (size_t)ring * tile + Fit8<NB, T, W>::kBytes;
    train8_kernel<NB, T, W, C><<<p.ctas, Fit8<NB, T, W>::kThreads, smem, st>>>(p, map, emap, (int)ring);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};          // set up while the gradient kernel ends
    cfg.gridDim = dim3((unsigned)((p.d + 2 + 31) / 32));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, train8_adam_kernel, p, 1.0 - pow(p.beta1, (double)p.t), 1.0 - pow(p.beta2, (double)p.t));
}

// Three tiles of 32 rows fit four CTAs to an SM up to 512 columns, two up to 1024 and one up to 2048; above that
// three of 16 rows, whose residuals two blocks share a warp for.
cudaError_t launch_train8_any(const TrainParams &tp, cudaStream_t st)
{
    if (tp.d <= 512) return launch_train8<4, 32, 4, 4>(tp, st);
    if (tp.d <= 1024) return launch_train8<4, 32, 8, 2>(tp, st);
    if (tp.d <= 2048) return launch_train8<4, 32, 16, 1>(tp, st);
    return launch_train8<8, 16, 16, 1>(tp, st);
}

}  // namespace

}  // namespace spr

using namespace spr;

static int train_step8(const void *packed, const uint8_t *labels, int64_t N, int d, float *theta, float *adam_m, float *adam_v,
                       int t, double lr, double beta1, double beta2, double eps, float *loss, void *ws, size_t ws_bytes,
                       void *cuda_stream, int flags, unsigned spin_limit)
{
    if (N < 0 || d <= 0 || t < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !(lr == lr))
        return SPR_ERR_INVALID_ARG;
    if (d % 16 != 0 || d > 4096 || N > 0x7fff0000) return SPR_ERR_UNSUPPORTED;      // rows are 32-bit coordinates
    if (N == 0) {        // no samples: no step, and the mean of nothing is not a number (all bits set)
        if (!loss) return SPR_OK;
        if (!aligned(loss, 4)) return SPR_ERR_INVALID_ARG;
        const int rc = device_supported();
        return rc != SPR_OK ? rc : finish(cudaMemsetAsync(loss, 0xff, sizeof(float), static_cast<cudaStream_t>(cuda_stream)));
    }
    if (!packed || !labels || !theta || !adam_m || !adam_v) return SPR_ERR_INVALID_ARG;
    if (!aligned(packed, 16) || !aligned(theta, 4) || !aligned(adam_m, 4) || !aligned(adam_v, 4) || (loss && !aligned(loss, 4)))
        return SPR_ERR_INVALID_ARG;
    Carver cv = carve(ws_bytes);
    const size_t part_off = train_ws_layout(cv, d);
    if (!ws || !aligned(ws, 256) || !cv.fits()) return SPR_ERR_WORKSPACE;
    const int rc = device_supported();
    if (rc != SPR_OK) return rc;

    TrainParams tp;
    memset(&tp, 0, sizeof tp);
    tp.hidden = packed;
    tp.labels = labels;
    tp.N = N;
    tp.d = d;
    tp.theta = theta;
    tp.m = adam_m;
    tp.v = adam_v;
    tp.t = t;
    tp.lr = lr;
    tp.beta1 = beta1;
    tp.beta2 = beta2;
    tp.eps = eps;
    tp.loss = loss;
    tp.part = at<float>(ws, part_off);
    tp.status = at<int>(ws, 0);
    tp.spin_limit = spin_limit ? spin_limit : kTrainSpin;
    tp.test_flags = flags;
    return finish(launch_train8_any(tp, static_cast<cudaStream_t>(cuda_stream)));
}

extern "C" {

int verifier_train_step8(const void *packed, const uint8_t *labels, int64_t N, int d, float *theta, float *adam_m,
                         float *adam_v, int t, double lr, double beta1, double beta2, double eps, float *loss, void *ws,
                         size_t ws_bytes, void *cuda_stream)
{
    return train_step8(packed, labels, N, d, theta, adam_m, adam_v, t, lr, beta1, beta2, eps, loss, ws, ws_bytes,
                       cuda_stream, 0, 0u);
}

int spr_test_verifier_train_step8(const void *packed, const uint8_t *labels, int64_t N, int d, float *theta, float *adam_m,
                                  float *adam_v, int t, double lr, double beta1, double beta2, double eps, float *loss,
                                  void *ws, size_t ws_bytes, void *cuda_stream, int flags, unsigned spin_limit)
{
    if (flags & ~TRAIN_TEST_NO_FETCH) return SPR_ERR_INVALID_ARG;
    return train_step8(packed, labels, N, d, theta, adam_m, adam_v, t, lr, beta1, beta2, eps, loss, ws, ws_bytes,
                       cuda_stream, flags, spin_limit);
}

}  // extern "C"
