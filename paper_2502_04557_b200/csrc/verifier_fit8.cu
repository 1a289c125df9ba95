// One Adam step of the linear verifier on hidden states kept in 8 bits (hidden_pack.cu):
//   z_i = b + sum_j w_j q_ij 2^e_ij,  r = sigma(z) - y,  grad_j = sum_i r_i 2^e_ij q_ij
// Floor: the packed rows once, 1.03 d bytes a sample (2^18 rows of 2048: 554 MB, 86 us; measured 157 us).  At that
// rate an SM takes in some 24 elements a clock, and on the CUDA cores it is instructions that bound the pass: a byte
// turned into a float costs as much as the two products it goes into (measured: 244 us that way, 180 us with the
// dot products in dp4a).  So both sums are integer products on the tensor cores (mma.m16n8k32, s8 x s8 -> s32):
//   - a block of 32 columns shares its exponent within a row, so a block is one step of the contraction of
//     the dot products.  A weight is written as 24 bits relative to the largest of its block, in three balanced
//     signed digits, w = 2^E (256^2 d0 + 256 d1 + d2): three columns of the second operand.  What is left per
//     block and row is one conversion and the row's scale.  Rounding a weight costs at most 2^-24 of twice
//     the largest weight of its block, what fp32 products cost.
//   - for the gradient the contraction runs over the rows of a tile: r_i 2^e_ij of the block, written as 22 bits
//     relative to the largest of the tile in three digits, times the bytes, which ldmatrix transposes.  The
//     integer sums are exact; per tile and column one conversion, and an fp32 sum over tiles.
// A CTA takes tiles of consecutive rows through a ring in shared memory, by TMA in boxes of 128 bytes by all rows
// with the 128-byte swizzle, which keeps ldmatrix free of bank conflicts (a copy per row into a padded pitch took
// 100 clocks each to issue, half of a tile's time: 181 us).  Dot products by all warps, a barrier, then residuals
// by two warps while the others form the sums of their blocks of columns in the tile before (a row's residual by a
// warp of its own instead: 178 us; every warp then has the latency of a sigmoid in its way).  What bounds it now is
// instructions again, a conversion, a scale and the digits of every block and row, and the barrier per tile.
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

constexpr int kFitThreads = 1024;
constexpr int kFitWarps = kFitThreads / 32;
constexpr int kMaxTiles = 8;             // tiles of the ring
constexpr int kAhead = 2;                // tiles on their way into L2 behind those of the ring
constexpr size_t kSmemBytes = 221 * 1024;     // dynamic; the static arrays take some 5 KB more

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
// 1, 2 or 4 exponent bytes from a shared address that is a multiple of as many
template <int N>
__device__ __forceinline__ uint32_t load_exponents(uint32_t addr)
{
    static_assert(N == 1 || N == 2 || N == 4, "exponent bytes");
    uint32_t w;
    if (N == 1) asm volatile("ld.shared.u8 %0, [%1];" : "=r"(w) : "r"(addr));
    else if (N == 2) asm volatile("ld.shared.u16 %0, [%1];" : "=r"(w) : "r"(addr));
    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(addr));
    return w;
}
// three balanced digits of a 24-bit integer: v = 256^2 d0 + 256 d1 + d2, as the bytes 2, 1, 0
__device__ __forceinline__ uint32_t digits(int v) { return ((uint32_t)v + 0x808080u) ^ 0x808080u; }

// Digits of 32 numbers (a lane each) where the lanes of a product want them: plane p (d0, d1, d2), then for each t
// of 4 the numbers 4 t .. 4 t + 3 and 16 + 4 t .. + 3.  96 bytes.
__device__ __forceinline__ void put_digits(uint32_t dst, uint32_t u, int lane)
{
    const uint32_t at = dst + (uint32_t)(((lane & 15) >> 2) * 8 + (lane >> 4) * 4 + (lane & 3));
    asm volatile("st.shared.u8 [%0], %1;\n\tst.shared.u8 [%0 + 32], %2;\n\tst.shared.u8 [%0 + 64], %3;" ::"r"(at), "r"(u >> 16),
                 "r"(u >> 8), "r"(u)
                 : "memory");
}
// The second operand of a product: column n is plane n, and the columns from the fourth on are zero (lanes that stand for
// them read a place that holds zeros).
__device__ __forceinline__ uint2 get_digits(uint32_t addr)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
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

// A tile in shared memory: boxes of 128 bytes x T rows, one after the other; inside, 16-byte units are swizzled.
// Byte c of row r:
template <int T>
__device__ __forceinline__ uint32_t tile_at(int r, int c)
{
    return (uint32_t)((c >> 7) * (T * 128) + r * 128 + (((c >> 4) ^ r) & 7) * 16 + (c & 15));
}
// Unit k past a unit whose own index is a multiple of the units asked for: the swizzle's exclusive or is linear in it.
__device__ __forceinline__ uint32_t unit_at(uint32_t base, int k) { return base ^ (uint32_t)(k << 4); }
__host__ __device__ constexpr int tile_boxes(int d) { return (pack8_pitch(d) + 127) / 128; }

// NB: blocks of 32 columns per warp; T: rows per tile (16 or 32)
template <int NB, int T>
__global__ void __launch_bounds__(kFitThreads, 1) train8_kernel(const TrainParams prm, const __grid_constant__ CUtensorMap map, int ring_tiles)
{
    constexpr int kRowGroups = T / 16;                     // of 16 rows, for the dot products
    constexpr int kNB1 = NB * kRowGroups;                  // blocks a warp takes of its row group there
    constexpr int kSlices = kFitWarps / kRowGroups;        // warps that share a row's dot product
    constexpr int kDig = NB < 2 ? NB : 2;                  // blocks whose residuals a warp splits at a time
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t bars[kMaxTiles];
    __shared__ __align__(16) uint32_t zeros[4];
    __shared__ float zpart[2][kSlices][T];
    __shared__ float residual[2][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int d = prm.d, blocks = (d + 31) / 32;
    const int boxes = tile_boxes(d), tile_bytes = boxes * T * 128;
    // digits of the weights [blocks][96], of the scaled residuals (kDig blocks per warp), units of the weights [blocks], the ring
    const uint32_t wdig = fit_addr(smem), rdig = wdig + (uint32_t)(kFitWarps * NB * 96 + warp * kDig * 96);
    float *unit = reinterpret_cast<float *>(smem + kFitWarps * (NB + kDig) * 96);
    const uint32_t ring = (fit_addr(unit + kFitWarps * NB) + 1023u) & ~1023u;
    pdl_trigger();

    // this CTA's tiles: blockIdx.x, + gridDim.x, ...; only the last tile of the data can be short
    const int N = (int)prm.N;
    const int all = (N + T - 1) / T;
    const int n = (int)blockIdx.x < all ? (all - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
    const int row_step = (int)gridDim.x * T;
    const bool feed = !(prm.test_flags & TRAIN_TEST_NO_FETCH);
    // Every warp asks for a box of the tile at row0 (the first for a 33rd); rows and bytes that do not exist arrive as zeros.
    auto fetch = [&](int slot, int row0) {
        if (lane == 0) {
            if (warp == 0)
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(fit_addr(&bars[slot])), "r"((uint32_t)tile_bytes) : "memory");
            for (int b = warp; b < boxes; b += kFitWarps)
                fetch_box(ring + (uint32_t)(slot * tile_bytes + b * T * 128), &map, b * 128, row0, &bars[slot]);
        }
    };
    // Three tiles of 2048 columns are all that shared memory holds, and two of them are in use: what comes after the next
    // tile is asked for as far as L2, so that memory always has kAhead tiles to bring.
    auto prefetch = [&](int row0) {
        if (lane == 0)
            for (int b = warp; b < boxes; b += kFitWarps) prefetch_box(&map, b * 128, row0);
    };
    if (tid == 0) {
        for (int s = 0; s < ring_tiles; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(fit_addr(&bars[s])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < 4) zeros[tid] = 0u;
    __syncthreads();
    for (int k = 0; feed && k < ring_tiles && k < n; ++k) fetch(k, (int)blockIdx.x * T + k * row_step);
    for (int k = ring_tiles; feed && k < ring_tiles + kAhead && k < n; ++k) prefetch((int)blockIdx.x * T + k * row_step);
    // Labels, one row per lane, two tiles ahead and as the bytes they are: a label fetched when it is wanted would cost
    // a trip to memory.
    auto tile_label = [&](int64_t row) -> uint32_t { return prm.labels[lane < T && row + lane < prm.N ? row + lane : 0]; };
    uint32_t y_raw[2] = {0u, 0u};
    if (warp < 2) {
        y_raw[0] = tile_label((int64_t)blockIdx.x * T);
        y_raw[1] = tile_label((int64_t)blockIdx.x * T + row_step);
    }

    for (int b = warp; b < kFitWarps * NB; b += kFitWarps) {
        const int c = b * 32 + lane;
        const float w = c < d ? prm.theta[c] : 0.f;
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(w) & 0x7fffffffu);
        // unit 2^E with |w| <= 8355711 units (three digits reach that); weights below 2^-100 count as zero
        int E = max((int)(top >> 23) - 127, -100) - 22;
        if (rintf(ldexpf(__uint_as_float(top), -E)) > 8355711.f) ++E;
        const bool finite = top < 0x7f800000u;             // a weight that is not finite shows in every sum
        put_digits(wdig + (uint32_t)(b * 96), finite ? digits(__float2int_rn(ldexpf(w, -E))) : 0u, lane);
        if (lane == 0) unit[b] = finite ? ldexpf(1.f, E) : __int_as_float(0x7fc00000);
    }
    const float bias = prm.theta[d];

    // A lane's part of a product's result: columns 2 (lane % 4) and + 1, hence d0 and d1, or d2 and 0, or nothing.  The
    // integers 256 d0 + d1 and d2 are added up apart and weighted at the very end.
    const int m0 = (lane & 3) == 0 ? 256 : 1;
    const float weight = (lane & 3) == 0 ? 256.f : 1.f;
    // where the second operand stands, block by block
    const bool holds = lane < 12;
    const uint32_t dig_lane = (uint32_t)((lane >> 2) * 32 + (lane & 3) * 8), dig_step = holds ? 96u : 0u;
    // dot products: 16 rows of row group rg by blocks b1 .. b1 + kNB1 - 1
    const int rg = warp % kRowGroups, slice = warp / kRowGroups, b1 = slice * kNB1;
    const int n1 = min(kNB1, blocks - b1);
    const uint32_t a1 = tile_at<T>(rg * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, b1 * 32 + (lane >> 4) * 16);      // ldmatrix of 16 x 32
    const uint32_t e1 = tile_at<T>(rg * 16 + (lane >> 2), d + b1);         // rows lane / 4 and, 8 x 128 bytes on, + 8
    const uint32_t d1 = holds ? wdig + (uint32_t)(b1 * 96) + dig_lane : fit_addr(zeros);
    // columns: blocks b2 .. b2 + NB - 1, a row per lane
    const int my_row = lane & (T - 1), b2 = warp * NB, n2 = min(NB, blocks - b2);
    const uint32_t a2 = tile_at<T>(my_row, b2 * 32), e2 = tile_at<T>(my_row, d + b2);
    const uint32_t d2 = holds ? rdig + dig_lane : fit_addr(zeros);
    float grad[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) grad[i][e] = 0.f;
    double acc_b = 0.0, acc_loss = 0.0;        // warp 1
    __syncthreads();                           // the weights' digits are there

    // One barrier per tile: after that of tile k its dot products are there, and while two warps turn them into
    // residuals first, the others are at the columns of tile k - 1.
    bool ok = true;
    int k = 0, slot = 0, before = 0, row0 = (int)blockIdx.x * T;      // slot of tile k, of tile k - 1; first row of tile k
    uint32_t parity = 0;
    for (; k <= n; ++k) {
        const uint32_t now = ring + (uint32_t)(slot * tile_bytes);
        if (k < n) {
            // ---- dot products of tile k
            ok = fit_wait(&bars[slot], parity, prm.spin_limit);
            float z0 = 0.f, z1 = 0.f;
            if (n1 > 0) {
                const uint32_t x0 = load_exponents<kNB1>(now + e1), x1 = load_exponents<kNB1>(now + e1 + 1024);
#pragma unroll
                for (int i = 0; i < kNB1; ++i) {
                    if (i < n1) {
                        uint32_t a[4];
                        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                                     : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
                                     : "r"(unit_at(now + a1, 2 * i)));
                        int c[4];
                        mma_s8(c, a, get_digits(d1 + (uint32_t)i * dig_step));
                        const float u = unit[b1 + i];
                        z0 = fmaf((float)(c[0] * m0 + c[1]) * u, block_scale(x0, i), z0);
                        z1 = fmaf((float)(c[2] * m0 + c[3]) * u, block_scale(x1, i), z1);
                    }
                }
            }
            z0 *= weight;
            z1 *= weight;
            z0 += __shfl_xor_sync(0xffffffffu, z0, 1);
            z1 += __shfl_xor_sync(0xffffffffu, z1, 1);
            if ((lane & 3) == 0) {
                zpart[k & 1][slice][rg * 16 + (lane >> 2)] = z0;
                zpart[k & 1][slice][rg * 16 + (lane >> 2) + 8] = z1;
            }
        }
        ok = __syncthreads_and(ok) != 0;
        if (!ok) break;
        if (k > 1 && k - 2 + ring_tiles < n) {         // tile k - 2 is done with: its slot is the one before that of tile k - 1
            const int free_slot = before == 0 ? ring_tiles - 1 : before - 1;
            fetch(free_slot, row0 + (ring_tiles - 2) * row_step);
            if (k - 2 + ring_tiles + kAhead < n) prefetch(row0 + (ring_tiles - 2 + kAhead) * row_step);
        }
        if (warp < 2 && k < n) {
            // ---- residuals of tile k, a row per lane: warp 0 hands them on, warp 1 has the loss and the bias's gradient
            const float y = (float)y_raw[0];
            y_raw[0] = y_raw[1];
            y_raw[1] = tile_label((int64_t)row0 + 2 * (int64_t)row_step);
            float z = bias;
#pragma unroll
            for (int s = 0; s < kSlices; ++s) z += zpart[k & 1][s][lane & (T - 1)];
            const bool live = lane < T && row0 + lane < N;
            const float r = live ? 1.f / (1.f + expf(-z)) - y : 0.f;
            if (warp == 0) {
                residual[k & 1][lane] = r;
            } else if (live) {
                acc_b += (double)r;
                acc_loss += (double)(fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))) - y * z);
            }
        }
        if (k > 0 && n2 > 0) {
            // ---- columns of this warp's blocks in tile k - 1
            const uint32_t tile = ring + (uint32_t)(before * tile_bytes);
            const float r = residual[(k - 1) & 1][lane];
            const float show = __any_sync(0xffffffffu, r != r) ? __int_as_float(0x7fc00000) : 1.f;    // NaN has no digits
            const uint32_t x = load_exponents<NB>(tile + e2);
#pragma unroll
            for (int i0 = 0; i0 < NB; i0 += kDig) {
                float scale[kDig];
                __syncwarp();                      // the digits that stood there are read
#pragma unroll
                for (int i = 0; i < kDig; ++i) {
                    // a row that does not exist has r = 0, a block that does not exist is not read below
                    const float v = r != 0.f ? r * block_scale(x, i0 + i) : 0.f;
                    const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu);
                    const int E = max((int)(top >> 23), 27) - 148;                 // |v| < 2^22 units of 2^E
                    // v 2^-E + 1.5 2^23 rounds to the unit; the integer stands in the low bits of the sum
                    const int q = (int)(__float_as_uint(fmaf(v, __int_as_float((127 - E) << 23), 12582912.f)) - 0x4b400000u);
                    put_digits(rdig + (uint32_t)(i * 96), digits(q), lane);
                    scale[i] = __int_as_float((E + 127) << 23) * show;
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < kDig; ++i) {
                    if (i0 + i < n2) {
                        const uint2 bd = get_digits(d2 + (uint32_t)i * dig_step);
                        float *g = grad[i0 + i];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t at = unit_at(tile + a2, 2 * (i0 + i) + h);      // a last block of 16 reads on, into what follows in the row
                            int c[4];
                            if constexpr (T == 32) {
                                uint32_t a[4];
                                asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];"
                                             : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
                                             : "r"(at));
                                mma_s8(c, a, bd);
                            } else {
                                uint32_t a0, a4;
                                asm volatile("ldmatrix.sync.aligned.m16n16.x1.trans.shared.b8 {%0,%1}, [%2];" : "=r"(a0), "=r"(a4) : "r"(at));
                                mma_s8_k16(c, a0, a4, bd.x);
                            }
                            g[2 * h] = fmaf((float)(c[0] * m0 + c[1]), scale[i], g[2 * h]);
                            g[2 * h + 1] = fmaf((float)(c[2] * m0 + c[3]), scale[i], g[2 * h + 1]);
                        }
                    }
                }
            }
        }
        before = slot;
        if (++slot == ring_tiles) {
            slot = 0;
            parity ^= 1u;
        }
        row0 += row_step;
    }
    if (!ok) {
        // A wait ran out: report it, then give the copies still on their way the same bounded time to
        // land before the CTA's shared memory goes away.
        if (tid == 0) {
            raise_status(prm.status, SPR_ERR_TIMEOUT);
            for (int i = k; feed && i < n && i < k - 2 + ring_tiles; ++i)
                fit_wait(&bars[i % ring_tiles], (uint32_t)(i / ring_tiles) & 1u, prm.spin_limit);
        }
        __syncthreads();
    }
    float *out = prm.part + (int64_t)blockIdx.x * (d + 2);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float g = grad[i][e] * weight, s = g + __shfl_xor_sync(0xffffffffu, g, 1);
            const int c = (warp * NB + i) * 32 + (e >> 1) * 16 + (e & 1) * 8 + (lane >> 2);
            if ((lane & 3) == 0 && c < d) out[c] = s;
        }
    }
    if (warp == 1) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            acc_b += __shfl_xor_sync(0xffffffffu, acc_b, o);
            acc_loss += __shfl_xor_sync(0xffffffffu, acc_loss, o);
        }
        if (lane == 0) {
            out[d] = (float)acc_b;
            out[d + 1] = (float)acc_loss;
        }
    }
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

// [N, pack8_pitch(d)] bytes in boxes of 128 bytes x `rows` rows
bool packed_map(CUtensorMap *map, const void *base, int64_t N, int d, int rows)
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
    const cuuint32_t box[2] = {128, (cuuint32_t)rows}, elem[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, elem,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NB, int T>
cudaError_t launch_train8(const TrainParams &tp, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(train8_kernel<NB, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    TrainParams p = tp;
    const int64_t all = (tp.N + T - 1) / T;
    p.ctas = (int)(all < sms ? all : sms);
    if (p.ctas > kTrainMaxCtas) p.ctas = kTrainMaxCtas;
    const size_t tables = kFitWarps * ((NB + (NB < 2 ? NB : 2)) * 96 + NB * sizeof(float)), tile = (size_t)tile_boxes(tp.d) * T * 128;
    int64_t ring = (int64_t)((kSmemBytes - tables - 1024) / tile);
    if (ring > kMaxTiles) ring = kMaxTiles;
    const int64_t most = (all + p.ctas - 1) / p.ctas;       // tiles of one CTA
    if (ring < 3 && most >= 3) return cudaErrorInvalidConfiguration;      // two tiles are in use while the next arrives
    if (ring > most) ring = most;
    CUtensorMap map;
    if (!packed_map(&map, tp.hidden, tp.N, tp.d, T)) return cudaErrorInvalidValue;
    train8_kernel<NB, T><<<p.ctas, kFitThreads, tables + 1024 + (size_t)ring * tile, st>>>(p, map, (int)ring);
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

// Tiles of 32 rows, of 16 above 2048 columns: three of every width fit the ring.
cudaError_t launch_train8_any(const TrainParams &tp, cudaStream_t st)
{
    const int nb = ((tp.d + 31) / 32 + kFitWarps - 1) / kFitWarps;
    if (nb <= 1) return launch_train8<1, 32>(tp, st);
    if (nb <= 2) return launch_train8<2, 32>(tp, st);
    return launch_train8<4, 16>(tp, st);
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
    if (N == 0) return SPR_OK;
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
