// One Adam step of the linear verifier on hidden states kept in 8 bits (hidden_pack.cu):
//   z_i = b + sum_j w_j q_ij 2^e_ij,  r = sigma(z) - y,  grad_j = sum_i r_i 2^e_ij q_ij
// Floor: the packed rows once, 1.03 d bytes a sample.  At that rate an SM takes in some 24 elements a
// clock, and turning a byte into a float costs as much as the two products it goes into: the pass
// is bound by instructions before it is bound by memory.  So:
//   - the dot product stays in integers.  A weight is written as 24 bits relative to the largest of
//     its 16 (a lane's vector), in three signed bytes, w = 2^E (d0 2^16 + d1 2^8 + d2); then sum q d is
//     four dp4a per 16 elements and byte, exact, and one conversion per vector is left.  Rounding a
//     weight costs at most 2^-23 of the largest weight beside it, what fp32 products cost.
//   - the gradient is formed with columns, not rows, in registers: a thread owns 16 columns and walks
//     over the rows of a tile.  Its sums are 16 registers instead of the 64 that a warp per row needs, so
//     that 16 warps fit on an SM, and rows are independent.
// A CTA takes tiles of consecutive rows (one bulk copy each, a ring of tiles in shared memory):
// first a warp per row (two for d > 2048) forms the dot products, one barrier, then every warp has the
// tile's residuals in its lanes and the columns' sums are formed.  Tiles are dealt in a fixed
// pattern and all sums have a fixed order: a step is reproducible bit for bit.
#include <math.h>
#include <string.h>

#include <atomic>

#include "host_util.h"
#include "launch.h"
#include "vocab_common.cuh"

namespace spr {

namespace {

constexpr int kFitThreads = 512;
constexpr int kFitWarps = kFitThreads / 32;
constexpr int kMaxTiles = 8;             // tiles of the ring
constexpr size_t kRingBytes = 200 * 1024;

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

// 2^e of an exponent byte.  -128 marks a block that held an infinity or NaN, with bytes of zero: the same
// shift makes that minus infinity, and its product with a zero byte NaN.
__device__ __forceinline__ float block_scale(const unsigned char *p)
{
    return __int_as_float((int)*reinterpret_cast<const signed char *>(p) * (1 << 23) + 127 * (1 << 23));
}

// Sixteen weights as three planes of signed bytes, and their unit 2^E.
__device__ __forceinline__ float split_weights(const float (&w)[16], uint32_t (&digit)[3][4])
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(w[e]) & 0x7fffffffu);
#pragma unroll
    for (int k = 0; k < 4; ++k) digit[0][k] = digit[1][k] = digit[2][k] = 0u;
    if (top >= 0x7f800000u) return __int_as_float(0x7fc00000);      // a weight that is not finite shows
    // unit 2^E with |w| <= 8355711 units (three digits reach that); weights below 2^-100 count as zero
    int E = max((int)(top >> 23) - 127, -100) - 22;
    if (rintf(ldexpf(__uint_as_float(top), -E)) > 8355711.f) ++E;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int v = __float2int_rn(ldexpf(w[e], -E));
        const int d2 = (int)(signed char)(v & 255), v1 = (v - d2) >> 8;
        const int d1 = (int)(signed char)(v1 & 255), d0 = (v1 - d1) >> 8;
        digit[0][e >> 2] |= (uint32_t)(d0 & 255) << (8 * (e & 3));
        digit[1][e >> 2] |= (uint32_t)(d1 & 255) << (8 * (e & 3));
        digit[2][e >> 2] |= (uint32_t)(d2 & 255) << (8 * (e & 3));
    }
    return ldexpf(1.f, E);
}

// VPL: 16-byte vectors per lane of a row; WPR: warps per row; T: rows per tile
template <int VPL, int WPR, int T>
__global__ void __launch_bounds__(kFitThreads, 1) train8_kernel(const TrainParams prm, int ring_tiles)
{
    constexpr int kRowsPerWarp = T * WPR / kFitWarps;     // rows a warp forms dot products of, per tile
    static_assert(kRowsPerWarp >= 1 && T <= 64, "tile height");
    constexpr int kLaneRows = (T + 31) / 32;
    extern __shared__ __align__(128) unsigned char tiles[];
    __shared__ __align__(8) uint64_t bars[kMaxTiles];
    __shared__ float zpart[2][T][WPR];
    __shared__ float res_of[kFitWarps][T];    // the tile's residuals, a copy per warp
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int d = prm.d, nv = d / 16;
    const int pitch = pack8_pitch(d);
    const uint32_t tile_bytes = (uint32_t)(T * pitch);
    pdl_trigger();

    // this CTA's tiles: blockIdx.x, + gridDim.x, ...; only the last tile of the data can be short
    const int64_t all = (prm.N + T - 1) / T;
    const int n = (int64_t)blockIdx.x < all ? (int)((all - blockIdx.x + gridDim.x - 1) / gridDim.x) : 0;
    auto first_row = [&](int k) { return ((int64_t)blockIdx.x + (int64_t)k * gridDim.x) * T; };
    auto rows_of = [&](int k) { return (int)min((int64_t)T, prm.N - first_row(k)); };
    auto fetch = [&](int k) {
        const uint32_t bytes = (uint32_t)(rows_of(k) * pitch);
        uint64_t *bar = &bars[k % ring_tiles];
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(fit_addr(bar)), "r"(bytes) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                         fit_addr(tiles + (size_t)(k % ring_tiles) * tile_bytes)),
                     "l"(static_cast<const unsigned char *>(prm.hidden) + first_row(k) * pitch), "r"(bytes), "r"(fit_addr(bar))
                     : "memory");
    };
    if (tid == 0) {
        for (int s = 0; s < ring_tiles; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(fit_addr(&bars[s])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int k = 0; !(prm.test_flags & TRAIN_TEST_NO_FETCH) && k < ring_tiles && k < n; ++k) fetch(k);
    }
    // labels of the next tile, one row per lane (a label fetched when it is wanted would cost a trip to memory)
    auto tile_labels = [&](int k, float (&y)[kLaneRows]) {
#pragma unroll
        for (int h = 0; h < kLaneRows; ++h) {
            const int r = lane + 32 * h;
            y[h] = k < n && r < rows_of(k) && r < T ? (float)prm.labels[first_row(k) + r] : 0.f;
        }
    };
    float y_next[kLaneRows];
    tile_labels(0, y_next);

    // weights of this lane's vectors of a row: v0 + 32 j
    const int part = warp % WPR, v0 = part * VPL * 32 + lane;
    uint32_t digit[VPL][3][4];
    float unit[VPL];
    int at[VPL], scale_at[VPL];      // a lane past the row's end reads the last vector, with weights of zero
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const int vi = v0 + 32 * j;
        at[j] = min(vi, nv - 1) * 16;
        scale_at[j] = d + (min(vi, nv - 1) >> 1);
        float w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = vi < nv ? prm.theta[vi * 16 + e] : 0.f;
        unit[j] = split_weights(w, digit[j]);
    }
    const float bias = prm.theta[d];

    // columns of this thread: vector cv, rows sub, sub + subs, ... of every tile
    const int subs = min(kFitThreads / nv, T);
    const int cv = tid % nv, sub = tid / nv;
    uint64_t acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = pack2(0.f, 0.f);
    double acc_b = 0.0, acc_loss = 0.0;        // warp 0
    const uint64_t off = pack2(-8388736.f, -8388736.f);
    __syncthreads();                           // the barriers are set up

    bool ok = true;
    int k = 0;
    for (; k < n; ++k) {
        const unsigned char *tile = tiles + (size_t)(k % ring_tiles) * tile_bytes;
        ok = fit_wait(&bars[k % ring_tiles], (uint32_t)(k / ring_tiles) & 1u, prm.spin_limit);
        float y[kLaneRows];
#pragma unroll
        for (int h = 0; h < kLaneRows; ++h) y[h] = y_next[h];
        tile_labels(k + 1, y_next);
        const int rows = rows_of(k);
        // ---- dot products, a warp (pair) per row; rows behind the last hold older bytes and are not used
        float dot[kRowsPerWarp];
#pragma unroll
        for (int i = 0; i < kRowsPerWarp; ++i) {
            const unsigned char *row = tile + (warp / WPR + i * (kFitWarps / WPR)) * pitch;
            dot[i] = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const uint4 x = *reinterpret_cast<const uint4 *>(row + at[j]);
                const int q[4] = {(int)x.x, (int)x.y, (int)x.z, (int)x.w};
                int s0 = 0, s1 = 0, s2 = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    s0 = __dp4a(q[c], (int)digit[j][0][c], s0);
                    s1 = __dp4a(q[c], (int)digit[j][1][c], s1);
                    s2 = __dp4a(q[c], (int)digit[j][2][c], s2);
                }
                const float s = fmaf((float)s0, 65536.f, (float)(s1 * 256 + s2));     // |s1| < 2^18
                dot[i] = fmaf(s * unit[j], block_scale(row + scale_at[j]), dot[i]);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < kRowsPerWarp; ++i) dot[i] += __shfl_xor_sync(0xffffffffu, dot[i], o);
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < kRowsPerWarp; ++i) zpart[k & 1][warp / WPR + i * (kFitWarps / WPR)][part] = dot[i];
        }
        ok = __syncthreads_and(ok) != 0;       // the dot products are there, and the tile before this one is done with
        if (!ok) break;
        if (tid == 0 && k > 0 && k - 1 + ring_tiles < n) fetch(k - 1 + ring_tiles);
        // ---- residuals, a row per lane, in every warp
#pragma unroll
        for (int h = 0; h < kLaneRows; ++h) {
            const int r = lane + 32 * h;
            float z = bias;
            if (r < T) {
                z += zpart[k & 1][r][0];
                if (WPR > 1) z += zpart[k & 1][r][WPR - 1];
            }
            const float res = r < rows ? 1.f / (1.f + expf(-z)) - y[h] : 0.f;
            if (r < T) res_of[warp][r] = res;
            if (warp == 0 && r < rows) {
                acc_b += (double)res;
                acc_loss += (double)(fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))) - y[h] * z);
            }
        }
        __syncwarp();
        // ---- columns
        const unsigned char *row = tile + sub * pitch + cv * 16, *row_e = tile + sub * pitch + d + (cv >> 1);
#pragma unroll 4
        for (int r = sub < subs ? sub : rows; r < rows; r += subs, row += subs * pitch, row_e += subs * pitch) {
            const uint4 x = *reinterpret_cast<const uint4 *>(row);
            const float rs = res_of[warp][r] * block_scale(row_e);
            const uint64_t rs2 = pack2(rs, rs);
            // byte + 128 as the low mantissa byte of 2^23, which is then taken off
            const uint32_t w[4] = {x.x ^ 0x80808080u, x.y ^ 0x80808080u, x.z ^ 0x80808080u, x.w ^ 0x80808080u};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint64_t a = pack2(__uint_as_float(__byte_perm(w[c], 0x4b000000u, 0x7440)),
                                         __uint_as_float(__byte_perm(w[c], 0x4b000000u, 0x7441)));
                const uint64_t b = pack2(__uint_as_float(__byte_perm(w[c], 0x4b000000u, 0x7442)),
                                         __uint_as_float(__byte_perm(w[c], 0x4b000000u, 0x7443)));
                acc[2 * c] = fma2(rs2, add2(a, off), acc[2 * c]);
                acc[2 * c + 1] = fma2(rs2, add2(b, off), acc[2 * c + 1]);
            }
        }
        __syncwarp();                          // the residuals are overwritten for the next tile
    }
    if (!ok) {
        // A wait ran out: report it, then give the copies still on their way the same bounded time to
        // land before the CTA's shared memory goes away.
        if (tid == 0) {
            raise_status(prm.status, SPR_ERR_TIMEOUT);
            for (int i = k; !(prm.test_flags & TRAIN_TEST_NO_FETCH) && i < n && i < k - 1 + ring_tiles; ++i)
                fit_wait(&bars[i % ring_tiles], (uint32_t)(i / ring_tiles) & 1u, prm.spin_limit);
        }
    }
    __syncthreads();
    // sums of the row subsets, in order
    float *red = reinterpret_cast<float *>(tiles);
    if (sub < subs) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float lo, hi;
            unpack2(acc[e], lo, hi);
            *reinterpret_cast<float2 *>(red + (size_t)sub * d + cv * 16 + 2 * e) = make_float2(lo, hi);
        }
    }
    __syncthreads();
    float *out = prm.part + (int64_t)blockIdx.x * (d + 2);
    for (int j = tid; j < d; j += kFitThreads) {
        float s = red[j];
        for (int i = 1; i < subs; ++i) s += red[(size_t)i * d + j];
        out[j] = s;
    }
    if (warp == 0) {
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

template <int VPL, int WPR, int T>
cudaError_t launch_train8(const TrainParams &tp, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t tile = (size_t)T * pack8_pitch(tp.d);
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(train8_kernel<VPL, WPR, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes + 4096);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    TrainParams p = tp;
    const int64_t all = (tp.N + T - 1) / T;
    p.ctas = (int)(all < sms ? all : sms);
    if (p.ctas > kTrainMaxCtas) p.ctas = kTrainMaxCtas;
    int64_t ring = (int64_t)(kRingBytes + 4096) / (int64_t)tile;
    if (ring > kMaxTiles) ring = kMaxTiles;
    const int64_t most = (all + p.ctas - 1) / p.ctas;       // tiles of one CTA
    if (ring > most) ring = most;
    size_t smem = (size_t)ring * tile;
    const size_t red = 4 * (size_t)kFitThreads * 16;        // the row subsets' sums: subs * d <= 512 * 16 floats
    if (smem < red) smem = red;
    train8_kernel<VPL, WPR, T><<<p.ctas, kFitThreads, smem, st>>>(p, (int)ring);
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

// Tiles of 16, 32 or 64 rows: about 64 KB, so that three fit and a barrier is worth some thousand
// elements; no higher than what deals every SM a tile.
cudaError_t launch_train8_any(const TrainParams &tp, cudaStream_t st)
{
    const int vpl = (tp.d / 16 + 31) / 32;
    const bool few = tp.N < (int64_t)148 * 64;
    if (vpl <= 1) return few ? launch_train8<1, 1, 16>(tp, st) : launch_train8<1, 1, 64>(tp, st);
    if (vpl <= 2) return few ? launch_train8<2, 1, 16>(tp, st) : launch_train8<2, 1, 64>(tp, st);
    if (vpl <= 3) return few ? launch_train8<3, 1, 16>(tp, st) : launch_train8<3, 1, 32>(tp, st);
    if (vpl <= 4) return few ? launch_train8<4, 1, 16>(tp, st) : launch_train8<4, 1, 32>(tp, st);
    if (vpl <= 6) return launch_train8<3, 2, 16>(tp, st);
    return launch_train8<4, 2, 16>(tp, st);
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
    if (d % 16 != 0 || d > 4096) return SPR_ERR_UNSUPPORTED;
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
