// The vocabulary head's products where they are small: a few million multiply-adds, bound by latency.
//
// The tensor-core kernels (head_gemm.cu) want operands laid out for them, tiles of 256 x 256 and some
// microseconds to start: a problem of 67 x 257 x 1003 keeps 8 of 148 SMs busy there.  Here a CTA forms
// a 32 x 32 tile in fp32 on the CUDA cores from the caller's own tensors, whatever their alignment.  Its
// 1024 threads are four groups that each take a quarter of the contraction (the chain of loads is what
// takes the time), double-buffered through registers; the four sums are added in order.
#include "head_small.h"

#include "common.cuh"
#include "launch.h"

namespace spr {

namespace {

constexpr int kTile = 32;
constexpr int kGroups = 4;
constexpr int kSmallThreads = 256 * kGroups;
constexpr int kPitch = kTile + 2;        // even: pairs are read as float2

template <typename T>
__device__ __forceinline__ float load_one(const SmallOperand &o, int64_t at)
{
    return o.f32 ? static_cast<const float *>(o.p)[at] : (float)static_cast<const T *>(o.p)[at];
}
// Four elements per thread of a 32 (k) x 32 (m) tile; neighbouring threads follow the contiguous axis.
// Where `live` is given, entry k of the contraction counts only if live[k] is a token of the vocabulary.
template <typename T>
__device__ __forceinline__ void fetch(const SmallOperand &o, int m0, int ms, int k0, int k_end, int t, const int32_t *live, int V,
                                      float (&x)[4])
{
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int a = t & 31, b = (t >> 5) + 8 * u;
        const int k = k0 + (o.across ? b : a), m = m0 + (o.across ? a : b);
        bool there = k < k_end && m < ms;
        if (there && live) {
            const int tok = live[k];
            there = tok >= 0 && tok < V;
        }
        x[u] = there ? load_one<T>(o, (int64_t)m * o.sm + (int64_t)k * o.sk) : 0.f;
    }
}
__device__ __forceinline__ void put(float (*s)[kPitch], bool across, int t, const float (&x)[4])
{
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int a = t & 31, b = (t >> 5) + 8 * u;
        s[across ? b : a][across ? a : b] = x[u];
    }
}

template <int MODE, typename T>
__global__ void __launch_bounds__(kSmallThreads) small_kernel(const SmallParams prm)
{
    __shared__ float sa[kGroups][kTile][kPitch], sb[kGroups][kTile][kPitch];
    pdl_trigger();
    int tile = blockIdx.x;
    const int first = prm.job[0].tiles_m * prm.job[0].tiles_n * prm.job[0].splits;      // CTAs of the first product
    const bool second = tile >= first;
    if (second) tile -= first;
    const SmallJob &j = prm.job[second ? 1 : 0];
    const int tiles = j.tiles_m * j.tiles_n, split = tile / tiles;
    tile -= split * tiles;
    const int m0 = (tile / j.tiles_n) * kTile, n0 = (tile % j.tiles_n) * kTile;
    const int g = threadIdx.x >> 8, t = threadIdx.x & 255;
    const int ty = t >> 4, tx = t & 15;
    const int per = (j.K + kGroups * j.splits - 1) / (kGroups * j.splits);
    const int k_lo = min(j.K, (split * kGroups + g) * per), k_hi = min(j.K, k_lo + per);
    float c[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
    float xa[4], xb[4];
    if (MODE == SMALL_OUT) pdl_wait();
    fetch<T>(j.a, m0, j.rows, k_lo, k_hi, t, nullptr, 0, xa);
    fetch<T>(j.b, n0, j.cols, k_lo, k_hi, t, j.live, prm.V, xb);
    for (int k = k_lo; k < k_hi; k += kTile) {
        put(sa[g], j.a.across, t, xa);
        put(sb[g], j.b.across, t, xb);
        asm volatile("bar.sync %0, 256;" ::"r"(g + 1) : "memory");
        if (k + kTile < k_hi) {
            fetch<T>(j.a, m0, j.rows, k + kTile, k_hi, t, nullptr, 0, xa);
            fetch<T>(j.b, n0, j.cols, k + kTile, k_hi, t, j.live, prm.V, xb);
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) xa[u] = xb[u] = 0.f;
        }
#pragma unroll 8
        for (int i = 0; i < kTile; ++i) {
            const float2 a = *reinterpret_cast<const float2 *>(&sa[g][i][2 * ty]);
            const float2 b = *reinterpret_cast<const float2 *>(&sb[g][i][2 * tx]);
            c[0][0] = fmaf(a.x, b.x, c[0][0]);
            c[0][1] = fmaf(a.x, b.y, c[0][1]);
            c[1][0] = fmaf(a.y, b.x, c[1][0]);
            c[1][1] = fmaf(a.y, b.y, c[1][1]);
        }
        asm volatile("bar.sync %0, 256;" ::"r"(g + 1) : "memory");
    }
    // the groups' sums, in order
    float4 *red = reinterpret_cast<float4 *>(&sa[0][0][0]);
    __syncthreads();
    if (g > 0) red[(g - 1) * 256 + t] = make_float4(c[0][0], c[0][1], c[1][0], c[1][1]);
    __syncthreads();
    if (g > 0) return;
#pragma unroll
    for (int i = 0; i < kGroups - 1; ++i) {
        const float4 y = red[i * 256 + t];
        c[0][0] += y.x;
        c[0][1] += y.y;
        c[1][0] += y.z;
        c[1][1] += y.w;
    }
    if (MODE == SMALL_OUT && j.splits > 1) {
        // the CTA that takes the tile's last ticket adds the splits' sums up, in order
        __shared__ int last;
        float4 *mine = reinterpret_cast<float4 *>(j.acc) + ((int64_t)split * tiles + tile) * 256 + t;
        *mine = make_float4(c[0][0], c[0][1], c[1][0], c[1][1]);
        __threadfence();
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (t == 0) last = take_ticket(&j.tickets[tile], j.splits);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (!last) return;
        __threadfence();
        const float4 *from = reinterpret_cast<const float4 *>(j.acc) + (int64_t)tile * 256 + t;
        float4 sum = __ldcg(from);
#pragma unroll 4
        for (int s = 1; s < j.splits; ++s) {
            const float4 y = __ldcg(from + (int64_t)s * tiles * 256);
            sum = make_float4(sum.x + y.x, sum.y + y.y, sum.z + y.z, sum.w + y.w);
        }
        c[0][0] = sum.x;
        c[0][1] = sum.y;
        c[1][0] = sum.z;
        c[1][1] = sum.w;
    }
    const int col = n0 + 2 * tx;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = m0 + 2 * ty + h;
        if (MODE == SMALL_STATS) {
            // (max, sum of exp) over the tile's columns: a row is 16 lanes
            float m = fmaxf(col < j.cols ? c[h][0] : neg_inf(), col + 1 < j.cols ? c[h][1] : neg_inf());
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float ref = m == neg_inf() ? 0.f : m;
            float s = (col < j.cols ? ex2((c[h][0] - ref) * kLog2e) : 0.f) + (col + 1 < j.cols ? ex2((c[h][1] - ref) * kLog2e) : 0.f);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (tx == 0 && row < j.rows) j.part[(int64_t)row * j.tiles_n + n0 / kTile] = make_float2(m, s);
        } else if (row < j.rows) {
            if (MODE == SMALL_DLOGITS) {
                const int tok = j.targets[row];
                const bool keep = tok >= 0 && tok < prm.V;
                if (tok >= prm.V && n0 == 0 && tx == 0) raise_status(prm.status, SPR_ERR_BAD_TOKEN);
                const float lse = keep ? j.lse[row] : 0.f, w = keep ? j.grad_loss[row] : 0.f;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (col + e < j.cols)
                        j.d[(int64_t)row * j.d_pitch + col + e] = keep ? w * expf(c[h][e] - lse) - (col + e == tok ? w : 0.f) : 0.f;
            } else {
                T *o = static_cast<T *>(j.out) + (int64_t)row * j.out_pitch + col;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (col + e < j.cols) o[e] = (T)c[h][e];
            }
        }
    }
}

template <int MODE>
cudaError_t launch_mode(const SmallParams &prm, unsigned ctas, bool f32, bool behind, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = behind ? 1 : 0;
    return f32 ? cudaLaunchKernelEx(&cfg, small_kernel<MODE, float>, prm) : cudaLaunchKernelEx(&cfg, small_kernel<MODE, __nv_bfloat16>, prm);
}

}  // namespace

cudaError_t launch_small(SmallMode mode, bool f32, SmallParams &prm, int njobs, cudaStream_t st)
{
    int64_t ctas = 0;
    for (int i = 0; i < njobs; ++i) {
        SmallJob &j = prm.job[i];
        j.tiles_m = (int)((j.rows + kTile - 1) / kTile);
        j.tiles_n = (int)((j.cols + kTile - 1) / kTile);
        if (j.splits < 1) j.splits = 1;
        ctas += (int64_t)j.tiles_m * j.tiles_n * j.splits;
    }
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    switch (mode) {
    case SMALL_STATS: return launch_mode<SMALL_STATS>(prm, (unsigned)ctas, f32, false, st);
    case SMALL_DLOGITS: return launch_mode<SMALL_DLOGITS>(prm, (unsigned)ctas, f32, false, st);
    default: return launch_mode<SMALL_OUT>(prm, (unsigned)ctas, f32, true, st);
    }
}

}  // namespace spr
