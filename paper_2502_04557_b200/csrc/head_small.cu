// The vocabulary head's products in fp32 where they are small: some million multiply-adds, bound by latency.
//
// The tensor-core kernels (head_gemm.cu) want operands laid out for them, tiles of 256 x 256 and some
// microseconds to start: a problem of 67 x 257 x 1003 keeps 8 of 148 SMs busy there.  Here a CTA forms
// a 32 x 32 tile on the CUDA cores from the caller's own tensors, whatever their alignment.  Its 1024 threads
// fetch 256 entries of the contraction at once, all loads in flight (a product of that depth then waits for memory once);
// 16 groups of 64 threads take a sixteenth of them each, 4 x 4 results per thread (with 2 x 2 it was shared
// memory that took the time: 30 us for the gradient of 67 x 257 x 1003), and a thread per result adds up the groups,
// in order.
#include <atomic>

#include "head_small.h"

#include "common.cuh"
#include "launch.h"

namespace spr {

namespace {

constexpr int kTile = 32;
constexpr int kDepth = 256;              // entries of the contraction in shared memory
constexpr int kGroups = 16;
constexpr int kSmallThreads = 1024;
constexpr int kLoads = kTile * kDepth / kSmallThreads;
constexpr int kPitch = kTile + 4;        // rows of 16-byte vectors
constexpr int kOperand = kDepth * kPitch;
constexpr size_t kSmallSmem = 2 * kOperand * sizeof(float);
static_assert(kGroups * kTile * kTile <= 2 * kOperand, "the groups' sums take the operands' place");

// A thread's elements of a 32 (m) x 256 (k) piece, u = 0 .. 7: neighbouring threads follow the contiguous axis, across
// it in runs of eight so that the copies to shared memory meet no bank twice.
template <bool ACROSS>
struct Place {
    int m, k;
    __device__ __forceinline__ explicit Place(int t) : m(ACROSS ? t & 31 : (t & 31) >> 3), k(ACROSS ? t >> 5 : 8 * (t >> 5) + (t & 7)) {}
    __device__ __forceinline__ int mu(int u) const { return ACROSS ? m : m + 4 * u; }
    __device__ __forceinline__ int ku(int u) const { return ACROSS ? k + 32 * u : k; }
};
// Entries k0 .. k0 + depth - 1 of the contraction.  Every address is inside the operand (ms, depth >= 1; operands have less
// than 2^31 elements), so that all loads are issued at once; what does not count is dropped behind them.  Where `live` is
// given, entry k counts only if live[k] is a token of the vocabulary.
template <bool ACROSS>
__device__ __forceinline__ void fetch(const SmallOperand &o, int m0, int ms, int k0, int depth, const int32_t *live, int V,
                                      float (&x)[kLoads])
{
    const Place<ACROSS> p(threadIdx.x);
    const int stride = (int)(ACROSS ? o.sk : o.sm), rest = ms - m0;
    const float *base = o.p + (ACROSS ? (int64_t)k0 * o.sk + m0 + min(p.m, rest - 1) : (int64_t)m0 * o.sm + k0 + min(p.k, depth - 1));
#pragma unroll
    for (int u = 0; u < kLoads; ++u) x[u] = base[(ACROSS ? min(p.ku(u), depth - 1) : min(p.mu(u), rest - 1)) * stride];
    if (live) {
        int tok[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) tok[u] = live[k0 + min(p.ku(u), depth - 1)];
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (tok[u] < 0 || tok[u] >= V) x[u] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
        if (p.ku(u) >= depth || p.mu(u) >= rest) x[u] = 0.f;
}
template <bool ACROSS>
__device__ __forceinline__ void put(float *s, const float (&x)[kLoads])
{
    const Place<ACROSS> p(threadIdx.x);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) s[p.ku(u) * kPitch + p.mu(u)] = x[u];
}

template <int MODE>
__global__ void __launch_bounds__(kSmallThreads) small_kernel(const SmallParams prm)
{
    extern __shared__ __align__(16) float smem[];
    float *sa = smem, *sb = smem + kOperand;
    pdl_trigger();
    int tile = blockIdx.x;
    const int first = prm.job[0].tiles_m * prm.job[0].tiles_n * prm.job[0].splits;      // CTAs of the first product
    const bool second = tile >= first;
    if (second) tile -= first;
    const SmallJob &j = prm.job[second ? 1 : 0];
    const int tiles = j.tiles_m * j.tiles_n, split = tile / tiles;
    tile -= split * tiles;
    const int m0 = (tile / j.tiles_n) * kTile, n0 = (tile % j.tiles_n) * kTile;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int per = (j.K + j.splits - 1) / j.splits;
    const int k_lo = min(j.K, split * per), k_hi = min(j.K, k_lo + per);
    const int rounds = (k_hi - k_lo + kDepth - 1) / kDepth, depth = rounds ? (k_hi - k_lo + rounds - 1) / rounds : 0;
    // 4 x 4 results of a group: rows 4 ty .. + 3, columns 4 tx .. + 3
    const int g = t >> 6, ty = (t >> 3) & 7, tx = t & 7;
    float c[4][4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[r][e] = 0.f;
    constexpr bool kBAcross = MODE == SMALL_OUT;
    const bool a_across = MODE == SMALL_OUT && j.a_across;
    float xa[kLoads], xb[kLoads];
    auto fetch_a = [&](int k, int n) {
        if (a_across) fetch<true>(j.a, m0, j.rows, k, n, nullptr, 0, xa);
        else fetch<false>(j.a, m0, j.rows, k, n, nullptr, 0, xa);
    };
    if (rounds) fetch<kBAcross>(j.b, n0, j.cols, k_lo, depth, j.live, prm.V, xb);
    if (MODE == SMALL_OUT) pdl_wait();        // the first operand is the kernel's before this one
    if (rounds) fetch_a(k_lo, depth);
    for (int k0 = k_lo; k0 < k_hi; k0 += depth) {
        if (k0 > k_lo) __syncthreads();
        if (a_across) put<true>(sa, xa);
        else put<false>(sa, xa);
        put<kBAcross>(sb, xb);
        __syncthreads();
        const int here = min(depth, k_hi - k0), next = min(depth, k_hi - k0 - depth);
        if (next > 0) {
            fetch_a(k0 + depth, next);
            fetch<kBAcross>(j.b, n0, j.cols, k0 + depth, next, j.live, prm.V, xb);
        }
        const int share = (here + kGroups - 1) / kGroups, i1 = min(here, (g + 1) * share);
#pragma unroll 4
        for (int i = g * share; i < i1; ++i) {
            const float4 a = *reinterpret_cast<const float4 *>(sa + i * kPitch + 4 * ty);
            const float4 b = *reinterpret_cast<const float4 *>(sb + i * kPitch + 4 * tx);
            const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) c[r][e] = fmaf(av[r], bv[e], c[r][e]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
        *reinterpret_cast<float4 *>(smem + (g * kTile + 4 * ty + r) * kTile + 4 * tx) = make_float4(c[r][0], c[r][1], c[r][2], c[r][3]);
    __syncthreads();
    float x = smem[t];               // row `warp`, column `lane` of the tile
#pragma unroll
    for (int i = 1; i < kGroups; ++i) x += smem[i * kTile * kTile + t];
    if (MODE == SMALL_OUT && j.splits > 1) {
        // the CTA that takes the tile's last ticket adds the splits' sums up, in order
        __shared__ int last;
        j.acc[((int64_t)split * tiles + tile) * kSmallThreads + t] = x;
        __threadfence();
        __syncthreads();
        if (t == 0) last = take_ticket(&j.tickets[tile], j.splits);
        __syncthreads();
        if (!last) return;
        __threadfence();
        const float *from = j.acc + (int64_t)tile * kSmallThreads + t;
        x = __ldcg(from);
#pragma unroll 8
        for (int s = 1; s < j.splits; ++s) x += __ldcg(from + (int64_t)s * tiles * kSmallThreads);
    }
    const int row = m0 + warp, col = n0 + lane;
    if (row >= j.rows) return;       // a whole warp
    if (MODE == SMALL_STATS) {
        // (max, sum of exp) over the tile's columns
        float m = col < j.cols ? x : neg_inf();
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        float s = col < j.cols ? ex2((x - (m == neg_inf() ? 0.f : m)) * kLog2e) : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) j.part[(int64_t)row * j.tiles_n + n0 / kTile] = make_float2(m, s);
    } else if (MODE == SMALL_DLOGITS) {
        const int tok = j.targets[row];
        const bool keep = tok >= 0 && tok < prm.V;
        if (tok >= prm.V && n0 == 0 && lane == 0) raise_status(prm.status, SPR_ERR_BAD_TOKEN);
        const float lse = keep ? j.lse[row] : 0.f, w = keep ? j.grad_loss[row] : 0.f;
        if (col < j.cols) j.d[(int64_t)row * j.d_pitch + col] = keep ? w * expf(x - lse) - (col == tok ? w : 0.f) : 0.f;
    } else if (col < j.cols) {
        j.out[(int64_t)row * j.out_pitch + col] = x;
    }
}

template <int MODE>
cudaError_t launch_mode(const SmallParams &prm, unsigned ctas, bool behind, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(small_kernel<MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallSmem);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = kSmallSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = behind ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, small_kernel<MODE>, prm);
}

}  // namespace

cudaError_t launch_small(SmallMode mode, SmallParams &prm, int njobs, cudaStream_t st)
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
    case SMALL_STATS: return launch_mode<SMALL_STATS>(prm, (unsigned)ctas, false, st);
    case SMALL_DLOGITS: return launch_mode<SMALL_DLOGITS>(prm, (unsigned)ctas, false, st);
    default: return launch_mode<SMALL_OUT>(prm, (unsigned)ctas, true, st);
    }
}

}  // namespace spr
