// The vocabulary head for a handful of tokens: a pass over W for every eight of them.
//
// With so few rows a product reads W and does little with it: it is bound by memory, and the tensor-core
// kernels would lay out fp32 or unaligned heads in the workspace first, three to six times the traffic.
// Here the hidden states lie in shared memory as fp32 and W streams through registers as it is:
//   forward    a warp takes four rows of W at a time, a lane 16 bytes of each; the 4 x N logits are
//              formed by one scatter-reduction across the lanes, and every lane keeps (max, sum of exp) of its own
//   gradient   a CTA takes 32 rows: first their logits, hence D (in shared memory), as above; then a
//              thread per 16 bytes of columns reads the rows again (out of L2), writes dW = D^T H for them and adds
//              D W to its columns of dH, which it keeps in registers.  W is read from memory once, dW
//              written once: the floor.  The CTAs' dH are added up in order by the kernel behind.
// Measured (d = 2048, V = 32000): loss fp32 N = 1 46 us (5.7 TB/s), N = 8 82 us, bf16 N = 1 27 us; gradient fp32 N = 1 141 us,
// N = 8 218 us, bf16 N = 1 79 us.  The gradient's bytes alone are 81 and 41 us: with one CTA on an SM and a barrier between the logits
// of 32 rows and the products with them, the reads of one phase and the writes of the other overlap in part only.
// With more tokens it is the products of every vector of W with all of them.  A small head takes 4 to 7 us for
// the loss and 9 us for the gradient: launches.
#include <atomic>

#include "head_stream.h"

#include "common.cuh"
#include "launch.h"
#include "vocab_common.cuh"

namespace spr {

namespace {

constexpr int kStatWarps = 16;
constexpr int kGradThreads = 512, kGradWarps = kGradThreads / 32;
constexpr int kGradRows = 32;              // rows of W a CTA takes at a time

// hidden states as fp32 [NT][pitch], zeros behind column d, in rows past N and in rows without a target
template <typename T>
__device__ __forceinline__ void stage_hidden(const StreamParams &prm, int nt, float *h, bool masked)
{
    const T *src = static_cast<const T *>(prm.hidden);
    const int total = nt * prm.pitch;
    for (int i0 = threadIdx.x; i0 < total; i0 += 8 * blockDim.x) {
        float x[8];
        int tok[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {              // addresses that exist, all loads at once
            const int i = min(i0 + u * (int)blockDim.x, total - 1), n = i / prm.pitch, c = i - n * prm.pitch, m = min(n, prm.N - 1);
            x[u] = (float)src[(int64_t)m * prm.d + min(c, prm.d - 1)];
            tok[u] = masked ? prm.targets[m] : 0;
            if (n >= prm.N || c >= prm.d) tok[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i0 + u * (int)blockDim.x < total) h[i0 + u * (int)blockDim.x] = tok[u] >= 0 && tok[u] < prm.V ? x[u] : 0.f;
    }
}

// elements c .. of a row, zeros past d; CHANGED: by this call
template <typename T, bool CHANGED>
__device__ __forceinline__ uint4 load_vec(const T *row, int c, int d, bool vec)
{
    constexpr int N = Vec<T>::N;
    if (vec && CHANGED) return c < d ? *reinterpret_cast<const uint4 *>(row + c) : make_uint4(0u, 0u, 0u, 0u);
    if (vec) return c < d ? __ldg(reinterpret_cast<const uint4 *>(row + c)) : make_uint4(0u, 0u, 0u, 0u);
    T x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = c + e < d ? row[c + e] : (T)0.f;
    return *reinterpret_cast<const uint4 *>(x);
}

// v[R * NT] summed over the lanes: lane l gets the sum of value l >> (5 - log2(R NT))
template <int NV>
__device__ __forceinline__ float scatter_sum(float (&v)[NV], int lane)
{
    int n = NV;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (n > 1) {
            n /= 2;
#pragma unroll
            for (int i = 0; i < NV / 2; ++i) {
                if (i < n) {
                    const bool up = lane & o;
                    const float keep = up ? v[i + n] : v[i], send = up ? v[i] : v[i + n];
                    v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
            }
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        }
    }
    return v[0];
}
__host__ __device__ constexpr int log2i(int x) { return x <= 1 ? 0 : 1 + log2i(x / 2); }

// logits of R rows of W (row0, row0 + 1, ...) and NT tokens; the lane's is the one that scatter_sum gives it.  U vectors
// of every row are asked for at once, from addresses that are always inside the row: what does not exist is dropped
// behind the loads (loads that depend on a condition would wait for one another).
template <typename T, int NT, int R, int U>
__device__ __forceinline__ float row_logits(const StreamParams &prm, const float *h, int64_t row0, int lane)
{
    constexpr int N = Vec<T>::N;
    const T *w = static_cast<const T *>(prm.W);
    uint64_t acc[R * NT];
#pragma unroll
    for (int i = 0; i < R * NT; ++i) acc[i] = pack2(0.f, 0.f);
    const T *row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) row[r] = w + min(row0 + r, (int64_t)prm.V - 1) * prm.d;
    const int last = (prm.d - 1) / N * N;
    auto add = [&](const float (&f)[R][N], int c) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const float4 y = *reinterpret_cast<const float4 *>(h + n * prm.pitch + c + e);
                const uint64_t y0 = pack2(y.x, y.y), y1 = pack2(y.z, y.w);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    acc[r * NT + n] = fma2(pack2(f[r][e + 2], f[r][e + 3]), y1, fma2(pack2(f[r][e], f[r][e + 1]), y0, acc[r * NT + n]));
            }
        }
    };
    if (prm.vec) {
        for (int c = lane * N; c < prm.d; c += U * 32 * N) {
            uint4 x[U][R];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < R; ++r) x[u][r] = __ldg(reinterpret_cast<const uint4 *>(row[r] + min(c + u * 32 * N, last)));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (c + u * 32 * N > last)
#pragma unroll
                    for (int r = 0; r < R; ++r) x[u][r] = make_uint4(0u, 0u, 0u, 0u);
                float f[R][N];
#pragma unroll
                for (int r = 0; r < R; ++r) Vec<T>::unpack(x[u][r], f[r]);
                add(f, min(c + u * 32 * N, last));
            }
        }
    } else {
        for (int c = lane * N; c < prm.d; c += 32 * N) {
            float f[R][N];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < N; ++e) f[r][e] = (float)row[r][min(c + e, prm.d - 1)];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (c + e >= prm.d) f[r][e] = 0.f;
            add(f, c);
        }
    }
    float v[R * NT];
#pragma unroll
    for (int i = 0; i < R * NT; ++i) {
        float lo, hi;
        unpack2(acc[i], lo, hi);
        v[i] = lo + hi;
    }
    return scatter_sum<R * NT>(v, lane);
}

template <typename T, int NT>
__global__ void __launch_bounds__(32 * kStatWarps) stream_stats_kernel(const StreamParams prm)
{
    constexpr int R = 4, kShift = 5 - log2i(R * NT);
    extern __shared__ float4 hidden4[];
    float *h = reinterpret_cast<float *>(hidden4);
    __shared__ float2 part[kStatWarps][8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_trigger();
    stage_hidden<T>(prm, NT, h, false);
    __syncthreads();
    MS a = {neg_inf(), 0.f};
    const int idx = lane >> kShift, my_row = idx / NT;
    const int64_t stride = (int64_t)gridDim.x * kStatWarps * R;
    for (int64_t row0 = ((int64_t)blockIdx.x * kStatWarps + warp) * R; row0 < prm.V; row0 += stride) {
        const float l = row_logits<T, NT, R, NT <= 2 ? 4 : 2>(prm, h, row0, lane);
        if (row0 + my_row < prm.V) a = ms_merge(a, MS{l, 1.f});
    }
    // merge the four rows' slots of a token (the lanes that differ in the row bits), then the warps
#pragma unroll
    for (int o = NT << kShift; o < 32; o <<= 1) {
        MS b;
        b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
        b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
        a = ms_merge(a, b);
    }
    if (lane < (NT << kShift) && (lane & ((1 << kShift) - 1)) == 0) part[warp][idx] = make_float2(a.m, a.s);
    __syncthreads();
    const int n = threadIdx.x;
    if (n < prm.N) {
        MS s = {part[0][n].x, part[0][n].y};
#pragma unroll
        for (int w = 1; w < kStatWarps; ++w) s = ms_merge(s, MS{part[w][n].x, part[w][n].y});
        prm.part[(int64_t)n * gridDim.x + blockIdx.x] = make_float2(s.m, s.s);
    }
}

template <typename T, int NT>
__global__ void __launch_bounds__(kGradThreads, 1) stream_grad_kernel(const StreamParams prm)
{
    constexpr int N = Vec<T>::N, R = kGradRows / kGradWarps, kShift = 5 - log2i(R * NT);
    extern __shared__ float4 hidden4[];
    float *h = reinterpret_cast<float *>(hidden4);
    __shared__ __align__(16) float D[2][kGradRows][NT < 4 ? 4 : NT];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_trigger();
    stage_hidden<T>(prm, NT, h, true);
    // this lane's logit of a row: row idx / NT of the warp's, token idx % NT
    const int idx = lane >> kShift, my_row = idx / NT, my_tok = idx % NT;
    int tok = -1;
    if (my_tok < prm.N) tok = prm.targets[my_tok];
    const bool keep = tok >= 0 && tok < prm.V;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        for (int n = 0; n < prm.N; ++n)
            if (prm.targets[n] >= prm.V) raise_status(prm.status, SPR_ERR_BAD_TOKEN);
    }
    const float lse = keep ? prm.lse[my_tok] : 0.f, g = keep ? prm.grad_loss[my_tok] : 0.f;
    __syncthreads();
    const T *w = static_cast<const T *>(prm.W);
    T *dw = static_cast<T *>(prm.d_W);
    const int c0 = threadIdx.x * N;                       // this thread's columns
    const bool mine = c0 < prm.d;
    float hr[NT][N], acc[NT][N];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            hr[n][e] = mine ? h[n * prm.pitch + c0 + e] : 0.f;
            acc[n][e] = 0.f;
        }
    int buf = 0;
    for (int64_t base = (int64_t)blockIdx.x * kGradRows; base < prm.V; base += (int64_t)gridDim.x * kGradRows, buf ^= 1) {
        // the next rows are asked for as far as L2 while these are worked on
        const int64_t next = base + (int64_t)gridDim.x * kGradRows + threadIdx.x;
        if (threadIdx.x < kGradRows && prm.vec && next < prm.V)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(w + next * prm.d), "r"((uint32_t)(prm.d * sizeof(T)))
                         : "memory");
        const int64_t row = base + warp * R + my_row;
        const float l = row_logits<T, NT, R, NT <= 2 ? 4 : 2>(prm, h, base + warp * R, lane);
        if ((lane & ((1 << kShift) - 1)) == 0 && idx < R * NT)
            D[buf][warp * R + my_row][my_tok] = keep && row < prm.V ? g * expf(l - lse) - (row == tok ? g : 0.f) : 0.f;
        __syncthreads();          // D is there; the other buffer's readers are a barrier behind
        const int rows = (int)min((int64_t)kGradRows, prm.V - base);
        // Four rows of W at a time, all loads of them ahead of the stores (which might be to the same place for all the
        // compiler knows)
        for (int r0 = 0; mine && r0 < rows; r0 += 4) {
            uint4 x[4], before[4];
            if (sizeof(T) == 4 && dw && prm.add) {
#pragma unroll
                for (int i = 0; i < 4; ++i) before[i] = load_vec<T, true>(dw + (base + min(r0 + i, rows - 1)) * prm.d, c0, prm.d, prm.vec);
            }
            if (prm.d_hidden) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = load_vec<T, false>(w + (base + min(r0 + i, rows - 1)) * prm.d, c0, prm.d, prm.vec);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + i;
                if (r >= rows) break;
                float f[N];
                if (prm.d_hidden) Vec<T>::unpack(x[i], f);
                float o[N];
                if (sizeof(T) == 4 && dw && prm.add) {
                    Vec<T>::unpack(before[i], o);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) o[e] = 0.f;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float y = D[buf][r][n];
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        o[e] = fmaf(y, hr[n][e], o[e]);
                        if (prm.d_hidden) acc[n][e] = fmaf(y, f[e], acc[n][e]);
                    }
                }
                if (dw) {
                    T *p = dw + (base + r) * prm.d + c0;
                    __align__(16) T y[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) y[e] = (T)o[e];
                    if (prm.vec) {
                        *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(y);
                    } else {
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (c0 + e < prm.d) p[e] = y[e];
                    }
                }
            }
        }
    }
    if (prm.d_hidden && mine) {      // acc [cta][N][pitch]
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (n < prm.N)
#pragma unroll
                for (int e = 0; e < N; e += 4)
                    *reinterpret_cast<float4 *>(prm.acc + ((int64_t)blockIdx.x * prm.N + n) * prm.pitch + c0 + e) =
                        make_float4(acc[n][e], acc[n][e + 1], acc[n][e + 2], acc[n][e + 3]);
    }
}

// The attribute belongs to the kernel and the device, not to the call: it is set once, to the most that any call takes, so that
// host threads with states of different widths do not take shared memory from each other.
template <auto KERNEL>
cudaError_t start(const StreamParams &prm, int ctas, int threads, size_t smem, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kStreamSmem);
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    KERNEL<<<ctas, threads, smem, st>>>(prm);
    return cudaGetLastError();
}
template <typename T, int NT>
cudaError_t start_any(bool grad, const StreamParams &prm, int ctas, cudaStream_t st)
{
    const size_t smem = 4 * (size_t)NT * prm.pitch;
    return grad ? start<stream_grad_kernel<T, NT>>(prm, ctas, kGradThreads, smem, st)
                : start<stream_stats_kernel<T, NT>>(prm, ctas, 32 * kStatWarps, smem, st);
}
template <typename T>
cudaError_t start_typed(bool grad, const StreamParams &prm, int ctas, cudaStream_t st)
{
    if (prm.N <= 1) return start_any<T, 1>(grad, prm, ctas, st);
    if (prm.N <= 2) return start_any<T, 2>(grad, prm, ctas, st);
    if (prm.N <= 4) return start_any<T, 4>(grad, prm, ctas, st);
    if constexpr (sizeof(T) == 4) return start_any<T, 8>(grad, prm, ctas, st);
    return cudaErrorInvalidValue;          // bf16: at most four
}

}  // namespace

cudaError_t launch_stream(bool grad, bool f32, const StreamParams &prm, cudaStream_t st)
{
    return f32 ? start_typed<float>(grad, prm, prm.ctas, st) : start_typed<__nv_bfloat16>(grad, prm, prm.ctas, st);
}

}  // namespace spr
