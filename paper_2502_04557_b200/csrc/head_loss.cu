// Softmax cross entropy of hidden states under a vocabulary head, its gradient, and training
// labels of the verifier from the hidden states and heads of two models - logits are never kept.
//
// With l = H W^T (H [N,d] hidden states, W [V,d] head, as in nn.Linear):
//   lse_i = log sum_v exp(l_iv),  loss_i = lse_i - l_{i,t_i}
//   D_iv = g_i (exp(l_iv - lse_i) - [v = t_i]),  dH = D W,  dW = D^T H
//   log p(x_i) = l_{i,x_i} - lse_i
// The products run on CTA pairs (head_gemm.cu).  Forward: one product whose epilogue leaves (max,
// sum of exp) per row and 128 columns, then a CTA per row that merges them and forms the target's
// logit as a dot product of its own - N rows of W, nothing beside the product, and exact to a few
// units of fp32 however the product's accumulator rounds.  Backward: the vocabulary goes by in
// pieces; a piece's D is kept in the workspace (one or two bf16 parts, three for fp32), and one launch
// then adds D W to dH and writes the piece's rows of dW.  Small fp32 problems and a handful of tokens take
// kernels of their own on the CUDA cores (head_small.cu, head_stream.cu; see small_head() and stream_head()).
//
// D is kept in bf16, in two parts for few tokens (see d_parts()); sums over D are held in fp32 throughout.
#include <string.h>

#include "common.cuh"
#include "head_gemm.h"
#include "head_small.h"
#include "head_stream.h"
#include "host_util.h"
#include "launch.h"

namespace spr {

namespace {

constexpr int kHeadMaxLambdas = 8;
// Blocks of 64 that an accumulator takes at most (head_gemm.cu): it truncates, up to 2^-23 of the running sum per 16 elements.
// A sum that is rounded to bf16 (2^-8 at most) may be low by 1/16 of that rounding at the very most, 2^-12: 512 blocks.  (All of
// a contraction of 2^20 tokens came out 1.4e-3 low.)  A logit behind an exponential counts by its absolute error: 64 blocks leave
// at most 3e-5 of it, 6e-4 of D for a logit of 20 (65536 columns in one accumulator: 1.8e-3 low).  For row statistics
// the contraction is cut into chunks of one length, at most 8: what truncation takes off grows with the length (N(0, 9)
// logits: a log-sum-exp is 2.2e-7 of itself low with 8, 1.2e-7 with 4), and so does the rate (4096x2048x128256: 1570 us
// with 8, 1728 with 4).
constexpr int kChunkStats = 8, kChunkStatsLeast = 2, kChunkF32 = 2, kChunkLogits = 64, kChunkOut = 512;
constexpr size_t kPieceBytes = (size_t)256 << 20;        // D of one vocabulary piece (see pieces())

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// ---------------------------------------------------------------- operands in tensor-core form
// fp32 and rows that are not a multiple of 16 bytes are copied into [rows, parts * pitch] bf16, pitch
// a multiple of 64, zeros behind column d.  Rows whose target is negative or outside the
// vocabulary are zeroed, so that whatever a padded row holds (infinities, NaN) reaches no sum.
template <typename T>
__global__ void __launch_bounds__(256) head_pack_kernel(const T *src, int64_t rows, int d, int pitch,
                                                        const int32_t *targets, int V, __nv_bfloat16 *dst, int *status)
{
    constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    const int groups = pitch / 8;
    const int64_t n = rows * groups;
    const bool vec = sizeof(T) == 4 ? d % 4 == 0 : d % 8 == 0;      // whole 16-byte vectors (the base is aligned)
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = i / groups;
        const int c = (int)(i - r * groups) * 8;
        const T *p = src + r * d + c;
        bool keep = true;
        if (targets) {
            const int t = targets[r];
            keep = t >= 0 && t < V;
            if (t >= V && c == 0) raise_status(status, SPR_ERR_BAD_TOKEN);
        }
        float x[8];
        if (keep && vec && c + 8 <= d) {
            if (sizeof(T) == 4) {
                const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
                x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
            } else {
                const uint4 a = *reinterpret_cast<const uint4 *>(p);
                const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[2 * e] = __uint_as_float(w[e] << 16);
                    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = keep && c + e < d ? (float)p[e] : 0.f;
        }
        __nv_bfloat16 *q = dst + r * (int64_t)(kParts * pitch) + c;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t *>(&b);
                x[2 * e] -= __low2float(b);
                x[2 * e + 1] -= __high2float(b);
            }
            *reinterpret_cast<uint4 *>(q + (int64_t)part * pitch) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// ---------------------------------------------------------------- row statistics -> outputs
struct HeadRow {
    const void *hidden, *W;
    const float2 *part;      // [N, parts]: (max, sum of exp) per 128 columns
    int d, parts;
};

constexpr int kRowThreads = 128;         // one CTA per row: its loads are all in flight at once

// log-sum-exp of row i; the result is that of thread 0
__device__ __forceinline__ double row_lse(const HeadRow &h, int64_t i, float2 *smem)
{
    const float2 *p = h.part + i * h.parts;
    const int tid = threadIdx.x;
    MS a = {neg_inf(), 0.f};
    for (int t0 = 0; t0 < h.parts; t0 += 8 * kRowThreads) {
        float2 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int t = t0 + k * kRowThreads + tid;
            x[k] = p[min(t, h.parts - 1)];        // unconditional: eight loads in flight
            if (t >= h.parts) x[k] = make_float2(neg_inf(), 0.f);
        }
        float m = a.m;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, x[k].x);
        const float ref = m == neg_inf() ? 0.f : m;
        float s = a.s * ex2((a.m - ref) * kLog2e);
#pragma unroll
        for (int k = 0; k < 8; ++k) s += x[k].y * ex2((x[k].x - ref) * kLog2e);
        a.m = m;
        a.s = s;
    }
    a = warp_ms(a);
    if ((tid & 31) == 0) smem[tid >> 5] = make_float2(a.m, a.s);
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int w = 1; w < kRowThreads / 32; ++w) a = ms_merge(a, MS{smem[w].x, smem[w].y});
    }
    __syncthreads();
    return (double)a.m + (double)logf(a.s);
}
// hidden_i . W_t: a thread adds fp32 products (eight of bf16, exact in fp32), the threads are added up in
// double; the result is that of thread 0
template <typename T>
__device__ __forceinline__ double row_logit(const HeadRow &h, int64_t i, int t, double *smem)
{
    constexpr int N = 16 / (int)sizeof(T);
    const T *a = static_cast<const T *>(h.hidden) + i * h.d, *b = static_cast<const T *>(h.W) + (int64_t)t * h.d;
    const int tid = threadIdx.x;
    double s = 0.0;
    if (h.d % N == 0) {
#pragma unroll 4
        for (int c = tid * N; c < h.d; c += kRowThreads * N) {
            const uint4 x = *reinterpret_cast<const uint4 *>(a + c), y = *reinterpret_cast<const uint4 *>(b + c);
            const uint32_t u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
            float f = 0.f;
            if (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) f = fmaf(__uint_as_float(u[e]), __uint_as_float(v[e]), f);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f = fmaf(__uint_as_float(u[e] << 16), __uint_as_float(v[e] << 16), f);
                    f = fmaf(__uint_as_float(u[e] & 0xffff0000u), __uint_as_float(v[e] & 0xffff0000u), f);
                }
            }
            s += (double)f;
        }
    } else {
#pragma unroll 4
        for (int c = tid; c < h.d; c += kRowThreads) s += (double)((float)a[c] * (float)b[c]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((tid & 31) == 0) smem[tid >> 5] = s;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int w = 1; w < kRowThreads / 32; ++w) s += smem[w];
    }
    __syncthreads();
    return s;
}

__device__ __forceinline__ bool gave_up(const int *status) { return *reinterpret_cast<const volatile int *>(status) == SPR_ERR_TIMEOUT; }

template <typename T>
__global__ void __launch_bounds__(kRowThreads) head_finish_kernel(const HeadRow h, int V, const int32_t *targets, float *loss,
                                                                  float *lse, int *status)
{
    __shared__ double sums[kRowThreads / 32];
    __shared__ float2 stats[kRowThreads / 32];
    const int64_t i = blockIdx.x;
    const int t = targets[i];
    const bool live = t >= 0 && t < V;
    const double at = live ? row_logit<T>(h, i, t, sums) : 0.0;       // before the product: it may still be running
    pdl_wait();
    const double z = row_lse(h, i, stats);
    if (threadIdx.x != 0) return;
    float l = 0.f, zf = (float)z;
    if (live) {
        l = (float)(z - at);
        if (l < 0.f) l = 0.f;        // -log p is not negative: rounding alone can make it so (NaN stays)
    } else if (t >= V) {
        l = -1.f;
        raise_status(status, SPR_ERR_BAD_TOKEN);
    }
    if (gave_up(status)) l = zf = __int_as_float(0x7fc00000);
    loss[i] = l;
    if (lse) lse[i] = zf;
}

struct HeadLabels {
    int n_lambda;
    float lambdas[kHeadMaxLambdas];
    uint8_t *labels;     // [n_lambda, N]
    float *ratio;        // [N] or null
};
template <typename T>
__global__ void __launch_bounds__(kRowThreads) head_labels_kernel(const HeadRow p, const HeadRow q, int64_t N, int V,
                                                                  const int32_t *tokens, const HeadLabels out, int *status)
{
    __shared__ double sums[kRowThreads / 32];
    __shared__ float2 stats[kRowThreads / 32];
    __shared__ double answer;
    const int64_t i = blockIdx.x;
    const int x = tokens[i];
    const bool valid = x >= 0 && x < V;
    double at = 0.0;
    if (valid) {
        at = row_logit<T>(q, i, x, sums);
        at -= row_logit<T>(p, i, x, sums);
    }
    pdl_wait();
    if (valid) {
        const double zp = row_lse(p, i, stats), zq = row_lse(q, i, stats);
        if (threadIdx.x == 0) answer = gave_up(status) ? (double)__int_as_float(0x7fc00000) : exp(at - (zq - zp));
    } else if (threadIdx.x == 0) {
        answer = -1.0;
        raise_status(status, SPR_ERR_BAD_TOKEN);
    }
    __syncthreads();
    const int l = threadIdx.x;
    if (l < out.n_lambda) out.labels[(int64_t)l * N + i] = (valid && answer <= (double)out.lambdas[l]) ? 1 : 0;
    if (l == 0 && out.ratio) out.ratio[i] = (float)answer;
}

// out[r, c] = sum over the slices: 32 groups of four columns per CTA and round; each of eight warps adds up
// every eighth slice, eight loads at a time, and the eight sums are added in order
template <typename T>
__global__ void __launch_bounds__(256) head_sum_kernel(const float *acc, int slices, int64_t stride, int pitch, int64_t rows,
                                                       int d, T *out)
{
    __shared__ float4 sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int groups = (d + 3) / 4;
    const int64_t n = rows * groups;
    pdl_wait();
    for (int64_t i0 = (int64_t)blockIdx.x * 32; i0 < n; i0 += (int64_t)gridDim.x * 32) {
        const int64_t i = min(i0 + lane, n - 1);
        const int64_t r = i / groups;
        const int c = (int)(i - r * groups) * 4;
        const float *p = acc + r * pitch + c;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = warp; k0 < slices; k0 += 64) {
            float4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = *reinterpret_cast<const float4 *>(p + min(k0 + 8 * k, slices - 1) * stride);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool there = k0 + 8 * k < slices;
                s.x += there ? x[k].x : 0.f;
                s.y += there ? x[k].y : 0.f;
                s.z += there ? x[k].z : 0.f;
                s.w += there ? x[k].w : 0.f;
            }
        }
        __syncthreads();
        sums[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && i0 + lane < n) {
#pragma unroll
            for (int k = 1; k < 8; ++k) {
                const float4 x = sums[k][lane];
                s = make_float4(s.x + x.x, s.y + x.y, s.z + x.z, s.w + x.w);
            }
            const float v[4] = {s.x, s.y, s.z, s.w};
            T *o = out + r * d + c;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < d) o[e] = (T)v[e];
        }
    }
}

// ---------------------------------------------------------------- workspace
bool needs_pack(int d, int dt) { return dt == SPR_F32 || d % 8 != 0; }
int parts(int dt) { return dt == SPR_F32 ? 3 : 1; }
// Parts that D is kept in.  Rounded to bf16 it brings the error of a gradient from that of rounding the result,
// 0.0017, to 0.0024 where there are many tokens.  With few of them the rounding of the targets' entries does not average
// out (measured up to 0.0026 of 9 or 128 tokens, against 0.0017 with two parts), and a second part of the contraction
// is beside sweeps over W and dW (64x768x50257 86 -> 104 us, 128x4096x32000 222 -> 280 us; 256x768x50257 would take 117
// for 88).
constexpr int kTwoPartTokens = 128;
int d_parts(int64_t N, int dt) { return dt == SPR_F32 ? 3 : N <= kTwoPartTokens ? 2 : 1; }
size_t packed_bytes(int64_t rows, int d, int dt) { return 2 * (size_t)rows * parts(dt) * (size_t)round_up(d, 64); }

// Whether an fp32 problem is small enough for tiles of 32 x 32 on the CUDA cores (see small_head()).
double small_limit(bool grad) { return (grad ? 0.75 : 1.0) * (1 << 27); }
bool small_size(bool grad, int64_t N, int d, int64_t V)
{
    return (double)round_up(N, kSmallTile) * (double)round_up(V, kSmallTile) * (d + 200.0) <= small_limit(grad);
}
// A handful of tokens: passes over W as it is (head_stream.cu), one for every eight tokens.  fp32: up to eight tokens,
// whatever the size, and up to 24 (16 for the gradient, which has a thread per four columns: from 512 columns) where W
// has 2^24 elements; bf16: up to four, two for the gradient where TMA can take the rows.  Measured (us, passes / tensor
// cores, loss and gradient):
//   d = 2048, V = 32000   f32 N = 8 82 / 293 and 218 / 730, N = 16 163 / 274 and 579 / 730, N = 24 243 / 275 and 878 / 734
//                         bf16 N = 1 27 / 46 and 79 / 139, N = 2 29 / 44 and 85 / 134, N = 4 37 / 40 and 121 / 129
//   d = 960, V = 116326   f32 N = 9 190 / 518 and 844 / 1347, N = 32 loss 480 / 465
//   d = 256, V = 70000    f32 N = 16 54 / 91 and 384 / 240;  V = 20000: N = 24 40 / 40 and 187 / 100
//   d = 768, V = 50257    bf16 N = 2 22 / 28 and 86 / 86, N = 4 28 / 28 and 110 / 87
//   d = 1001, V = 32000   bf16 N = 4 41 / 53 and 131 / 183
// One pass / tiles of head_small.cu: f32 4x256x1000 5.4 / 8.2 and 9 / 16.8, 8x64x500 5.3 / 6.8 and 11 / 11.7, 8x1024x512
// 14 / 18 and 24 / 37, 1x768x1000 6.3 / 15 and 10 / 41.
constexpr int kMostLoss = 24, kMostGrad = 16;
bool stream_head(bool grad, int64_t N, int d, int64_t V, int dt)
{
    int64_t most = grad && d % 8 == 0 ? 2 : 4;
    if (dt == SPR_F32) {
        const bool passes = V * d >= (1 << 24) && (!grad || d >= 512) && !small_size(grad, N, d, V);
        most = !passes ? kStreamTokens : grad ? kMostGrad : kMostLoss;
    }
    return N <= most && stream_fits(grad, (int)N, d, dt == SPR_F32);
}
// tokens of pass i
int pass_tokens(int N, int i) { return N - i * kStreamTokens < kStreamTokens ? N - i * kStreamTokens : kStreamTokens; }
// More fp32 tokens go to the CUDA cores where that is less than 2^27 multiply-adds, 3/4 of it for the gradient
// (head_small.cu: whole tiles of 32 x 32, each of which costs what 200 entries of its contraction do); above that the six
// bf16 products on the tensor cores are faster.  Measured (us, CUDA cores / tensor cores), below: loss 67x257x1003
// 10 / 21.5, 64x256x4000 15 / 19.5, 128x512x1000 13 / 28, 9x1024x2000 19 / 46, 300x64x1000 16 / 13; gradient 67x257x1003
// 24.5 / 56, 128x512x1000 44 / 61, 200x100x1000 23 / 46, 9x1024x2000 88 / 85.  Above: loss 64x512x4000 29 / 29, 256x128x2000
// 23 / 15; gradient 64x256x4000 60 / 58, 9x256x8000 83 / 59, 256x128x4000 103 / 57.  (bf16: 16x256x4000 11 / 9 and
// worse from there.)
bool small_head(bool grad, int64_t N, int d, int64_t V, int dt)
{
    return dt == SPR_F32 && !stream_head(grad, N, d, V, dt) && small_size(grad, N, d, V);
}
// dH's contraction over the vocabulary there: 256 of it per CTA
int small_splits(int V) { return (int)(ceil_div(V, 256) < 64 ? ceil_div(V, 256) : 64); }

struct HeadLossWs {
    size_t hidden, W;     // packed operands (0 bytes where the caller's tensors serve)
    size_t part;          // float2 [N, tiles]
};
// pair: on CTA pairs whatever the sizes
HeadLossWs head_loss_layout(Carver &c, int64_t N, int d, int V, int dt, bool pair = false)
{
    HeadLossWs w;
    if (!pair && small_head(false, N, d, V, dt)) {
        w.hidden = w.W = 0;
        w.part = c.take_data(8 * (size_t)N * (size_t)ceil_div(V, kSmallTile));
        return w;
    }
    if (!pair && stream_head(false, N, d, V, dt)) {
        w.hidden = w.W = 0;
        w.part = c.take_data(8 * (size_t)N * (size_t)stream_ctas(false, (int)N, d, V));
        return w;
    }
    w.hidden = c.take_data(needs_pack(d, dt) ? packed_bytes(N, d, dt) : 0);
    w.W = c.take_data(needs_pack(d, dt) ? packed_bytes(V, d, dt) : 0);
    w.part = c.take_data(16 * (size_t)N * (size_t)ceil_div(V, kPairTile));
    return w;
}

// How the vocabulary is cut.  A piece's D takes about 256 MB, so that the workspace does not grow with
// N V, but has at least 8192 columns: dH is read and written once per piece, which a contraction that
// deep hides.  The pieces are of one width, a multiple of the tile.
struct Pieces {
    int width, count;
    int kb_per, splits;   // dH = D W: the contraction over a piece is cut into `splits` ranges
};
Pieces pieces(int64_t N, int d, int V, int dt)
{
    Pieces p;
    int64_t most = (int64_t)(kPieceBytes / (2 * (size_t)d_parts(N, dt) * (size_t)N)) / kPairTile * kPairTile;
    if (most < 8192) most = 8192;
    p.count = (int)ceil_div(V, most);
    p.width = (int)round_up(ceil_div(V, p.count), kPairTile);
    p.count = (int)ceil_div(V, p.width);
    // dH has few tiles with a long contraction, dW many with a short one, in one launch: dH is cut so
    // that every one of the 74 pairs has one item of it, and dW evens them out
    const int64_t kb_v = ceil_div(p.count > 1 ? p.width : V, kPairBlockK);
    int64_t s = 74 / (ceil_div(N, kPairTile) * ceil_div(d, kPairTile));
    if (s > kb_v / 4) s = kb_v / 4;
    if (s < 1) s = 1;
    p.kb_per = (int)ceil_div(kb_v, s);
    p.splits = (int)ceil_div(kb_v, p.kb_per);
    return p;
}

struct HeadGradWs {
    size_t hidden;        // packed hidden states, rows without a target zeroed
    size_t W;             // packed head (0 bytes where the caller's serves)
    size_t dlogits;       // bf16 [N, parts * width]
    size_t acc;           // float [splits, N, round_up(d, 64)], where dH takes more than one launch or range
    size_t tickets;       // int32 per tile of dH (ticket zone; CUDA cores only)
};
HeadGradWs head_grad_layout(Carver &c, int64_t N, int d, int V, int dt)
{
    HeadGradWs w;
    if (small_head(true, N, d, V, dt)) {
        const size_t tiles = (size_t)ceil_div(N, kSmallTile) * (size_t)ceil_div(d, kSmallTile);
        w.hidden = w.W = 0;
        w.tickets = c.take_tickets(tiles);
        w.dlogits = c.take_data(4 * (size_t)N * (size_t)V);       // fp32 here
        w.acc = c.take_data(4 * 1024 * tiles * (size_t)small_splits(V));
        return w;
    }
    if (stream_head(true, N, d, V, dt)) {
        w.hidden = w.W = w.tickets = w.dlogits = 0;
        const int64_t tokens = N < kStreamTokens ? N : kStreamTokens;      // of a pass
        w.acc = c.take_data(4 * (size_t)stream_ctas(true, (int)N, d, V) * (size_t)tokens * (size_t)round_up(d, 64));
        return w;
    }
    const Pieces p = pieces(N, d, V, dt);
    w.tickets = 0;
    w.hidden = c.take_data(packed_bytes(N, d, dt));
    w.W = c.take_data(needs_pack(d, dt) ? packed_bytes(V, d, dt) : 0);
    w.dlogits = c.take_data(2 * (size_t)N * d_parts(N, dt) * (size_t)p.width);
    w.acc = c.take_data(p.count * p.splits > 1 ? 4 * (size_t)p.splits * (size_t)N * (size_t)round_up(d, 64) : 0);
    return w;
}

// ---------------------------------------------------------------- workspace that serves every number of tokens up to N
// What a call takes does not simply grow with its tokens: few of them keep D in two parts, dH's contraction is cut into fewer
// ranges as the tiles of tokens become more, pieces are of whole tiles, and kernels change.  The size that is asked for is
// the most of any call up to N, so that a short batch at the end of a run fits where the others did.
struct Need {
    size_t tickets, data;
    template <typename F>
    void at_least(F layout)
    {
        Carver c;
        c.tickets = c.data = 0;
        c.tickets_end = c.data_end = ~(size_t)0;
        layout(c);
        if (c.tickets > tickets) tickets = c.tickets;
        if (c.data > data) data = c.data;
    }
};
// Numbers of tokens up to N at which a kernel other than the pair's needs most: every handful, and the most that tiles on the
// CUDA cores are taken for (what those need grows with the tokens).  f(n) for each of them, and for N.
template <typename F>
void for_token_counts(bool grad, int64_t N, int d, int64_t V, F f)
{
    for (int64_t n = 1; n <= N && n <= kMostLoss; ++n) f(n);
    const double tile = (double)kSmallTile * (double)round_up(V, kSmallTile) * (d + 200.0);
    const int64_t most = kSmallTile * (int64_t)(small_limit(grad) / tile);
    if (most >= 1) f(most < N ? most : N);
    f(N);
}
Need head_loss_need(int64_t N, int d, int V, int dt)
{
    Need need = {0, 0};
    for_token_counts(false, N, d, V, [&](int64_t n) { need.at_least([&](Carver &c) { head_loss_layout(c, n, d, V, dt); }); });
    return need;
}
// D of a piece: 2 parts n width bytes, and width is at most V and at most 256 MB of it or 8192 columns
size_t most_dlogits(int64_t n, int parts, int V)
{
    const size_t row = 2 * (size_t)parts * (size_t)n, all = row * (size_t)round_up(V, kPairTile);
    const size_t piece = row * 8192 > kPieceBytes ? row * 8192 : kPieceBytes;
    return all < piece ? all : piece;
}
// the layout of the gradient on CTA pairs with the most of every part for any number of tokens up to N
void most_pair_grad(Carver &c, int64_t N, int d, int V, int dt)
{
    const int64_t few = N < kTwoPartTokens ? N : kTwoPartTokens;
    size_t D = most_dlogits(N, d_parts(N, dt), V);
    const size_t D_few = most_dlogits(few, d_parts(few, dt), V);
    if (D_few > D) D = D_few;
    const bool cut = pieces(N, d, V, dt).count > 1 || pieces(few, d, V, dt).count > 1;
    int64_t rows = cut ? N : 0;        // of acc: N in one range, or those of every number of tiles of tokens that has more
    const int64_t kb = ceil_div(V, kPairBlockK), across = ceil_div(d, kPairTile);
    for (int64_t m = 1; m <= ceil_div(N, kPairTile); ++m) {
        int64_t s = 74 / (m * across);
        if (s > kb / 4) s = kb / 4;
        if (s < 2) break;
        if (!cut) s = ceil_div(kb, ceil_div(kb, s));      // as pieces() rounds it; of a piece's blocks it is at most s
        const int64_t n = m * kPairTile < N ? m * kPairTile : N;
        if (n * s > rows) rows = n * s;
    }
    c.take_data(packed_bytes(N, d, dt));
    c.take_data(needs_pack(d, dt) ? packed_bytes(V, d, dt) : 0);
    c.take_data(D);
    c.take_data(4 * (size_t)rows * (size_t)round_up(d, 64));
}
Need head_grad_need(int64_t N, int d, int V, int dt)
{
    Need need = {0, 0};
    for_token_counts(true, N, d, V, [&](int64_t n) { need.at_least([&](Carver &c) { head_grad_layout(c, n, d, V, dt); }); });
    if (!small_head(true, N, d, V, dt) && !stream_head(true, N, d, V, dt))
        need.at_least([&](Carver &c) { most_pair_grad(c, N, d, V, dt); });
    return need;
}

// A ratio is as exact as what truncation takes off both log-sum-exps alike (see verifier_labels_head).  The kernels on the CUDA
// cores round to nearest: where one model of bf16 would be theirs and the other the tensor pipe's, the pipe takes both.
// (4 tokens, 20480 and 2048 columns, V = 32000: ratios off by 3.9e-6 on two kernels at 310 us, by 0.8e-6 on one at 293 us, and by as
// much on two with chunks of two blocks at 505 us.)
bool both_on_pairs(int64_t N, int dp, int dq, int V, int dt)
{
    return dt != SPR_F32 && stream_head(false, N, dp, V, dt) != stream_head(false, N, dq, V, dt);
}
struct HeadLabelsWs {
    HeadLossWs p, q;
};
HeadLabelsWs head_labels_layout(Carver &c, int64_t N, int dp, int dq, int V, int dt)
{
    const bool pair = both_on_pairs(N, dp, dq, V, dt);
    HeadLabelsWs w;
    w.p = head_loss_layout(c, N, dp, V, dt, pair);
    w.q = head_loss_layout(c, N, dq, V, dt, pair);
    return w;
}
Need head_labels_need(int64_t N, int dp, int dq, int V, int dt)
{
    Need need = {0, head_loss_need(N, dp, V, dt).data + head_loss_need(N, dq, V, dt).data};
    for (int64_t n = 1; n <= N && n <= kStreamTokens; ++n) need.at_least([&](Carver &c) { head_labels_layout(c, n, dp, dq, V, dt); });
    return need;
}

// ---------------------------------------------------------------- launches
// A kernel that starts while the one before it in the stream ends (programmatic dependent launch) and
// calls pdl_wait() before it touches what that one writes.
template <typename... P, typename... A>
cudaError_t launch_behind(void (*kernel)(P...), int64_t ctas, int threads, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

template <typename T>
cudaError_t pack_rows(const void *src, int64_t rows, int d, const int32_t *targets, int V, void *dst, int *status, cudaStream_t st)
{
    const int pitch = (int)round_up(d, 64);
    const int64_t blocks = ceil_div(rows * (pitch / 8), 256);
    head_pack_kernel<T><<<(unsigned)(blocks < 148 * 16 ? blocks : 148 * 16), 256, 0, st>>>(
        static_cast<const T *>(src), rows, d, pitch, targets, V, static_cast<__nv_bfloat16 *>(dst), status);
    return cudaGetLastError();
}
cudaError_t pack(const void *src, int64_t rows, int d, int dt, const int32_t *targets, int V, void *dst, int *status, cudaStream_t st)
{
    return dt == SPR_F32 ? pack_rows<float>(src, rows, d, targets, V, dst, status, st)
                         : pack_rows<__nv_bfloat16>(src, rows, d, targets, V, dst, status, st);
}
// a packed operand, or the caller's tensor where it already has that form
PairOperand packed_operand(const void *base, int64_t rows, int d, int dt)
{
    const int64_t pitch = parts(dt) * round_up(d, 64);
    return PairOperand{base, rows, pitch, pitch};
}
PairOperand plain_operand(const void *base, int64_t rows, int d) { return PairOperand{base, rows, d, d}; }

// over k elements, in ranges of kb_per blocks (0: in one)
void contraction(PairJob &j, int64_t k, int dt, int kb_per, int most)
{
    j.kb = (int)ceil_div(k, kPairBlockK);
    j.kb_per = kb_per ? kb_per : j.kb;
    j.splits = (int)ceil_div(j.kb, j.kb_per);
    j.nprod = dt == SPR_F32 ? 6 : 1;
    // bf16: chunks of one length
    j.kc = dt == SPR_F32 ? kChunkF32 : (int)ceil_div(j.kb_per, ceil_div(j.kb_per, most));
}

// job and operands of the row statistics of hidden [N,d] under W [V,d]; packs what has to be packed
cudaError_t stats_job(PairJob &j, PairOperand &a, PairOperand &b, const void *hidden, const void *W, int64_t N, int d, int V,
                      int dt, void *ws, const HeadLossWs &lay, cudaStream_t st)
{
    cudaError_t e = cudaSuccess;
    if (needs_pack(d, dt)) {
        void *h = at<char>(ws, lay.hidden), *w = at<char>(ws, lay.W);
        e = pack(hidden, N, d, dt, nullptr, 0, h, nullptr, st);
        if (e == cudaSuccess) e = pack(W, V, d, dt, nullptr, 0, w, nullptr, st);
        a = packed_operand(h, N, d, dt);
        b = packed_operand(w, V, d, dt);
    } else {
        a = plain_operand(hidden, N, d);
        b = plain_operand(W, V, d);
    }
    memset(&j, 0, sizeof j);
    contraction(j, d, dt, 0, kChunkStats);
    j.tiles_m = (int)ceil_div(N, kPairTile);
    j.tiles_n = (int)ceil_div(V, kPairTile);
    j.a_seg = j.b_seg = (int)round_up(d, 64);
    j.rows = N;
    j.cols = V;
    j.part = at<float2>(ws, lay.part);
    return e;
}

// the same on the CUDA cores
void small_stats_job(SmallJob &j, const void *hidden, const void *W, int N, int d, int V, const float2 *part)
{
    j.a = SmallOperand{static_cast<const float *>(hidden), d, 1};
    j.b = SmallOperand{static_cast<const float *>(W), d, 1};
    j.rows = N;
    j.cols = V;
    j.K = d;
    j.part = const_cast<float2 *>(part);
}

// d_hidden [N, d] = the sum over acc [slices, N, round_up(d, 64)]
cudaError_t sum_slices(const float *acc, int slices, int N, int d, int dt, void *d_hidden, cudaStream_t st)
{
    const int pitch = (int)round_up(d, 64);
    const int64_t blocks = ceil_div((int64_t)N * ((d + 3) / 4), 32);
    const unsigned ctas = (unsigned)(blocks < 148 * 16 ? blocks : 148 * 16);
    return dt == SPR_F32 ? launch_behind(head_sum_kernel<float>, ctas, 256, st, acc, slices, (int64_t)N * pitch, pitch, (int64_t)N, d,
                                         static_cast<float *>(d_hidden))
                         : launch_behind(head_sum_kernel<__nv_bfloat16>, ctas, 256, st, acc, slices, (int64_t)N * pitch, pitch,
                                         (int64_t)N, d, static_cast<__nv_bfloat16 *>(d_hidden));
}

StreamParams stream_params(const void *hidden, const void *W, int N, int d, int V, int dt)
{
    StreamParams p;
    memset(&p, 0, sizeof p);
    p.hidden = hidden;
    p.W = W;
    p.N = N;
    p.d = d;
    p.V = V;
    p.pitch = (int)round_up(d, 64);
    p.vec = (size_t)d * elem_size(dt) % 16 == 0;      // the bases are 16-byte aligned
    return p;
}

// row statistics of one model by whichever kernel the sizes call for, except the tensor cores'
cudaError_t other_stats(HeadRow &r, int N, int V, int dt, int *status, cudaStream_t st)
{
    if (stream_head(false, N, r.d, V, dt)) {
        r.parts = stream_ctas(false, N, r.d, V);
        cudaError_t e = cudaSuccess;
        for (int i = 0; i * kStreamTokens < N && e == cudaSuccess; ++i) {
            const int64_t n0 = i * kStreamTokens;
            const char *h = static_cast<const char *>(r.hidden) + n0 * r.d * elem_size(dt);
            StreamParams p = stream_params(h, r.W, pass_tokens(N, i), r.d, V, dt);
            p.part = const_cast<float2 *>(r.part) + n0 * r.parts;
            p.ctas = r.parts;
            e = launch_stream(false, dt == SPR_F32, p, st);
        }
        return e;
    }
    SmallParams sp;
    memset(&sp, 0, sizeof sp);
    sp.V = V;
    sp.status = status;
    small_stats_job(sp.job[0], r.hidden, r.W, N, r.d, V, r.part);
    r.parts = (int)ceil_div(V, kSmallTile);
    return launch_small(SMALL_STATS, sp, 1, st);
}

// head_loss_grad on the CUDA cores: D in fp32, then both products in one launch
cudaError_t small_grad(const void *hidden, const void *W, const int32_t *targets, const float *lse, const float *grad_loss, int N,
                       int d, int V, void *d_hidden, void *d_W, float *D, float *acc, int *tickets, int *status, cudaStream_t st)
{
    SmallParams sp;
    memset(&sp, 0, sizeof sp);
    sp.V = V;
    sp.status = status;
    SmallJob &j = sp.job[0];
    small_stats_job(j, hidden, W, N, d, V, nullptr);
    j.d = D;
    j.d_pitch = V;
    j.targets = targets;
    j.lse = lse;
    j.grad_loss = grad_loss;
    cudaError_t e = launch_small(SMALL_DLOGITS, sp, 1, st);
    if (e != cudaSuccess) return e;
    memset(sp.job, 0, sizeof sp.job);
    int jobs = 0;
    if (d_hidden) {               // dH [N, d] = D [N, V] W [V, d]: the longer contraction first
        SmallJob &h = sp.job[jobs++];
        h.a = SmallOperand{D, V, 1};
        h.b = SmallOperand{static_cast<const float *>(W), 1, d};
        h.rows = N;
        h.cols = d;
        h.K = V;
        h.splits = small_splits(V);
        h.acc = acc;
        h.tickets = tickets;
        h.out = static_cast<float *>(d_hidden);
        h.out_pitch = d;
    }
    if (d_W) {                    // dW [V, d] = D^T [V, N] H [N, d]
        SmallJob &w = sp.job[jobs++];
        w.a = SmallOperand{D, 1, V};
        w.a_across = 1;
        w.b = SmallOperand{static_cast<const float *>(hidden), 1, d};
        w.live = targets;         // a row without a target may hold anything
        w.rows = V;
        w.cols = d;
        w.K = N;
        w.out = static_cast<float *>(d_W);
        w.out_pitch = d;
    }
    return launch_small(SMALL_OUT, sp, jobs, st);
}

bool head_sizes_ok(int64_t N, int d, int V) { return N >= 0 && d > 0 && d <= (1 << 20) && V > 0 && V <= (1 << 30); }

}  // namespace

size_t head_loss_ws_bytes(int64_t N, int d, int V, int dt)
{
    if (N <= 0 || !head_sizes_ok(N, d, V)) return 0;
    const Need need = head_loss_need(N, d, V, dt);
    return ws_bytes_for(need.tickets, need.data);
}
size_t head_grad_ws_bytes(int64_t N, int d, int V, int dt)
{
    if (N <= 0 || !head_sizes_ok(N, d, V)) return 0;
    const Need need = head_grad_need(N, d, V, dt);
    return ws_bytes_for(need.tickets, need.data);
}
size_t head_labels_ws_bytes(int64_t N, int dp, int dq, int V, int dt)
{
    if (N <= 0 || !head_sizes_ok(N, dp, V) || !head_sizes_ok(N, dq, V)) return 0;
    const Need need = head_labels_need(N, dp, dq, V, dt);
    return ws_bytes_for(need.tickets, need.data);
}

}  // namespace spr

using namespace spr;

extern "C" {

int head_loss(const void *hidden, const void *W, const int32_t *targets, int N, int d, int V, int dt, float *loss, float *lse,
              void *ws, size_t ws_bytes, void *cuda_stream)
{
    if (!dtype_ok(dt)) return SPR_ERR_UNSUPPORTED;
    if (!head_sizes_ok(N, d, V)) return SPR_ERR_INVALID_ARG;
    if (N == 0) return SPR_OK;
    if (!hidden || !W || !targets || !loss) return SPR_ERR_INVALID_ARG;
    if (!aligned(hidden, 16) || !aligned(W, 16) || !aligned(targets, 4) || !aligned(loss, 4) || (lse && !aligned(lse, 4)))
        return SPR_ERR_INVALID_ARG;
    Carver cv = carve(ws_bytes);
    const HeadLossWs lay = head_loss_layout(cv, N, d, V, dt);
    if (!ws || !aligned(ws, 256) || !cv.fits()) return SPR_ERR_WORKSPACE;
    int rc = device_supported();
    if (rc != SPR_OK) return rc;

    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    PairParams prm;
    memset(&prm, 0, sizeof prm);
    prm.status = at<int>(ws, 0);
    HeadRow h = {hidden, W, at<float2>(ws, lay.part), d, 0};
    cudaError_t e;
    if (small_head(false, N, d, V, dt) || stream_head(false, N, d, V, dt)) {
        e = other_stats(h, N, V, dt, prm.status, st);
    } else {
        PairOperand a, b;
        e = stats_job(prm.job[0], a, b, hidden, W, N, d, V, dt, ws, lay, st);
        if (e == cudaSuccess) e = launch_pair(PAIR_STATS, dt == SPR_F32, prm, 1, &a, &b, needs_pack(d, dt), st);
        h.parts = 2 * prm.job[0].tiles_n;
    }
    if (e == cudaSuccess) {
        e = dt == SPR_F32 ? launch_behind(head_finish_kernel<float>, N, kRowThreads, st, h, V, targets, loss, lse, prm.status)
                          : launch_behind(head_finish_kernel<__nv_bfloat16>, N, kRowThreads, st, h, V, targets, loss, lse, prm.status);
    }
    return finish(e);
}

int head_loss_grad(const void *hidden, const void *W, const int32_t *targets, const float *lse, const float *grad_loss, int N,
                   int d, int V, int dt, void *d_hidden, void *d_W, void *ws, size_t ws_bytes, void *cuda_stream)
{
    if (!dtype_ok(dt)) return SPR_ERR_UNSUPPORTED;
    if (!head_sizes_ok(N, d, V)) return SPR_ERR_INVALID_ARG;
    if (!d_hidden && !d_W) return SPR_ERR_INVALID_ARG;
    if ((d_hidden && !aligned(d_hidden, 16)) || (d_W && !aligned(d_W, 16))) return SPR_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (N == 0) {        // no samples: the head's gradient is zero
        if (!d_W) return SPR_OK;
        const int rc = device_supported();
        return rc != SPR_OK ? rc : finish(cudaMemsetAsync(d_W, 0, (size_t)V * d * elem_size(dt), st));
    }
    if (!hidden || !W || !targets || !lse || !grad_loss) return SPR_ERR_INVALID_ARG;
    if (!aligned(hidden, 16) || !aligned(W, 16) || !aligned(targets, 4) || !aligned(lse, 4) || !aligned(grad_loss, 4))
        return SPR_ERR_INVALID_ARG;
    Carver cv = carve(ws_bytes);
    const HeadGradWs lay = head_grad_layout(cv, N, d, V, dt);
    if (!ws || !aligned(ws, 256) || !cv.fits()) return SPR_ERR_WORKSPACE;
    int rc = device_supported();
    if (rc != SPR_OK) return rc;

    if (small_head(true, N, d, V, dt))
        return finish(small_grad(hidden, W, targets, lse, grad_loss, N, d, V, d_hidden, d_W, at<float>(ws, lay.dlogits),
                                 at<float>(ws, lay.acc), at<int>(ws, lay.tickets), at<int>(ws, 0), st));
    const bool f32 = dt == SPR_F32;
    const size_t es = elem_size(dt);
    if (stream_head(true, N, d, V, dt)) {
        cudaError_t e = cudaSuccess;
        for (int i = 0; i * kStreamTokens < N && e == cudaSuccess; ++i) {
            const int64_t n0 = i * kStreamTokens;
            StreamParams p = stream_params(static_cast<const char *>(hidden) + n0 * d * es, W, pass_tokens(N, i), d, V, dt);
            p.targets = targets + n0;
            p.lse = lse + n0;
            p.grad_loss = grad_loss + n0;
            p.d_hidden = d_hidden ? static_cast<char *>(d_hidden) + n0 * d * es : nullptr;
            p.d_W = d_W;
            p.add = i > 0;
            p.acc = at<float>(ws, lay.acc);      // of one pass after the other
            p.ctas = stream_ctas(true, N, d, V);
            p.status = at<int>(ws, 0);
            e = launch_stream(true, f32, p, st);
            if (e == cudaSuccess && d_hidden) e = sum_slices(p.acc, p.ctas, p.N, d, dt, p.d_hidden, st);
        }
        return finish(e);
    }
    const Pieces pc = pieces(N, d, V, dt);
    const int dp = (int)round_up(d, 64);
    void *hp = at<char>(ws, lay.hidden);
    cudaError_t e = pack(hidden, N, d, dt, targets, V, hp, at<int>(ws, 0), st);
    PairOperand wv = plain_operand(W, V, d);
    if (e == cudaSuccess && needs_pack(d, dt)) {
        e = pack(W, V, d, dt, nullptr, 0, at<char>(ws, lay.W), nullptr, st);
        wv = packed_operand(at<char>(ws, lay.W), V, d, dt);
    }
    const PairOperand hv = packed_operand(hp, N, d, dt);
    const int dparts = d_parts(N, dt);
    const PairOperand dv = {at<char>(ws, lay.dlogits), N, (int64_t)dparts * pc.width, (int64_t)dparts * pc.width};
    for (int i = 0; i < pc.count && e == cudaSuccess; ++i) {
        const int v0 = i * pc.width, width = V - v0 < pc.width ? V - v0 : pc.width;
        PairOperand wp = wv;      // the piece's rows of W
        wp.base = static_cast<const char *>(wv.base) + 2 * (size_t)v0 * (size_t)wv.pitch;
        wp.rows = width;
        PairParams prm;
        memset(&prm, 0, sizeof prm);
        prm.status = at<int>(ws, 0);
        PairJob &j = prm.job[0];
        contraction(j, d, dt, 0, kChunkLogits);
        j.tiles_m = (int)ceil_div(N, kPairTile);
        j.tiles_n = (int)ceil_div(width, kPairTile);
        j.a_seg = j.b_seg = dp;
        j.rows = N;
        j.cols = width;
        j.dlogits = at<__nv_bfloat16>(ws, lay.dlogits);
        j.dl_pitch = dv.pitch;
        j.dl_parts = dparts;
        j.dl_seg = pc.width;
        j.v0 = v0;
        j.V = V;
        j.lse = lse;
        j.grad_loss = grad_loss;
        j.targets = targets;
        e = launch_pair(PAIR_DLOGITS, f32, prm, 1, &hv, &wp, true, st);
        if (e != cudaSuccess) break;

        memset(&prm, 0, sizeof prm);
        prm.status = at<int>(ws, 0);
        PairOperand a[2], b[2];
        int jobs = 0;
        if (d_hidden) {           // dH [N, d] += D [N, width] W [width, d]
            PairJob &h = prm.job[jobs];
            contraction(h, width, dt, pc.kb_per, kChunkOut);
            if (dparts == 2) h.nprod = 2;
            h.tiles_m = (int)ceil_div(N, kPairTile);
            h.tiles_n = (int)ceil_div(d, kPairTile);
            h.b_across = 1;
            h.a_seg = pc.width;
            h.b_seg = dp;
            h.rows = N;
            h.cols = d;
            if (pc.count * pc.splits > 1) {
                h.acc = at<float>(ws, lay.acc);
                h.acc_pitch = dp;
                h.acc_stride = (int64_t)N * dp;
                h.add_acc = i > 0;
            }
            if (pc.splits == 1 && i == pc.count - 1) {
                h.out = d_hidden;
                h.out_pitch = d;
            }
            a[jobs] = dv;
            b[jobs] = wp;
            ++jobs;
        }
        if (d_W) {                // dW [width, d] = D^T [width, N] H [N, d]
            PairJob &w = prm.job[jobs];
            contraction(w, N, dt, 0, kChunkOut);
            if (dparts == 2) w.nprod = 2;
            w.tiles_m = (int)ceil_div(width, kPairTile);
            w.tiles_n = (int)ceil_div(d, kPairTile);
            w.a_across = w.b_across = 1;
            w.a_seg = pc.width;
            w.b_seg = dp;
            w.rows = width;
            w.cols = d;
            w.out = static_cast<char *>(d_W) + (size_t)v0 * d * es;
            w.out_pitch = d;
            a[jobs] = dv;
            b[jobs] = hv;
            ++jobs;
        }
        e = launch_pair(PAIR_OUT, f32, prm, jobs, a, b, true, st);
    }
    if (e == cudaSuccess && d_hidden && pc.splits > 1) e = sum_slices(at<float>(ws, lay.acc), pc.splits, N, d, dt, d_hidden, st);
    return finish(e);
}

int verifier_labels_head(const void *p_hidden, const void *p_W, int dp, const void *q_hidden, const void *q_W, int dq,
                         const int32_t *draft_tokens, int N, int V, int dt, const float *lambdas, int n_lambda,
                         uint8_t *labels, float *ratio, void *ws, size_t ws_bytes, void *cuda_stream)
{
    if (!dtype_ok(dt)) return SPR_ERR_UNSUPPORTED;
    if (!head_sizes_ok(N, dp, V) || !head_sizes_ok(N, dq, V) || n_lambda <= 0 || n_lambda > kHeadMaxLambdas || !lambdas)
        return SPR_ERR_INVALID_ARG;
    if (N == 0) return SPR_OK;
    if (!p_hidden || !p_W || !q_hidden || !q_W || !draft_tokens || !labels) return SPR_ERR_INVALID_ARG;
    if (!aligned(p_hidden, 16) || !aligned(p_W, 16) || !aligned(q_hidden, 16) || !aligned(q_W, 16) ||
        !aligned(draft_tokens, 4) || (ratio && !aligned(ratio, 4)))
        return SPR_ERR_INVALID_ARG;
    Carver cv = carve(ws_bytes);
    const HeadLabelsWs lay = head_labels_layout(cv, N, dp, dq, V, dt);
    if (!ws || !aligned(ws, 256) || !cv.fits()) return SPR_ERR_WORKSPACE;
    int rc = device_supported();
    if (rc != SPR_OK) return rc;

    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    PairParams prm;
    memset(&prm, 0, sizeof prm);
    prm.status = at<int>(ws, 0);
    PairOperand a[2], b[2];
    HeadRow p = {p_hidden, p_W, at<float2>(ws, lay.p.part), dp, 0}, q = {q_hidden, q_W, at<float2>(ws, lay.q.part), dq, 0};
    cudaError_t e = cudaSuccess;
    int pairs = 0;
    const bool on_pairs = both_on_pairs(N, dp, dq, V, dt);
    // the longer products first
    for (int i = 0; i < 2 && e == cudaSuccess; ++i) {
        const bool is_p = (i == 0) == (dp >= dq);
        HeadRow &r = is_p ? p : q;
        if (!on_pairs && (small_head(false, N, r.d, V, dt) || stream_head(false, N, r.d, V, dt))) {
            e = other_stats(r, N, V, dt, prm.status, st);
        } else {
            e = stats_job(prm.job[pairs], a[pairs], b[pairs], r.hidden, r.W, N, r.d, V, dt, ws, is_p ? lay.p : lay.q, st);
            ++pairs;
            r.parts = 2 * (int)ceil_div(V, kPairTile);
        }
    }
    if (dt != SPR_F32 && pairs == 2) {
        // Chunks of one length in both products, so that truncation does the same to both log-sum-exps and cancels in the
        // ratio (768 and 1536 elements: off by 3e-7, where chunks of their own leave 1.3e-6).  A narrow model's chunk is all of its
        // blocks, and sets the length for the other down to two: with at least five, 128 and 256 elements were off by
        // 2.4e-6 instead of 2e-7, 64 and 576 by 4.2e-6 instead of 1.1e-6 (plain fp32: 0.5e-6 and 0.9e-6).  That is 48.7 ->
        // 52.5 us for the former (1024 tokens, V = 32000), 64 -> 79 us for the latter and 132 -> 170 us for 128 and 2048, whose
        // ratios were off by 2.9e-6; a single block as the least would take 64 and 2048 from 136 to 268 us.
        int kc = prm.job[0].kc < prm.job[1].kc ? prm.job[0].kc : prm.job[1].kc;
        if (kc < kChunkStatsLeast) kc = kChunkStatsLeast;
        prm.job[0].kc = prm.job[1].kc = kc;
    }
    if (e == cudaSuccess && pairs) e = launch_pair(PAIR_STATS, dt == SPR_F32, prm, pairs, a, b, false, st);
    if (e == cudaSuccess) {
        HeadLabels out;
        memset(&out, 0, sizeof out);
        out.n_lambda = n_lambda;
        for (int l = 0; l < n_lambda; ++l) out.lambdas[l] = lambdas[l];
        out.labels = labels;
        out.ratio = ratio;
        e = dt == SPR_F32 ? launch_behind(head_labels_kernel<float>, N, kRowThreads, st, p, q, (int64_t)N, V, draft_tokens, out, prm.status)
                          : launch_behind(head_labels_kernel<__nv_bfloat16>, N, kRowThreads, st, p, q, (int64_t)N, V, draft_tokens, out, prm.status);
    }
    return finish(e);
}

}  // extern "C"
