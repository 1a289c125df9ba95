// Hidden states kept in 8 bits: a shared power-of-two exponent per block of 32 elements and a
// signed byte per element.
//
//   e = max(floor(log2 max|x|) - 6, -126),  q = clamp(round-to-even(x 2^-e), -127, 127),  x ~ q 2^e
//
// The largest element of a block lies in [64, 128) 2^e, so an element is off by at most half a step
// 2^e (a whole step above 127.5, where q is clamped): between 1/128 and 1/256 of the block's
// largest magnitude.  Scales are powers of two so that nothing but q is rounded: 2^-e x is exact, and
// q 2^e is a bf16 number (7 bits), so states unpacked to bf16 are what the packed ones stand for,
// bit for bit.  Both directions are bound by memory: es + 1 + 1/32 bytes per element (measured, 2^18 x 2048 bf16: packing
// 287 us, 5.7 TB/s; unpacking 243 us, 6.7 TB/s; 2^17 x 2048 fp32 packing 202 us, 6.7 TB/s; 4096 x 2048 bf16 6.3 and 4.7 us).
#include "common.cuh"
#include "host_util.h"
#include "launch.h"

namespace spr {

namespace {

constexpr int kPackBlock = 32;           // elements per exponent
constexpr int kBadBlock = -128;          // exponent byte of a block that held an infinity or NaN
constexpr int kChunk = 256;              // elements a warp takes at a time: 8 per lane
constexpr int kPackWarps = 8;

// 8 consecutive elements, zeros behind column d
__device__ __forceinline__ void load8(const float *p, int left, bool vec, float (&x)[8])
{
    if (vec && left >= 8) {
        const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p + 4));
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < left ? p[e] : 0.f;
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, int left, bool vec, float (&x)[8])
{
    if (vec && left >= 8) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < left ? __bfloat162float(p[e]) : 0.f;
    }
}
__device__ __forceinline__ void store8(float *p, int left, bool vec, const float (&x)[8])
{
    if (vec && left >= 8) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = x[e];
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, int left, bool vec, const float (&x)[8])
{
    if (vec && left >= 8) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
            w[e] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = __float2bfloat16(x[e]);
    }
}

// 8 elements of a block whose largest magnitude has the bits `top`: their bytes and the exponent byte.
// x 2^-e is exact; with 1.5 2^23 added it is rounded to even at the units, and the low byte of the sum is
// the byte wanted.
__device__ __forceinline__ uint2 quantise(const float (&x)[8], uint32_t top, int &e2)
{
    const bool bad = top >= 0x7f800000u;
    e2 = max((int)(top >> 23) - 133, -126);
    const float scale = __int_as_float((127 - e2) << 23);
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(fmaf(x[e], scale, 12582912.f));
    // above 127.5 2^e a byte would be 128: only a block whose largest element starts 1.1111111 1 can hold one
    if (__any_sync(__activemask(), (top & 0x7fffffu) >= 0x7f0000u)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = min(max(b[e], 0x4b400000u - 127u), 0x4b400000u + 127u);
    }
    uint2 q;
    q.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    q.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    if (bad) {
        q = make_uint2(0u, 0u);
        e2 = kBadBlock;
    }
    return q;
}
// byte + 128 as the low mantissa byte of 2^23; less 2^23 + 128 that is q, and q 2^e is exact.  (With the subtraction behind
// the scaling, as (2^23 + 128) 2^e, it would be beyond fp32 from e = 105 on.)
__device__ __forceinline__ void dequantise(uint2 q, int e2, float (&x)[8])
{
    const float scale = e2 == kBadBlock ? __int_as_float(0x7fc00000) : __int_as_float((e2 + 127) << 23);
    const uint32_t w[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x[e] = (__uint_as_float(__byte_perm(w[e >> 2], 0x4b000000u, 0x7440 + (e & 3))) - 8388736.f) * scale;
}

// ---------------------------------------------------------------- any width and alignment
// chunk (row r, elements [c, c + 256)) of a warp; a lane has 8 elements, four lanes a block
template <typename T>
__global__ void __launch_bounds__(32 * kPackWarps) pack8_any_kernel(const T *src, int64_t N, int d, int pitch, bool vec, uint8_t *dst)
{
    const int lane = threadIdx.x & 31;
    const int per_row = (d + kChunk - 1) / kChunk;
    const int64_t chunks = N * per_row, stride = (int64_t)gridDim.x * kPackWarps;
    for (int64_t w = (int64_t)blockIdx.x * kPackWarps + (threadIdx.x >> 5); w < chunks; w += stride) {
        const int64_t r = w / per_row;
        const int c = (int)(w - r * per_row) * kChunk + lane * 8;
        float x[8];
        load8(src + r * d + c, d - c, vec, x);
        // largest magnitude of the block, as bits: infinities and NaN lie above all numbers
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        int e2;
        const uint2 q = quantise(x, top, e2);
        uint8_t *row = dst + r * pitch;
        if (c + 8 <= d) {
            *reinterpret_cast<uint2 *>(row + c) = q;
        } else if (c < d) {
            for (int e = 0; c + e < d; ++e) row[c + e] = (uint8_t)((e < 4 ? q.x : q.y) >> (8 * (e & 3)));
        }
        if ((lane & 3) == 0 && c < d) row[d + c / kPackBlock] = (uint8_t)e2;
        if (c < d && c + 8 >= d)       // the lane with the last elements clears the row's padding
            for (int b = d + (d + kPackBlock - 1) / kPackBlock; b < pitch; ++b) row[b] = 0;
    }
}

template <typename T>
__global__ void __launch_bounds__(32 * kPackWarps) unpack8_any_kernel(const uint8_t *src, int64_t N, int d, int pitch, bool vec, T *dst)
{
    const int lane = threadIdx.x & 31;
    const int per_row = (d + kChunk - 1) / kChunk;
    const int64_t chunks = N * per_row, stride = (int64_t)gridDim.x * kPackWarps;
    for (int64_t w = (int64_t)blockIdx.x * kPackWarps + (threadIdx.x >> 5); w < chunks; w += stride) {
        const int64_t r = w / per_row;
        const int c = (int)(w - r * per_row) * kChunk + lane * 8;
        if (c >= d) continue;
        const uint8_t *row = src + r * pitch;      // 8 bytes at c: inside the row, whose pitch is a multiple of 16
        float x[8];
        dequantise(*reinterpret_cast<const uint2 *>(row + c), reinterpret_cast<const signed char *>(row)[d + c / kPackBlock], x);
        store8(dst + r * d + c, d - c, vec, x);
    }
}

// ---------------------------------------------------------------- aligned rows of whole blocks
// A CTA of (x, y) threads takes kRows rows per thread row at a time, so that as many loads per thread are in
// flight; a thread has 8 elements of each.  d is a multiple of 32 and rows are 16-byte aligned.
constexpr int kRows = 4;

template <typename T>
__global__ void __launch_bounds__(256) pack8_kernel(const T *src, int64_t N, int d, int pitch, uint8_t *dst)
{
    const int64_t r0 = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * kRows;
    const int nv = d / 8;
    for (int v0 = 0; v0 < nv; v0 += blockDim.x) {
        const int v = v0 + threadIdx.x;
        float x[kRows][8];
#pragma unroll
        for (int k = 0; k < kRows; ++k)     // the last row and vector again where there is none: loads without a branch
            load8(src + min(r0 + k, N - 1) * d + min(v, nv - 1) * 8, 8, true, x[k]);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[k][e]) & 0x7fffffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            int e2;
            const uint2 q = quantise(x[k], top, e2);
            if (v >= nv || r0 + k >= N) continue;
            uint8_t *row = dst + (r0 + k) * pitch;
            *reinterpret_cast<uint2 *>(row + v * 8) = q;
            if ((v & 3) == 0) row[d + v / 4] = (uint8_t)e2;
            if (v == nv - 1)
                for (int b = d + d / kPackBlock; b < pitch; ++b) row[b] = 0;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) unpack8_kernel(const uint8_t *src, int64_t N, int d, int pitch, T *dst)
{
    const int64_t r0 = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * kRows;
    const int nv = d / 8;
    for (int v = threadIdx.x; v < nv; v += blockDim.x) {
        uint2 q[kRows];
        int e2[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const uint8_t *row = src + min(r0 + k, N - 1) * pitch;
            q[k] = *reinterpret_cast<const uint2 *>(row + v * 8);
            e2[k] = reinterpret_cast<const signed char *>(row)[d + v / 4];
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            float x[8];
            dequantise(q[k], e2[k], x);
            if (r0 + k < N) store8(dst + (r0 + k) * d + v * 8, 8, true, x);
        }
    }
}

unsigned any_ctas(int64_t N, int d)
{
    const int64_t want = (N * ((d + kChunk - 1) / kChunk) + kPackWarps - 1) / kPackWarps;
    return (unsigned)(want < 148 * 64 ? want : 148 * 64);
}
// (d >= 32) a thread per 8 elements of a row, as many rows side by side as 256 threads hold
dim3 row_threads(int d)
{
    const int x = d / 8 >= 256 ? 256 : (d / 8 + 31) / 32 * 32;
    return dim3((unsigned)x, (unsigned)(256 / x));
}
unsigned row_ctas(int64_t N, dim3 threads)
{
    const int64_t rows = (int64_t)threads.y * kRows;
    return (unsigned)((N + rows - 1) / rows);
}
bool whole_rows(const void *hidden, int64_t N, int d)
{
    return aligned(hidden, 16) && d % kPackBlock == 0 && N <= ((int64_t)1 << 32);
}

template <typename T>
cudaError_t pack_rows(const void *hidden, int64_t N, int d, void *packed, cudaStream_t st)
{
    const T *src = static_cast<const T *>(hidden);
    uint8_t *dst = static_cast<uint8_t *>(packed);
    if (whole_rows(hidden, N, d)) {
        const dim3 threads = row_threads(d);
        pack8_kernel<<<row_ctas(N, threads), threads, 0, st>>>(src, N, d, pack8_pitch(d), dst);
    } else
        pack8_any_kernel<<<any_ctas(N, d), 32 * kPackWarps, 0, st>>>(src, N, d, pack8_pitch(d), aligned(hidden, 16) && d % 8 == 0, dst);
    return cudaGetLastError();
}
template <typename T>
cudaError_t unpack_rows(const void *packed, int64_t N, int d, void *hidden, cudaStream_t st)
{
    const uint8_t *src = static_cast<const uint8_t *>(packed);
    T *dst = static_cast<T *>(hidden);
    if (whole_rows(hidden, N, d)) {
        const dim3 threads = row_threads(d);
        unpack8_kernel<<<row_ctas(N, threads), threads, 0, st>>>(src, N, d, pack8_pitch(d), dst);
    } else
        unpack8_any_kernel<<<any_ctas(N, d), 32 * kPackWarps, 0, st>>>(src, N, d, pack8_pitch(d), aligned(hidden, 16) && d % 8 == 0, dst);
    return cudaGetLastError();
}

int check_pack(const void *hidden, int64_t N, int d, int dt, const void *packed)
{
    if (!dtype_ok(dt)) return SPR_ERR_UNSUPPORTED;
    if (N < 0 || d <= 0 || d > (1 << 20)) return SPR_ERR_INVALID_ARG;
    if (N == 0) return SPR_OK;
    if (!hidden || !packed || !aligned(hidden, elem_size(dt)) || !aligned(packed, 16)) return SPR_ERR_INVALID_ARG;
    return device_supported();
}

}  // namespace

}  // namespace spr

using namespace spr;

extern "C" {

size_t spr_pack8_pitch(int d) { return d > 0 && d <= (1 << 20) ? (size_t)pack8_pitch(d) : 0; }

int hidden_pack8(const void *hidden, int64_t N, int d, int dt, void *packed, void *cuda_stream)
{
    const int rc = check_pack(hidden, N, d, dt, packed);
    if (rc != SPR_OK || N == 0) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return finish(dt == SPR_F32 ? pack_rows<float>(hidden, N, d, packed, st) : pack_rows<__nv_bfloat16>(hidden, N, d, packed, st));
}

int hidden_unpack8(const void *packed, int64_t N, int d, int dt, void *hidden, void *cuda_stream)
{
    const int rc = check_pack(hidden, N, d, dt, packed);
    if (rc != SPR_OK || N == 0) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return finish(dt == SPR_F32 ? unpack_rows<float>(packed, N, d, hidden, st) : unpack_rows<__nv_bfloat16>(packed, N, d, hidden, st));
}

}  // extern "C"
