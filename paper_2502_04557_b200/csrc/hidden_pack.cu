// Hidden states kept in 8 bits: a shared power-of-two exponent per block of 32 elements and a
// signed byte per element.
//
//   e = max(floor(log2 max|x|) - 6, -126),  q = clamp(round-to-even(x 2^-e), -127, 127),  x ~ q 2^e
//
// The largest element of a block lies in [64, 128) 2^e, so an element is off by at most half a step
// 2^e (a whole step above 127.5, where q is clamped): between 1/128 and 1/256 of the block's
// largest magnitude.  Scales are powers of two so that nothing but q is rounded: 2^-e x is exact, and
// q 2^e is a bf16 number (7 bits), so states unpacked to bf16 are what the packed ones stand for,
// bit for bit.  Both directions are bound by memory: es + 1 + 1/32 bytes per element.
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

// A warp takes chunks (row r, elements [c, c + 256)), kAhead of them at a time so that their loads are in
// flight together; a lane has 8 elements of each, four lanes a block.
constexpr int kAhead = 4;
struct Chunks {
    int64_t all, stride, at;       // chunks, and this warp's first and distance
    int per_row;
    __device__ Chunks(int64_t N, int d)
    {
        per_row = (d + kChunk - 1) / kChunk;
        all = N * per_row;
        stride = (int64_t)gridDim.x * kPackWarps;
        at = (int64_t)blockIdx.x * kPackWarps + (threadIdx.x >> 5);
    }
    __device__ void place(int64_t w, int64_t &r, int &c) const
    {
        if (all <= 0x7fffffff) {
            const uint32_t q = (uint32_t)w / (uint32_t)per_row;
            r = q;
            c = (int)((uint32_t)w - q * (uint32_t)per_row);
        } else {
            r = w / per_row;
            c = (int)(w - r * per_row);
        }
        c = c * kChunk + (int)(threadIdx.x & 31) * 8;
    }
};

template <typename T>
__global__ void __launch_bounds__(32 * kPackWarps) pack8_kernel(const T *src, int64_t N, int d, int pitch, bool vec, uint8_t *dst)
{
    const int lane = threadIdx.x & 31;
    const Chunks ch(N, d);
    for (int64_t w0 = ch.at; w0 < ch.all; w0 += kAhead * ch.stride) {
        float x[kAhead][8];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            int64_t r;
            int c;
            ch.place(min(w0 + k * ch.stride, ch.all - 1), r, c);
            load8(src + r * d + c, d - c, vec, x[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (w0 + k * ch.stride >= ch.all) break;
            int64_t r;
            int c;
            ch.place(w0 + k * ch.stride, r, c);
            // largest magnitude of the block, as bits: infinities and NaN lie above all numbers
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[k][e]) & 0x7fffffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const bool bad = top >= 0x7f800000u;
            const int e2 = bad ? 0 : max((int)(top >> 23) - 133, -126);
            const float scale = __int_as_float((127 - e2) << 23);
            uint32_t q[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // x 2^-e + 1.5 2^23 rounds to even at the units: the low byte of the sum is the byte wanted
                const float y = fminf(fmaxf(x[k][e] * scale, -127.f), 127.f) + 12582912.f;
                q[e >> 2] |= (__float_as_uint(y) & 255u) << (8 * (e & 3));
            }
            if (bad) q[0] = q[1] = 0u;
            uint8_t *row = dst + r * pitch;
            if (c + 8 <= d) {
                *reinterpret_cast<uint2 *>(row + c) = make_uint2(q[0], q[1]);
            } else if (c < d) {
                for (int e = 0; c + e < d; ++e) row[c + e] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
            }
            if ((lane & 3) == 0 && c < d) row[d + c / kPackBlock] = (uint8_t)(bad ? kBadBlock : e2);
            if (c < d && c + 8 >= d)       // the lane with the last elements clears the row's padding
                for (int b = d + (d + kPackBlock - 1) / kPackBlock; b < pitch; ++b) row[b] = 0;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(32 * kPackWarps) unpack8_kernel(const uint8_t *src, int64_t N, int d, int pitch, bool vec, T *dst)
{
    const Chunks ch(N, d);
    for (int64_t w0 = ch.at; w0 < ch.all; w0 += kAhead * ch.stride) {
        uint2 q[kAhead];
        int e2[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            int64_t r;
            int c;
            ch.place(min(w0 + k * ch.stride, ch.all - 1), r, c);
            const int at = min(c, d - 1);                  // lanes past the row's end load its last elements
            const uint8_t *row = src + r * pitch;          // 8 bytes from a multiple of 8: inside the row, whose pitch is one of 16
            q[k] = __ldcs(reinterpret_cast<const uint2 *>(row + (at & ~7)));
            e2[k] = reinterpret_cast<const signed char *>(row)[d + at / kPackBlock];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (w0 + k * ch.stride >= ch.all) break;
            int64_t r;
            int c;
            ch.place(w0 + k * ch.stride, r, c);
            const float scale = e2[k] == kBadBlock ? __int_as_float(0x7fc00000) : __int_as_float((e2[k] + 127) << 23);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)    // byte + 128 as the low mantissa byte of 2^23, which is then taken off
                x[e] = (__uint_as_float(__byte_perm((e < 4 ? q[k].x : q[k].y) ^ 0x80808080u, 0x4b000000u, 0x7440 + (e & 3))) - 8388736.f) * scale;
            if (c < d) store8(dst + r * d + c, d - c, vec, x);
        }
    }
}

// one round of kAhead chunks per warp where that fills the GPU, at most eight CTAs per SM
unsigned pack_ctas(int64_t N, int d)
{
    const int64_t chunks = N * ((d + kChunk - 1) / kChunk);
    const int64_t want = (chunks + kPackWarps - 1) / kPackWarps;       // one chunk per warp
    const int64_t rounds = (want + 148 * 8 * kAhead - 1) / (148 * 8 * kAhead);
    const int64_t ctas = (want + rounds * kAhead - 1) / (rounds * kAhead);
    return (unsigned)(want < 148 * 8 ? want : ctas < 148 * 4 ? 148 * 4 : ctas);
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
    const bool vec = aligned(hidden, 16) && d % 8 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SPR_F32)
        pack8_kernel<<<pack_ctas(N, d), 32 * kPackWarps, 0, st>>>(static_cast<const float *>(hidden), N, d, pack8_pitch(d), vec,
                                                                  static_cast<uint8_t *>(packed));
    else
        pack8_kernel<<<pack_ctas(N, d), 32 * kPackWarps, 0, st>>>(static_cast<const __nv_bfloat16 *>(hidden), N, d,
                                                                  pack8_pitch(d), vec, static_cast<uint8_t *>(packed));
    return finish(cudaGetLastError());
}

int hidden_unpack8(const void *packed, int64_t N, int d, int dt, void *hidden, void *cuda_stream)
{
    const int rc = check_pack(hidden, N, d, dt, packed);
    if (rc != SPR_OK || N == 0) return rc;
    const bool vec = aligned(hidden, 16) && d % 8 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SPR_F32)
        unpack8_kernel<<<pack_ctas(N, d), 32 * kPackWarps, 0, st>>>(static_cast<const uint8_t *>(packed), N, d, pack8_pitch(d),
                                                                    vec, static_cast<float *>(hidden));
    else
        unpack8_kernel<<<pack_ctas(N, d), 32 * kPackWarps, 0, st>>>(static_cast<const uint8_t *>(packed), N, d, pack8_pitch(d),
                                                                    vec, static_cast<__nv_bfloat16 *>(hidden));
    return finish(cudaGetLastError());
}

}  // extern "C"
