// tree_attention on fp32 tensors with more than 16 queries per cached head, on the CUDA cores.
//
// A CTA has 64 queries (32 where there are no more: 8 x 8, 32/8 heads of 128, 2000 tokens 89 -> 79 us) and walks their keys by 128
// with a running maximum and sum.  A warp owns eight (four) queries throughout, a
// lane four keys of each step for the scores, and D / 32 columns for the results: both products take 8 x 4 multiplications per
// 12 vectors read from shared memory, of which eight are the same for all lanes, and weights never leave the warp's
// rows of shared memory.  Keys of the next step are on their way (cp.async) while values are worked on, and the other way round.
// Bound by the multiplications, of which it does a third of the rate the CUDA cores have (eight warps on an SM, for 254 registers and 200 KB
// of shared memory, do not cover their reads of shared memory): 4 x 64 nodes, 32/8 heads of 128, 1500 tokens: 264 us, 89 us of
// multiplications; 16 x 17: 321 us.  By 16 queries at a time, as in attention_f32.cu, they would take twice as long (639 us against 280
// and 670 against 363, both measured on ragged batches).
// Steps that hold nodes, or slots without a page, test each pair of query and key.
#include <atomic>
#include <type_traits>

#include "attention_plan.cuh"
#include "host_util.h"
#include "launch.h"

namespace spr {

namespace {

constexpr int kThreads = 256, kWarps = 8;
constexpr int kStep = 128, kEach = kStep / 32;         // keys of a step, of a lane
constexpr int kLoads = kStep / kWarps;                 // keys that a warp brings
constexpr int kPitch = kStep + 4;                      // of a row of weights
constexpr float kUnseen = -1.f;                        // in place of a weight

size_t tile_smem(int rows, int D) { return sizeof(float) * ((size_t)(rows + kStep) * (D + 4) + (size_t)kStep * D + rows * kPitch); }

__device__ __forceinline__ void copy16(float *dst, const float *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void all_but_last() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// kRows: queries of a CTA; E: columns of a lane
template <int kRows, int E>
__global__ void __launch_bounds__(kThreads, 1) attention_f32_tile_kernel(const AttnParams p)
{
    constexpr int kOwn = kRows / kWarps;           // queries of a warp
    __shared__ int scratch[kWarps + 2];
    __shared__ int tree[kMaxTreeNodes];
    __shared__ uint32_t path[kRows][kMaxTreeNodes / 32];
    __shared__ uint8_t node_of[kRows];              // queries' rows of path
    __shared__ uint16_t there[2][kWarps];           // by steps in turn: which of a warp's keys have a page
    __shared__ int last;
    extern __shared__ __align__(16) float sm[];
    const int D = p.D, pitch = D + 4;
    float *qs = sm, *ks = qs + kRows * pitch, *vs = ks + kStep * pitch, *ps = vs + kStep * D;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row_of = warp * kOwn, col = lane * E;
    const bool in = col < D;
    AttnStretch s = attn_plan<kRows, kThreads, 2>(p, scratch);
    attn_clear_unused<float>(p, kThreads);
    const float *k_cache = static_cast<const float *>(p.k), *v_cache = static_cast<const float *>(p.v);
    AttnPart part;
    int tree_of = -1;
    while (attn_next<kRows>(p, s, part)) {
        const AttnTarget t = attn_target<kRows>(p, s, part);
        const int i0 = t.row0 / p.G, words = (s.seq.count + 31) / 32, nodes = (t.row0 + t.rows - 1) / p.G - i0 + 1;
        const int len = s.seq.len, keys = attn_keys(p, len, s.seq.count);
        if (keys < (int64_t)len + s.seq.count && tid == 0) raise_status(p.status, SPR_ERR_BAD_PAGE);
        const int slot0 = part.t0 * kAttnTile, end = min(slot0 + part.n * kAttnTile, keys), steps = (end - slot0 + kStep - 1) / kStep;

        // key j of the warp's in lane j: where its row begins in the caches, -1 where there is none
        auto find = [&](int step) -> int64_t {
            const int slot = slot0 + step * kStep + warp * kLoads + lane;
            if (lane >= kLoads || slot >= end) return -1;
            const int at = slot / p.page_size;
            const int page = __ldg(p.page_table + (int64_t)s.seq.b * p.max_pages + at);
            if (page < 0 || page >= p.num_pages) {
                raise_status(p.status, SPR_ERR_BAD_PAGE);
                return -1;
            }
            return (((int64_t)page * p.Hkv + part.head) * p.page_size + (slot - at * p.page_size)) * D;
        };
        auto fetch = [&](const float *cache, int64_t rows, float *to, int stride) {     // (keys that are not there are zeros)
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int64_t at = __shfl_sync(0xffffffffu, rows, j);
                if (lane * 4 < D) copy16(to + (warp * kLoads + j) * stride + lane * 4, cache + (at < 0 ? 0 : at) + lane * 4, at >= 0);
            }
            commit();
        };
        auto note = [&](int step, int64_t rows) {
            const uint32_t b = __ballot_sync(0xffffffffu, rows >= 0);
            if (lane == 0) there[step & 1][warp] = (uint16_t)b;
        };

        __syncthreads();                // (the part before has left shared memory)
        int64_t rows = find(0);
        note(0, rows);
        fetch(k_cache, rows, ks, pitch);
        fetch(v_cache, rows, vs, D);
        if (p.nodes.parents && tree_of != s.seq.b) {
            for (int j = tid; j < s.seq.count; j += kThreads) tree[j] = p.nodes.parents[(int64_t)s.seq.b * p.nodes.T + j];
            tree_of = s.seq.b;
            __syncthreads();
        }
        if (tid < nodes) attn_path_bits(p.nodes.parents ? tree : nullptr, i0 + tid, path[tid], words, p.status);
        if (tid < kRows) node_of[tid] = (uint8_t)min((t.row0 + tid) / p.G - i0, nodes - 1);
        for (int i = tid; i < kRows * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = (i - r * (D / 4)) * 4;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < t.rows) x = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.q) + attn_out_at(p, s, part, t.row0 + r) + c);     // (not __ldg: out may be q)
            x.x *= p.scale_log2, x.y *= p.scale_log2, x.z *= p.scale_log2, x.w *= p.scale_log2;
            *reinterpret_cast<float4 *>(qs + r * pitch + c) = x;
        }

        const bool busy = row_of < t.rows;
        float o[kOwn][E], m[kOwn], l[kOwn];
        uint32_t saw = 0;               // queries of the warp that have seen one of the lane's keys
#pragma unroll
        for (int r = 0; r < kOwn; ++r) {
            m[r] = neg_inf(), l[r] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) o[r][e] = 0.f;
        }
        for (int step = 0; step < steps; ++step) {
            all_but_last();             // keys
            __syncthreads();
            float sc[kOwn][kEach];
#pragma unroll
            for (int r = 0; r < kOwn; ++r)
#pragma unroll
                for (int j = 0; j < kEach; ++j) sc[r][j] = 0.f;
            const float *qr = qs + row_of * pitch, *kr = ks + lane * pitch;
#pragma unroll 2
            for (int c = 0; c < (busy ? D : 0); c += 4) {
                float4 k[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j) k[j] = *reinterpret_cast<const float4 *>(kr + 32 * j * pitch + c);
#pragma unroll
                for (int r = 0; r < kOwn; ++r) {
                    const float4 q = *reinterpret_cast<const float4 *>(qr + r * pitch + c);
#pragma unroll
                    for (int j = 0; j < kEach; ++j) {
                        sc[r][j] = fmaf(q.x, k[j].x, sc[r][j]);
                        sc[r][j] = fmaf(q.y, k[j].y, sc[r][j]);
                        sc[r][j] = fmaf(q.z, k[j].z, sc[r][j]);
                        sc[r][j] = fmaf(q.w, k[j].w, sc[r][j]);
                    }
                }
            }
            // keys of lane, lane + 32, ...: a word of bits each
            uint32_t have[kEach];
            bool all = slot0 + (step + 1) * kStep <= len;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                have[j] = there[step & 1][2 * j] | (uint32_t)there[step & 1][2 * j + 1] << 16;
                all &= have[j] == 0xffffffffu;
            }
            __syncthreads();
            if (step + 1 < steps) {
                rows = find(step + 1);
                note(step + 1, rows);
                fetch(k_cache, rows, ks, pitch);
            } else {
                commit();
            }
            auto sees = [&](int r, int j, uint32_t has) {
                const int node = slot0 + step * kStep + 32 * j + lane - len;
                const uint32_t *bits = path[node_of[row_of + r]];
                return (has >> lane & 1) && (node < 0 || (bits[node >> 5] >> (node & 31) & 1));
            };
            if (!all) {
#pragma unroll
                for (int r = 0; r < kOwn; ++r)
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
                        if (sees(r, j, have[j]))
                            saw |= 1u << r;
                        else
                            sc[r][j] = neg_inf();
            } else {
                saw = (1u << kOwn) - 1;
            }
            float *pr = ps + row_of * kPitch;
#pragma unroll
            for (int r = 0; r < kOwn; ++r) {
                float top = sc[r][0];
#pragma unroll
                for (int j = 1; j < kEach; ++j) top = fmaxf(top, sc[r][j]);
#pragma unroll
                for (int off = 16; off; off /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                top = fmaxf(top, m[r]);
                const float ref = top == neg_inf() ? 0.f : top, a = ex2(m[r] - ref);
                m[r] = top;
                l[r] *= a;
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] *= a;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const float w = ex2(sc[r][j] - ref);
                    l[r] += w;
                    pr[r * kPitch + 32 * j + lane] = w;
                }
            }
            if (!all) {
#pragma unroll
                for (int j = 0; j < kEach; ++j)
#pragma unroll 1
                    for (int r = 0; r < kOwn; ++r)
                        if (!sees(r, j, have[j])) pr[r * kPitch + 32 * j + lane] = kUnseen;
            }
            all_but_last();             // values
            __syncthreads();
            const float *vr = vs + (in ? col : 0);
            auto products = [&](auto test) {
#pragma unroll 2
                for (int k = 0; k < (busy ? kStep : 0); k += 4) {
                    float v[4][E];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (E == 4) {
                            const float4 x = *reinterpret_cast<const float4 *>(vr + (k + i) * D);
                            v[i][0] = x.x, v[i][1] = x.y, v[i][E - 2] = x.z, v[i][E - 1] = x.w;
                        } else {
                            const float2 x = *reinterpret_cast<const float2 *>(vr + (k + i) * D);
                            v[i][0] = x.x, v[i][1] = x.y;
                        }
                    }
#pragma unroll
                    for (int r = 0; r < kOwn; ++r) {
                        const float4 x = *reinterpret_cast<const float4 *>(pr + r * kPitch + k);
                        const float w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // a query takes nothing from a key that it does not see, not even 0 times infinity
                            const bool takes = !decltype(test)::value || w[i] != kUnseen;
#pragma unroll
                            for (int e = 0; e < E; ++e) o[r][e] = takes ? fmaf(w[i], v[i][e], o[r][e]) : o[r][e];
                        }
                    }
                }
            };
            if (all)
                products(std::false_type());
            else
                products(std::true_type());
            __syncthreads();
            if (step + 1 < steps)
                fetch(v_cache, rows, vs, D);
            else
                commit();
        }
        saw = __reduce_or_sync(0xffffffffu, saw);
#pragma unroll
        for (int r = 0; r < kOwn; ++r) {
            m[r] = attn_top(m[r], saw >> r & 1);
#pragma unroll
            for (int off = 16; off; off /= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], off);
            const int row = row_of + r;
            if (row >= t.rows) continue;
            float inv = 1.f;
            float *to;
            if (t.whole) {
                inv = attn_inverse(m[r], l[r]);
                to = static_cast<float *>(p.out) + attn_out_at(p, s, part, t.row0 + row) + col;
            } else {
                to = p.part + ((int64_t)t.slot * kRows + row) * D + col;
                if (lane == 0) __stcg(&p.part_ml[(int64_t)t.slot * kRows + row], make_float2(m[r], l[r]));
            }
            if (!in) continue;
            if (E == 4)
                __stcg(reinterpret_cast<float4 *>(to), make_float4(o[r][0] * inv, o[r][1] * inv, o[r][E - 2] * inv, o[r][E - 1] * inv));
            else
                __stcg(reinterpret_cast<float2 *>(to), make_float2(o[r][0] * inv, o[r][1] * inv));
        }
        if (!t.whole) {
            __syncthreads();
            if (tid == 0) last = attn_ticket(p, t);
            __syncthreads();
            if (last) attn_join<kRows, float>(p, s, part, t, warp, kWarps);
        }
    }
}

template <int ROWS, int E>
cudaError_t launch_tile(const AttnParams &p, int dev, cudaStream_t st)
{
    static std::atomic<bool> attr_set[64];   // host threads may race to set it: all of them store `true`
    if (dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_f32_tile_kernel<ROWS, E>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)tile_smem(ROWS, E * 32));
        if (e != cudaSuccess) return e;
        if (dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    attention_f32_tile_kernel<ROWS, E><<<p.ctas, kThreads, tile_smem(ROWS, p.D), st>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_f32_tile(const AttnParams &p, int rows, int dev, cudaStream_t st)
{
    if (rows == 32) return p.D <= 64 ? launch_tile<32, 2>(p, dev, st) : launch_tile<32, 4>(p, dev, st);
    return p.D <= 64 ? launch_tile<64, 2>(p, dev, st) : launch_tile<64, 4>(p, dev, st);
}

}  // namespace spr
