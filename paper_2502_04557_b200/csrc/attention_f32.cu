// tree_attention on fp32 tensors with up to 16 queries per cached head, on the CUDA cores.
//
// A warp walks its keys on its own, with a running maximum and sum: a lane holds E columns of all the block's queries
// and of their results in registers, a key's row is one coalesced load, and the products of a key with the block's ROWS
// queries are added up over the lanes by halves (half of the rows to the other half of the lanes, five times over), so
// that ROWS scores cost some ROWS shuffles.  The warps of a CTA share a tile's keys and are joined
// through shared memory at the end of a part.  Up to four
// rows the loads bound it, above that multiplications and shuffles: 64 x 1, 32/8 heads of 128, some 3000 tokens each: 396 us, 241 us
// of loads.
#include "attention_plan.cuh"
#include "host_util.h"
#include "launch.h"

namespace spr {

namespace {

constexpr int kGroup = 4;            // keys worked on at once
// Warps of a CTA: eight where their registers leave room for two such CTAs on an SM, so that more loads are on their way
template <int ROWS, int E>
constexpr int kWarpsFor = ROWS * E <= 16 ? 8 : 4;

template <int E>
struct Cols {
    float x[E];
    template <bool CONSTANT = true>             // nothing is written there while the kernel runs (unlike queries: out may be q)
    __device__ __forceinline__ void load(const float *p, bool there)
    {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.f;
        if (!there) return;
        if (E == 4) {
            const float4 *from = reinterpret_cast<const float4 *>(p), a = CONSTANT ? __ldg(from) : *from;
            x[0] = a.x, x[1] = a.y, x[E - 2] = a.z, x[E - 1] = a.w;
        } else {
            const float2 *from = reinterpret_cast<const float2 *>(p), a = CONSTANT ? __ldg(from) : *from;
            x[0] = a.x, x[1] = a.y;
        }
    }
};

template <int ROWS, int E>
__global__ void __launch_bounds__(32 * kWarpsFor<ROWS, E>, 2) attention_f32_kernel(const AttnParams p)
{
    constexpr int kF32Warps = kWarpsFor<ROWS, E>, kF32Threads = 32 * kF32Warps;
    constexpr int kKeys = kAttnTile / kF32Warps;    // of a tile, per warp
    constexpr int kLanes = 32 / ROWS;               // lanes that share a row's score
    __shared__ int scratch[kF32Warps + 2];
    __shared__ int tree[kMaxTreeNodes];
    __shared__ uint32_t path[ROWS][kMaxTreeNodes / 32];
    __shared__ float2 ml[kF32Warps][ROWS];
    __shared__ int last;
    extern __shared__ __align__(16) float obuf[];   // [kF32Warps][ROWS][D]

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int my_row = lane / kLanes, col = lane * E;
    const bool in = col < p.D;
    AttnStretch s = attn_plan<ROWS, kF32Threads, 1>(p, scratch);
    attn_clear_unused<float>(p, kF32Threads);
    const float *k_cache = static_cast<const float *>(p.k), *v_cache = static_cast<const float *>(p.v);
    AttnPart part;
    int tree_of = -1;
    while (attn_next<ROWS>(p, s, part)) {
        const AttnTarget t = attn_target<ROWS>(p, s, part);
        const int i0 = (int)(t.row0 / p.G);
        __syncthreads();
        if (p.nodes.parents && tree_of != s.seq.b) {
            for (int j = tid; j < s.seq.count; j += kF32Threads) tree[j] = p.nodes.parents[(int64_t)s.seq.b * p.nodes.T + j];
            tree_of = s.seq.b;
            __syncthreads();
        }
        const int words = (s.seq.count + 31) / 32;
        const int nodes = (int)((t.row0 + t.rows - 1) / p.G) - i0 + 1;
        if (tid < nodes) attn_path_bits(p.nodes.parents ? tree : nullptr, i0 + tid, path[tid], words, p.status);
        __syncthreads();

        float q[ROWS][E], o[ROWS][E];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            Cols<E> c;
            c.template load<false>(static_cast<const float *>(p.q) + (r < t.rows ? attn_out_at(p, s, part, t.row0 + r) : 0) + col, in && r < t.rows);
#pragma unroll
            for (int e = 0; e < E; ++e) q[r][e] = c.x[e] * p.scale_log2, o[r][e] = 0.f;
        }
        const uint32_t *bits = path[min((int)((t.row0 + my_row) / p.G) - i0, nodes - 1)];
        const int keys = attn_keys(p, s.seq.len, s.seq.count);
        if (keys < (int64_t)s.seq.len + s.seq.count && tid == 0) raise_status(p.status, SPR_ERR_BAD_PAGE);

        // rows of a tile's keys in the caches, key j of the warp's in lane j; -1 where there is none
        auto find = [&](int tile) -> int64_t {
            const int slot = tile * kAttnTile + warp * kKeys + lane;
            if (lane >= kKeys || slot >= keys) return -1;
            const int at = slot / p.page_size;
            const int page = __ldg(p.page_table + (int64_t)s.seq.b * p.max_pages + at);
            if (page < 0 || page >= p.num_pages) {
                raise_status(p.status, SPR_ERR_BAD_PAGE);
                return -1;
            }
            return (((int64_t)page * p.Hkv + part.head) * p.page_size + (slot - at * p.page_size)) * p.D;
        };
        Cols<E> kk[kGroup], vv[kGroup], kn[kGroup], vn[kGroup];
        auto fetch = [&](int64_t rows, int group, Cols<E> (&k)[kGroup], Cols<E> (&v)[kGroup]) {
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                const int64_t at = __shfl_sync(0xffffffffu, rows, group * kGroup + j);
                k[j].load(k_cache + at + col, in && at >= 0);
                v[j].load(v_cache + at + col, in && at >= 0);
            }
        };
        float m = neg_inf(), l = 0.f;       // (m is no less than kOnlyMinusInf once a key has been seen)
        auto use = [&](int64_t rows, int tile, int group, const Cols<E> (&k)[kGroup], const Cols<E> (&v)[kGroup]) {
            float sc[kGroup], top = m;
            uint32_t seen[kGroup];
            const int slot0 = tile * kAttnTile + warp * kKeys + group * kGroup;
            if (slot0 >= keys) return;
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                float x[ROWS];
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    x[r] = q[r][0] * k[j].x[0];
#pragma unroll
                    for (int e = 1; e < E; ++e) x[r] = fmaf(q[r][e], k[j].x[e], x[r]);
                }
                int off = 16;
#pragma unroll
                for (int n = ROWS / 2; n > 0; n /= 2, off /= 2) {
                    const bool upper = lane & off;
#pragma unroll
                    for (int r = 0; r < n; ++r) {
                        const float give = upper ? x[r] : x[r + n], keep = upper ? x[r + n] : x[r];
                        x[r] = keep + __shfl_xor_sync(0xffffffffu, give, off);
                    }
                }
#pragma unroll
                for (int o2 = kLanes / 2; o2 > 0; o2 /= 2) x[0] += __shfl_xor_sync(0xffffffffu, x[0], o2);
                sc[j] = x[0];
                const bool there = __shfl_sync(0xffffffffu, rows, group * kGroup + j) >= 0;
                const int node = slot0 + j - s.seq.len;
                const bool vis = there && (node < 0 || (bits[node >> 5] >> (node & 31) & 1));
                if (!vis) sc[j] = neg_inf();
                seen[j] = __ballot_sync(0xffffffffu, vis);
                if (vis) top = fmaxf(top, kOnlyMinusInf);
            }
#pragma unroll
            for (int j = 0; j < kGroup; ++j) top = fmaxf(top, sc[j]);
            const float ref = top == neg_inf() ? 0.f : top;
            if (__any_sync(0xffffffffu, top > m)) {
                const float a = ex2(m - ref);
                l *= a;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float ar = __shfl_sync(0xffffffffu, a, r * kLanes);
#pragma unroll
                    for (int e = 0; e < E; ++e) o[r][e] *= ar;
                }
                m = top;
            }
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                const float w = ex2(sc[j] - ref);
                l += w;
                if (seen[j] == 0xffffffffu) {
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        const float wr = __shfl_sync(0xffffffffu, w, r * kLanes);
#pragma unroll
                        for (int e = 0; e < E; ++e) o[r][e] = fmaf(wr, v[j].x[e], o[r][e]);
                    }
                } else {        // rows that do not see the key take nothing from it, not even 0 times infinity
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        const float wr = __shfl_sync(0xffffffffu, w, r * kLanes);
                        if (seen[j] >> (r * kLanes) & 1) {
#pragma unroll
                            for (int e = 0; e < E; ++e) o[r][e] = fmaf(wr, v[j].x[e], o[r][e]);
                        }
                    }
                }
            }
        };
        int64_t rows = find(part.t0), next = -1;
        fetch(rows, 0, kk, vv);
        for (int n = 0; n < part.n; ++n) {
            if (n + 1 < part.n) next = find(part.t0 + n + 1);
#pragma unroll
            for (int g = 0; g < kKeys / kGroup; g += 2) {
                fetch(rows, g + 1, kn, vn);
                use(rows, part.t0 + n, g, kk, vv);
                if (g + 2 < kKeys / kGroup)
                    fetch(rows, g + 2, kk, vv);
                else if (n + 1 < part.n)
                    fetch(next, 0, kk, vv);
                use(rows, part.t0 + n, g + 1, kn, vn);
            }
            rows = next;
        }

        // join the warps
        if (lane % kLanes == 0) ml[warp][my_row] = make_float2(m, l);
        if (in) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int e = 0; e < E; ++e) obuf[(warp * ROWS + r) * p.D + col + e] = o[r][e];
        }
        __syncthreads();
        const int cols = p.D / 4;
        for (int i = tid; i < t.rows * cols; i += kF32Threads) {
            const int row = i / cols, c = (i - row * cols) * 4;
            float top = neg_inf();
#pragma unroll
            for (int w = 0; w < kF32Warps; ++w) top = fmaxf(top, ml[w][row].x);
            const float ref = top == neg_inf() ? 0.f : top;
            float sum = 0.f;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kF32Warps; ++w) {
                const float a = ex2(ml[w][row].x - ref);
                sum = fmaf(a, ml[w][row].y, sum);
                const float4 x = *reinterpret_cast<const float4 *>(obuf + (w * ROWS + row) * p.D + c);
                y.x = fmaf(a, x.x, y.x), y.y = fmaf(a, x.y, y.y), y.z = fmaf(a, x.z, y.z), y.w = fmaf(a, x.w, y.w);
            }
            if (t.whole) {
                const float inv = attn_inverse(top, sum);
                store_out(static_cast<float *>(p.out) + attn_out_at(p, s, part, t.row0 + row) + c, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv), 4);
            } else {
                __stcg(reinterpret_cast<float4 *>(p.part + ((int64_t)t.slot * ROWS + row) * p.D + c), y);
                if (c == 0) __stcg(&p.part_ml[(int64_t)t.slot * ROWS + row], make_float2(top, sum));
            }
        }
        if (!t.whole) {
            __syncthreads();
            if (tid == 0) last = attn_ticket(p, t);
            __syncthreads();
            if (last) attn_join<ROWS, float>(p, s, part, t, warp, kF32Warps);
        }
    }
}

template <int ROWS, int E>
cudaError_t launch_rows(const AttnParams &p, cudaStream_t st)
{
    constexpr int warps = kWarpsFor<ROWS, E>;
    const size_t smem = sizeof(float) * warps * ROWS * p.D;      // 32 KB at most
    attention_f32_kernel<ROWS, E><<<p.ctas, 32 * warps, smem, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_f32(const AttnParams &p, int rows, cudaStream_t st)
{
    const bool narrow = p.D <= 64;
    switch (rows) {
    case 4: return narrow ? launch_rows<4, 2>(p, st) : launch_rows<4, 4>(p, st);
    case 8: return narrow ? launch_rows<8, 2>(p, st) : launch_rows<8, 4>(p, st);
    default: return narrow ? launch_rows<16, 2>(p, st) : launch_rows<16, 4>(p, st);
    }
}

}  // namespace spr
