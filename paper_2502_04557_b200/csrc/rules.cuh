// What the two kernels of logits_rules share.
#pragma once

#include "common.cuh"
#include "draft_tree.cuh"

namespace spr {

constexpr int kRuleMaxBiases = 1024;
constexpr int kRuleOnPath = (int)0x80000000u;

struct RuleParams {
    const void *logits;
    void *out;
    int64_t ldv, ld_out;
    int V, B;
    DraftNodes nodes;            // lens is not used
    const int32_t *history;
    int64_t ld_history;
    const int32_t *history_len;
    const int32_t *tokens;       // [B,T] or null
    const float *penalties;      // [B,3] or null
    const int32_t *bias_tokens;  // [B,n_bias]
    const float *bias_values;
    int n_bias;
    const uint32_t *masks;       // [num_masks, ld_mask]
    int64_t ld_mask;
    int num_masks;
    const int32_t *mask_rows;    // [B,T]
    int *status;
    int pieces, piece;           // of a row, and the vectors of one
    int row_groups, rows_per_group;
    int stages;                  // of the ring of rows, where there is one
    int same;                    // rows of both tensors lie alike on 16-byte boundaries
};

// a bit for each byte, as that byte's highest
__device__ __forceinline__ uint32_t byte_signs(uint32_t four) { return ((four & 0xfu) * 0x00204081u & 0x01010101u) << 7; }

template <typename T>
struct RuleLanes;            // a 16-byte vector as elements
template <>
struct RuleLanes<float> {
    static __device__ __forceinline__ void forbid(uint32_t (&w)[4], uint32_t allowed)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = allowed >> e & 1 ? w[e] : 0xff800000u;
    }
};
template <>
struct RuleLanes<__nv_bfloat16> {
    static __device__ __forceinline__ void forbid(uint32_t (&w)[4], uint32_t allowed)
    {
        const uint32_t s[2] = {byte_signs(allowed), byte_signs(allowed >> 4)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {       // a half of all ones where the element is allowed
            uint32_t m;
            asm("prmt.b32 %0, %1, %1, %2;" : "=r"(m) : "r"(s[e >> 1]), "r"(e & 1 ? 0xbbaa : 0x9988));    // signs of two bytes
            w[e] = (w[e] & m) | (0xff80ff80u & ~m);
        }
    }
};

// n <= 8 bits of a bit row from bit `at` on (bits before 0 and behind `words` words read as zero)
__device__ __forceinline__ uint32_t bits_at(const uint32_t *row, int at, int words)
{
    const int w = at >> 5;
    const uint32_t lo = w >= 0 && w < words ? row[w] : 0u, hi = w + 1 >= 0 && w + 1 < words ? row[w + 1] : 0u;
    return __funnelshift_r(lo, hi, at & 31);
}

// Rows that are few beside the sequences (logits_rules_single.cu).
template <typename T>
cudaError_t launch_rules_single(RuleParams &p, cudaStream_t st);

}  // namespace spr
