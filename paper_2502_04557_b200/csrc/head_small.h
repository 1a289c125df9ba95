// Small fp32 products of the vocabulary head on the CUDA cores (head_small.cu): parameter blocks and launcher.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace spr {

constexpr int kSmallTile = 32;

enum SmallMode {
    SMALL_STATS = 0,   // (max, sum of exp) of each row over the tile's 32 columns
    SMALL_DLOGITS,     // softmax gradient of each logit, fp32
    SMALL_OUT          // the product itself (launched behind the kernel before it)
};

// element (m, k) of an operand is p[m sm + k sk]
struct SmallOperand {
    const float *p;
    int64_t sm, sk;
};
struct SmallJob {
    SmallOperand a, b;          // k is the contiguous axis (SMALL_OUT: m is that of b)
    int a_across;               // SMALL_OUT: m is that of a, too
    int rows, cols, K;
    int splits;                 // CTAs that share a tile's contraction (SMALL_OUT; 0 counts as 1)
    float *acc;                 // splits > 1: their sums, [splits][tiles][1024]
    int *tickets;               // splits > 1: a counter per tile, zero before and after the launch
    int tiles_m, tiles_n;       // set by launch_small
    const int32_t *live;        // or null: entry k of the contraction counts only if live[k] is a token
    float2 *part;               // SMALL_STATS: part[row * tiles_n + tile]
    float *d;                   // SMALL_DLOGITS: d[row * d_pitch + column]
    int64_t d_pitch;
    const int32_t *targets;
    const float *lse, *grad_loss;
    float *out;                 // SMALL_OUT
    int64_t out_pitch;
};
struct SmallParams {
    SmallJob job[2];
    int V;
    int *status;
};
cudaError_t launch_small(SmallMode mode, SmallParams &prm, int njobs, cudaStream_t st);

}  // namespace spr
