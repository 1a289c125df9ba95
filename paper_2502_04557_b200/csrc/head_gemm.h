// Matrix products of the vocabulary head on CTA pairs: parameter blocks and launcher.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace spr {

constexpr int kPairTile = 256;       // rows and columns of one tile of a CTA pair
constexpr int kPairBlockK = 64;      // elements of the contraction per pipeline stage
constexpr int kMaxPairs = 128;       // CTA pairs of a launch (74 on a B200)

// What happens to a finished accumulator tile.
enum PairEpilogue {
    PAIR_STATS = 0,   // (max, sum of exp) of each row over the tile's columns
    PAIR_DLOGITS,     // softmax gradient of each logit in bf16 parts (dl_parts; three for fp32)
    PAIR_OUT          // the product itself, added to what is there or stored in the caller's type
};

// One product C[rows, cols] = A B over `kb` blocks of 64.  An operand is a 2-D bf16 tensor that
// runs along the contraction (its contiguous axis is K) or across it (its contiguous axis is M or
// N).  fp32 operands are kept as three bf16 parts that lie seg elements apart along the contiguous
// axis and are multiplied as six products (see head_gemm.cu).
struct PairJob {
    int tiles_m, tiles_n;         // tiles of 256 x 256
    int splits;                   // ranges of the contraction, each with a result of its own
    int kb, kb_per;               // blocks of the contraction; blocks per split
    int nprod;                    // products of parts: 1; 2 (A in two parts); 6 (A and B in three)
    int kc;                       // blocks that one accumulator takes before registers add it up
    int a_across, b_across;
    int a_seg, b_seg;
    int64_t rows;
    int cols;
    // PAIR_STATS: part[row * 2 tiles_n + 2 tile_n + half of the tile]
    float2 *part;
    // PAIR_DLOGITS: dlogits[row * dl_pitch + part * dl_seg + column], columns v0 .. v0 + cols of the vocabulary
    __nv_bfloat16 *dlogits;
    int64_t dl_pitch;
    int dl_parts;                 // bf16 operands: parts that D is kept in, 1 or 2
    int dl_seg, v0, V;
    const float *lse, *grad_loss;
    const int32_t *targets;
    // PAIR_OUT: out[row * out_pitch + column] in the caller's type if out, else fp32
    // acc[split * acc_stride + row * acc_pitch + column]; add_acc: acc is added to the product first
    void *out;
    int64_t out_pitch;
    int boxes;                    // PAIR_DLOGITS, PAIR_OUT: bf16 results go out as TMA boxes (set by launch_pair)
    float *acc;
    int64_t acc_stride, acc_pitch;
    int add_acc;
};

// Up to two products in one launch: the items (tile, split) of the first are dealt round to the
// pairs, those of the second in runs that even out the pairs' work.
struct PairParams {
    PairJob job[2];
    int items[2];
    int begin1[kMaxPairs], count1[kMaxPairs];
    int *status;
    uint32_t spin_limit;
    int test_flags;
};
enum { PAIR_TEST_NO_LOADS = 1 };     // test hook: nothing is loaded, so that the waits run out

struct PairOperand {
    const void *base;
    int64_t rows;       // outer axis
    int64_t cols;       // contiguous axis (all parts)
    int64_t pitch;      // elements, a multiple of 8
};

// njobs products; a[i], b[i] are the operands of job[i].  Fills in the schedule.  behind: the kernel before it in the
// stream is one of the same call, and this one may set itself up while that ends.
cudaError_t launch_pair(PairEpilogue epi, bool f32, PairParams &prm, int njobs, const PairOperand *a,
                        const PairOperand *b, bool behind, cudaStream_t st);

}  // namespace spr
