// Parameters and launchers of tree_attention's kernels.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "draft_tree.cuh"

namespace spr {

constexpr int kAttnTile = 64;            // keys per tile, the unit in which work is dealt out
constexpr int kAttnCtasPerSm = 2;        // at most
constexpr int kAttnMaxCtas = 148 * kAttnCtasPerSm;
constexpr int kAttnMaxDim = 128;

struct AttnParams {
    const void *q, *k, *v;               // [B,T,Hq,D]; caches [num_pages,Hkv,page_size,D]
    void *out;                           // [B,T,Hq,D]
    const int32_t *page_table;           // [B,max_pages]
    DraftNodes nodes;
    int B, Hq, Hkv, G, D;                // G = Hq / Hkv query heads share a cached head
    int max_pages, num_pages, page_size;
    int64_t capacity;                    // slots of a sequence that the page table can name
    float scale_log2;                    // scale * log2(e): scores are exponents of two
    float abs_scale_log2;                // its magnitude (not zero: masked scores, -inf, stay what they are under it) ...
    uint32_t flip;                       // ... and sign, as the sign bits of two bf16 numbers: queries take it over
    int ctas;
    // workspace
    int *status;
    int *counters;                       // [ctas] tickets of the items that several CTAs share, by the first of them
    float *part;                         // [2 * ctas][rows][D]   unnormalised results of parts of such items
    float2 *part_ml;                     // [2 * ctas][rows]      their maxima and sums
    uint32_t spin_limit;                 // polls after which a bounded wait gives up
    int test_flags;                      // ATTN_TEST_*
};
enum { ATTN_TEST_NO_LOADS = 1 };         // test hook: no tile is ever loaded, so that the first waits run out

// rows of a row block (queries of one cached head that are worked on together) for these sizes
int attention_block_rows(int T, int G, int dt);

cudaError_t launch_attention_f32(const AttnParams &p, int rows, cudaStream_t st);
cudaError_t launch_attention_f32_tile(const AttnParams &p, int rows, int dev, cudaStream_t st);
cudaError_t launch_attention_mma(const AttnParams &p, int dev, cudaStream_t st);
cudaError_t launch_attention_tc(const AttnParams &p, int dev, cudaStream_t st);

}  // namespace spr
