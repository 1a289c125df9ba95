// The vocabulary head for a handful of tokens, a pass over W for every eight of them (head_stream.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace spr {

constexpr int kStreamTokens = 8;       // of a pass
constexpr size_t kStreamSmem = 160 * 1024;      // most that the states of a pass take

struct StreamParams {
    const void *hidden, *W;         // [N, d], [V, d]
    int N, d, V;                    // N: tokens of this pass
    int ctas;                       // of the launch: stream_ctas()
    int add;                        // gradient, fp32: dW is added to what an earlier pass left
    int pitch;                      // d rounded up to 64
    int vec;                        // rows of W (and dW) are 16-byte aligned
    float2 *part;                   // forward: [N, ctas] (max, sum of exp)
    const int32_t *targets;         // gradient
    const float *lse, *grad_loss;
    void *d_hidden, *d_W;           // which are wanted (dH itself is written by the sum over acc)
    float *acc;                     // [ctas, N, pitch]
    int *status;
};

inline int stream_rows(int N) { return N <= 1 ? 1 : N <= 2 ? 2 : N <= 4 ? 4 : 8; }      // tokens a kernel is built for
// d that the kernels take: the states in shared memory, and for the gradient a thread per 16 bytes of columns
inline bool stream_fits(bool grad, int N, int d, bool f32)
{
    return (int64_t)4 * stream_rows(N) * ((d + 63) / 64 * 64) <= (int64_t)kStreamSmem && (!grad || d <= 512 * (f32 ? 4 : 8));
}
// CTAs of a pass, from the sizes alone (the workspace holds a partial result of each)
inline int stream_ctas(bool grad, int N, int d, int V)
{
    const int rows = grad ? 32 : 64;                                   // of W, per CTA and round
    const int64_t smem = (int64_t)4 * stream_rows(N) * ((d + 63) / 64 * 64);
    const int per_sm = grad ? 1 : smem <= 100 * 1024 ? 2 : 1;
    const int64_t most = (V + rows - 1) / rows;
    return (int)(most < 148 * per_sm ? most : 148 * per_sm);
}
cudaError_t launch_stream(bool grad, bool f32, const StreamParams &prm, cudaStream_t st);

}  // namespace spr
