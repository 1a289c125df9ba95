// tree_attention: entry point, workspace, and which kernel takes which call.
#include <math.h>

#include "attention.h"
#include "host_util.h"
#include "launch.h"
#include "tensor_pair.cuh"

namespace spr {

namespace {

// most rows of a row block, for the workspace
int most_rows(int dt) { return dt == SPR_F32 ? 64 : 128; }

thread_local int t_test_flags = 0;
thread_local unsigned t_spin_limit = 0;

}  // namespace

int attention_block_rows(int T, int G, int dt)
{
    const int64_t rows = (int64_t)T * G;
    if (dt == SPR_F32) return rows <= 4 ? 4 : rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    return rows <= 16 ? 16 : 128;
}

size_t attention_ws_bytes(int D, int dt)
{
    if (D <= 0 || D > kAttnMaxDim) return 0;
    return ws_bytes_of([&](Carver &c) { attention_ws_layout(c, kAttnMaxCtas, most_rows(dt), D); });
}

}  // namespace spr

using namespace spr;

extern "C" {

int tree_attention(const void *q, const void *k_cache, const void *v_cache, int B, int T, int Hq, int Hkv, int D, int dt,
                   const int32_t *lens, const int32_t *counts, const int32_t *parents, const int32_t *page_table,
                   int max_pages, int num_pages, int page_size, float scale, void *out, void *ws, size_t ws_bytes,
                   void *cuda_stream)
{
    if (!dtype_ok(dt)) return SPR_ERR_UNSUPPORTED;
    if (B < 0 || T < 0 || Hkv <= 0 || Hq <= 0 || Hq % Hkv || D <= 0 || max_pages <= 0 || num_pages <= 0 || page_size <= 0 ||
        !isfinite(scale) || (int64_t)B * T > 0x7fffffff || Hq > 65536)
        return SPR_ERR_INVALID_ARG;
    if (D % 8 || D > kAttnMaxDim || page_size % 8 || T > kMaxTreeNodes || (int64_t)num_pages * Hkv > 0x7fffffff / page_size)
        return SPR_ERR_UNSUPPORTED;
    if (B == 0 || T == 0) return SPR_OK;
    if (!q || !k_cache || !v_cache || !out || !lens || !page_table) return SPR_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) || !aligned(lens, 4) ||
        !aligned(counts, 4) || !aligned(parents, 4) || !aligned(page_table, 4))
        return SPR_ERR_INVALID_ARG;
    const int rows = attention_block_rows(T, Hq / Hkv, dt);
    // work is counted in tiles, in 32 bits; so are a sequence's slots
    const int64_t capacity = (int64_t)max_pages * page_size < 0x7fffff00 ? (int64_t)max_pages * page_size : 0x7fffff00;
    const int64_t blocks = ((int64_t)T * (Hq / Hkv) + rows - 1) / rows;
    if ((double)B * Hkv * blocks * ((capacity + kAttnTile - 1) / kAttnTile) > 2147483000.0) return SPR_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < (size_t)kHeaderBytes) return SPR_ERR_WORKSPACE;
    Carver c = carve(ws_bytes);
    const AttentionWs w = attention_ws_layout(c, kAttnMaxCtas, rows, D);
    if (!c.fits()) return SPR_ERR_WORKSPACE;
    const int rc = device_supported();
    if (rc != SPR_OK) return rc;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return finish(e);

    AttnParams p = {};
    p.q = q, p.k = k_cache, p.v = v_cache, p.out = out, p.page_table = page_table;
    p.nodes = DraftNodes{lens, counts, parents, T};
    p.B = B, p.Hq = Hq, p.Hkv = Hkv, p.G = Hq / Hkv, p.D = D;
    p.max_pages = max_pages, p.num_pages = num_pages, p.page_size = page_size;
    p.capacity = capacity;
    p.scale_log2 = scale * kLog2e;
    p.abs_scale_log2 = fmaxf(fabsf(p.scale_log2), 1e-37f);
    p.flip = scale < 0.f ? 0x80008000u : 0u;
    const int per_sm = rows > 16 ? 1 : kAttnCtasPerSm;
    p.ctas = sms < 148 ? sms * per_sm : 148 * per_sm;
    p.status = static_cast<int *>(ws);
    p.counters = at<int>(ws, w.counters);
    p.part = at<float>(ws, w.part);
    p.part_ml = at<float2>(ws, w.part_ml);
    p.spin_limit = t_spin_limit ? t_spin_limit : pairtc::kSpinLimit;
    p.test_flags = t_test_flags;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SPR_F32) return finish(rows > 16 ? launch_attention_f32_tile(p, rows, dev, st) : launch_attention_f32(p, rows, st));
    return finish(rows == 16 ? launch_attention_mma(p, dev, st) : launch_attention_tc(p, dev, st));
}

void spr_test_tree_attention(int flags, unsigned spin_limit)
{
    t_test_flags = flags & ATTN_TEST_NO_LOADS;
    t_spin_limit = spin_limit;
}

}  // extern "C"
