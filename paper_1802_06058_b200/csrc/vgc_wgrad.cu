// A linear layer's gradient and squared-gradient sums from its input's 8-bit checkpoint and its error delta (argument checks).
#include "vgc_wgrad.cuh"

namespace vgc {
namespace {

bool wgrad_shape_ok(int rows, int in, int out)
{
    return rows >= 0 && rows <= kMaxRows && in >= 0 && in <= (1 << 24) && out >= 0 && out <= (1 << 22);
}

}  // namespace
}  // namespace vgc

using namespace vgc;

extern "C" size_t vgc_wgrad_checkpoint_workspace_bytes(int rows, int in, int out, vgc_type type)
{
    if (!wgrad_shape_ok(rows, in, out) || rows == 0 || in == 0 || out == 0 || (type != VGC_FP32 && type != VGC_BF16)) return 0;
    return round_up(wgrad_tc_workspace_bytes(rows, in, out, type), 256);
}

extern "C" vgc_status vgc_wgrad_checkpoint(const void *checkpoint, const void *delta, vgc_type type, int rows, int in, int out,
                                           float scale_g, float scale_s, int accumulate_g, int accumulate_s, float *g, float *S,
                                           void *ws, size_t ws_bytes, vgc_stream_t stream)
{
    if (!wgrad_shape_ok(rows, in, out) || (type != VGC_FP32 && type != VGC_BF16)) return VGC_ERR_INVALID_ARG;
    if (!(scale_g == scale_g) || !(scale_s == scale_s)) return VGC_ERR_INVALID_ARG;
    if (in == 0 || out == 0) return VGC_OK;
    if ((!g && !S) || (reinterpret_cast<uintptr_t>(g) & 3u) || (reinterpret_cast<uintptr_t>(S) & 3u)) return VGC_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const size_t n = (size_t)in * out;
    if (rows == 0) {                                          // empty sums
        if (g && !accumulate_g) VGC_CUDA_OK(cudaMemsetAsync(g, 0, n * sizeof(float), st));
        if (S && !accumulate_s) VGC_CUDA_OK(cudaMemsetAsync(S, 0, n * sizeof(float), st));
        return VGC_OK;
    }
    if (!checkpoint || !delta || !aligned16(checkpoint) || !aligned16(delta)) return VGC_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < vgc_wgrad_checkpoint_workspace_bytes(rows, in, out, type)) return VGC_ERR_WORKSPACE;
    const Checkpoint c = checkpoint_at(const_cast<void *>(checkpoint), rows, in);
    WgradArgs p = {g, S, rows, in, out, scale_g, scale_s, accumulate_g, accumulate_s};
    return wgrad_tc(p, delta, type, c, ws, st);
}
