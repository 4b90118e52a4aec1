// Arguments that the kernels of a linear layer's gradient and statistic share.
#pragma once

#include "vgc_rowpass.cuh"

namespace vgc {

struct WgradArgs {
    float *g, *S;                    // [out][in], either may be null
    int rows, in, out;
    float scale_g, scale_s;
    int accumulate_g, accumulate_s;
    __device__ __forceinline__ void write_one(float *to, float v, float scale, int accumulate) const
    {
        v = __fmul_rn(scale, v);
        *to = accumulate ? __fadd_rn(ld_f(to), v) : v;
    }
};

size_t wgrad_tc_workspace_bytes(int rows, int in, int out, vgc_type type);
vgc_status wgrad_tc(const WgradArgs &p, const void *delta, vgc_type type, const Checkpoint &c, void *ws, cudaStream_t st);

}  // namespace vgc
