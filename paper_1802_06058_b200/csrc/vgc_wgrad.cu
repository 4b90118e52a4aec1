// A linear layer's gradient and squared-gradient sums from its input's 8-bit checkpoint and its error delta (argument checks,
// choice of kernel, the CUDA-core kernel).
#include "vgc_wgrad.cuh"

namespace vgc {
namespace {

// CUDA cores: 64 x 64 outputs a block, 4 x 4 of g and of S a thread, 16 rows at a time through shared memory.  Sums of
// 256 rows are added up one after another: a single chain over 16384 rows was 1.4e-5 off.
constexpr int kTile = 64, kDeep = 16, kChain = 256;

template <class T>
__global__ void __launch_bounds__(256) wgrad_simt(const WgradArgs p, const T *delta, Checkpoint c)
{
    __shared__ float xs[kDeep][kTile], ds[kDeep][kTile + 4];
    grid_release();
    grid_wait();
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, i0 = blockIdx.x * kTile, o0 = blockIdx.y * kTile;
    float g[4][4] = {}, S[4][4] = {}, sum_g[4][4] = {}, sum_S[4][4] = {};
    for (int r0 = 0; r0 < p.rows; r0 += kDeep) {
        {   // 16 rows x 64 features: four codes of one block a thread
            const int r = r0 + ty, i = i0 + 4 * tx;
            float v[4] = {};
            if (r < p.rows && i < c.wide) {
                const uint32_t q = *reinterpret_cast<const uint32_t *>(c.codes + (size_t)r * c.wide + i);
                const float s = scale_of(*scale_word(c, r, i >> 7) >> (8 * ((i >> 5) & 3)) & 255u);
                e4m3_values(q, v[0], v[1]);
                e4m3_values(q >> 16, v[2], v[3]);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] *= s;
            }
            *reinterpret_cast<float4 *>(&xs[ty][4 * tx]) = make_float4(v[0], v[1], v[2], v[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int o = o0 + 16 * k + tx;
                ds[ty][16 * k + tx] = r < p.rows && o < p.out ? (float)delta[(size_t)r * p.out + o] : 0.f;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            float x[4], d[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                x[a] = xs[k][16 * a + tx];
                d[a] = ds[k][4 * ty + a];
            }
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    g[a][b] = fmaf(d[a], x[b], g[a][b]);
                    S[a][b] = fmaf(d[a] * d[a], x[b] * x[b], S[a][b]);
                }
        }
        __syncthreads();
        if ((r0 + kDeep) % kChain == 0 || r0 + kDeep >= p.rows) {
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    sum_g[a][b] += g[a][b];
                    sum_S[a][b] += S[a][b];
                    g[a][b] = S[a][b] = 0.f;
                }
        }
    }
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int o = o0 + 4 * ty + a, i = i0 + 16 * b + tx;
            if (o < p.out && i < p.in) p.write(o, i, sum_g[a][b], sum_S[a][b]);
        }
}

template <class T>
vgc_status simt_as(const WgradArgs &p, const void *delta, const Checkpoint &c, cudaStream_t st)
{
    VGC_CUDA_OK(launch_kernel(wgrad_simt<T>, dim3((unsigned)((p.in + kTile - 1) / kTile), (unsigned)((p.out + kTile - 1) / kTile)),
                              dim3(256), 0, st, true, p, static_cast<const T *>(delta), c));
    count_launch();
    return VGC_OK;
}

bool on_cuda_cores(int rows, int in, int out) { return (double)rows * in * out <= 0; }

bool wgrad_shape_ok(int rows, int in, int out)
{
    return rows >= 0 && rows <= kMaxRows && in >= 0 && in <= (1 << 24) && out >= 0 && out <= (1 << 22) - kTile;
}

}  // namespace
}  // namespace vgc

using namespace vgc;

extern "C" size_t vgc_wgrad_checkpoint_workspace_bytes(int rows, int in, int out, vgc_type type)
{
    if (!wgrad_shape_ok(rows, in, out) || rows == 0 || in == 0 || out == 0 || (type != VGC_FP32 && type != VGC_BF16)) return 0;
    return round_up(on_cuda_cores(rows, in, out) ? 256 : wgrad_tc_workspace_bytes(rows, in, out, type), 256);
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
    if (!on_cuda_cores(rows, in, out)) return wgrad_tc(p, delta, type, c, ws, st);
    return type == VGC_FP32 ? simt_as<float>(p, delta, c, st) : simt_as<__nv_bfloat16>(p, delta, c, st);
}
