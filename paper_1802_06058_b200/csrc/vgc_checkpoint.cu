// Activation checkpoints in 8 bits: e4m3 codes with a power-of-two scale per 32 neighbouring features.
//
// Bound: HBM, 2 or 4 bytes in and 33/32 out per value, or the other way round.  A warp takes 256 neighbouring features of a
// row (one 16-byte load a lane in bf16), finds the blocks' maxima with two or three shuffles, and has kFlight such segments
// in flight.  Power-of-two scales make the scaling exact, so that the code's own rounding is the only one.
// Measured (B200, of the measured copy rate): 16384 x 16384 bf16 store 147 us (0.86), load 156 us (0.81); 16384 x 4096 fp32 58 us (0.90) and
// 61 us (0.85).  Rows that do not start on 16 bytes, 30000 x 1001: bf16, in aligned pieces shifted between lanes, 32 and 30 us (0.44, 0.47;
// by single elements 46 and 38); fp32, by single elements, 40 and 45 us (0.58, 0.52).  (With a 64-bit division for every segment and
// maxima on integers the store of 16384 x 16384 took 196 us.)
#include "vgc_rowpass.cuh"

namespace vgc {
namespace {

constexpr int kThreads = 256, kFlight = 4;

// The segments that a warp takes, numbered along the rows: neighbouring warps work on neighbouring memory.
struct Walk {
    uint32_t row, seg, rows_on, segs_on, segs;
    __device__ __forceinline__ Walk(uint32_t segs_) : segs(segs_)
    {
        const uint32_t warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
        row = warp / segs;
        seg = warp - row * segs;
        rows_on = warps / segs;
        segs_on = warps - rows_on * segs;
    }
    __device__ __forceinline__ void next()
    {
        row += rows_on;
        seg += segs_on;
        if (seg >= segs) {
            seg -= segs;
            ++row;
        }
    }
};

template <class T, bool kVec>
__global__ void __launch_bounds__(kThreads) checkpoint_store(const T *x, int rows, int features, uint32_t segs, Checkpoint c)
{
    grid_release();
    grid_wait();
    const int lane = threadIdx.x & 31;
    if (blockIdx.x == gridDim.x - 1) clear_row_padding(c, rows, threadIdx.x, kThreads);
    Walk ahead(segs), here = ahead;
    while (here.row < (uint32_t)rows) {
        Raw<T> r[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k, ahead.next()) {
            if (ahead.row >= (uint32_t)rows) continue;
            const int first = (int)ahead.seg * kSeg;
            load_seg<kVec>(x + (size_t)ahead.row * features + first, features - first, lane, r[k]);
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k, here.next())
            if (here.row < (uint32_t)rows) store_blocks<T, kVec>(c, (int)here.row, (int)here.seg * kSeg, lane, r[k]);
    }
}

template <class T, bool kVec>
__global__ void __launch_bounds__(kThreads) checkpoint_load(T *x, int rows, int features, uint32_t segs, Checkpoint c)
{
    grid_release();
    grid_wait();
    const int lane = threadIdx.x & 31;
    Walk ahead(segs), here = ahead;
    while (here.row < (uint32_t)rows) {
        uint32_t q[kFlight][2], w[kFlight][2];
#pragma unroll
        for (int k = 0; k < kFlight; ++k, ahead.next()) {
            if (ahead.row >= (uint32_t)rows) continue;
            const int first = (int)ahead.seg * kSeg, left = c.wide - first, unit = first >> 7;
            const uint8_t *const codes = c.codes + (size_t)ahead.row * c.wide + first;
            q[k][0] = q[k][1] = 0;
            if constexpr (sizeof(T) == 2) {
                if (8 * lane < left) {
                    const uint2 v = *reinterpret_cast<const uint2 *>(codes + 8 * lane);
                    q[k][0] = v.x; q[k][1] = v.y;
                    w[k][0] = *scale_word(c, (int)ahead.row, unit + (lane >> 4));
                }
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (128 * j >= left) continue;
                    w[k][j] = *scale_word(c, (int)ahead.row, unit + j);
                    if constexpr (kVec) {
                        q[k][j] = *reinterpret_cast<const uint32_t *>(codes + 128 * j + 4 * lane);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) q[k][j] |= (uint32_t)codes[128 * j + 32 * i + lane] << (8 * i);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k, here.next()) {
            if (here.row >= (uint32_t)rows) continue;
            const int first = (int)here.seg * kSeg;
            Raw<T> out;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float a, b;
                e4m3_values(q[k][j >> 1] >> (16 * (j & 1)), a, b);
                F2 scale;
                if constexpr (sizeof(T) == 2) scale = f2(scale_of(w[k][0] >> (8 * ((lane >> 2) & 3)) & 255u));
                else if constexpr (!kVec) scale = f2(scale_of(w[k][j >> 1] >> (16 * (j & 1)) & 255u), scale_of(w[k][j >> 1] >> (16 * (j & 1) + 8) & 255u));
                else scale = f2(scale_of(w[k][j >> 1] >> (8 * (lane >> 3)) & 255u));
                set_pair(out, j, mul2(f2(a, b), scale));
            }
            store_seg<kVec>(x + (size_t)here.row * features + first, features - first, lane, out);
        }
    }
}

bool sizes_ok(int rows, int features) { return rows >= 0 && rows <= kMaxRows && features >= 0 && features <= (1 << 24); }

// as many warps as have work, up to eight blocks an SM
unsigned blocks_for(int rows, uint32_t segs)
{
    const uint64_t blocks = ((uint64_t)rows * segs + kThreads / 32 - 1) / (kThreads / 32), most = (uint64_t)kSmCount * 8;
    return (unsigned)(blocks < most ? blocks : most);
}

// 16-byte pieces where every row starts on 16 bytes
template <class T> bool vectors(int features) { return (size_t)features * sizeof(T) % 16 == 0; }

template <class T>
vgc_status store_as(const void *x, int rows, int features, const Checkpoint &c, cudaStream_t st)
{
    const uint32_t segs = (uint32_t)((features + kSeg - 1) / kSeg);
    VGC_CUDA_OK(launch_kernel(vectors<T>(features) ? checkpoint_store<T, true> : checkpoint_store<T, false>, dim3(blocks_for(rows, segs)), dim3(kThreads), 0,
                              st, true, static_cast<const T *>(x), rows, features, segs, c));
    count_launch();
    return VGC_OK;
}
template <class T>
vgc_status load_as(void *x, int rows, int features, const Checkpoint &c, cudaStream_t st)
{
    const uint32_t segs = (uint32_t)((features + kSeg - 1) / kSeg);
    VGC_CUDA_OK(launch_kernel(vectors<T>(features) ? checkpoint_load<T, true> : checkpoint_load<T, false>, dim3(blocks_for(rows, segs)), dim3(kThreads), 0,
                              st, true, static_cast<T *>(x), rows, features, segs, c));
    count_launch();
    return VGC_OK;
}

}  // namespace
}  // namespace vgc

using namespace vgc;

extern "C" size_t vgc_checkpoint_bytes(int rows, int features)
{
    if (rows <= 0 || features <= 0 || !sizes_ok(rows, features)) return 0;
    const size_t wide = (size_t)wide_of(features), tall = (size_t)tall_of(rows);
    return (size_t)rows * wide + tall * (wide / 32);
}

extern "C" vgc_status vgc_checkpoint_store(const void *x, vgc_type type, int rows, int features, void *checkpoint,
                                           vgc_stream_t stream)
{
    if (!sizes_ok(rows, features) || (type != VGC_FP32 && type != VGC_BF16)) return VGC_ERR_INVALID_ARG;
    if (rows == 0 || features == 0) return VGC_OK;
    if (!x || !checkpoint || !aligned16(x) || !aligned16(checkpoint)) return VGC_ERR_INVALID_ARG;
    const Checkpoint c = checkpoint_at(checkpoint, rows, features);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return type == VGC_FP32 ? store_as<float>(x, rows, features, c, st) : store_as<__nv_bfloat16>(x, rows, features, c, st);
}

extern "C" vgc_status vgc_checkpoint_load(const void *checkpoint, int rows, int features, void *x, vgc_type type,
                                          vgc_stream_t stream)
{
    if (!sizes_ok(rows, features) || (type != VGC_FP32 && type != VGC_BF16)) return VGC_ERR_INVALID_ARG;
    if (rows == 0 || features == 0) return VGC_OK;
    if (!x || !checkpoint || !aligned16(x) || !aligned16(checkpoint)) return VGC_ERR_INVALID_ARG;
    const Checkpoint c = checkpoint_at(const_cast<void *>(checkpoint), rows, features);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return type == VGC_FP32 ? load_as<float>(x, rows, features, c, st) : load_as<__nv_bfloat16>(x, rows, features, c, st);
}
