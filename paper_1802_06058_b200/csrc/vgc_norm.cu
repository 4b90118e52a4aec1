// Layer norm over the rows of an activation matrix, its backward pass, and the gradient and squared-gradient sums of gain and bias.
//
// Forward: a row stays in the registers of its warps (8 features a lane, 16 beyond 8192) between the mean, the squared deviations
// from it and the write: one read and one write of the matrix, no cancellation in the variance.  The next row is loaded before
// the sums of this one.
// Backward: dx = rstd (w - mean(w) - xh mean(w xh)), w = dy gamma.  The same lanes keep the column sums of their features (dy xh, dy
// and their squares) in registers over all rows that their block takes, so x and dy are read once; each block leaves one row of
// partial sums, which norm_combine adds in the blocks' order.
//   samples of one row      four sums per feature
//   samples of many rows    whole samples where there are enough of them for every group of warps (the sample's sums, squared
//                           when it ends, beside the four), otherwise pieces of samples: a block's two sums belong to one sample, and
//                           norm_combine squares what a sample's pieces add up to
// Beyond 8192 features a block has no registers for a row's column sums: norm_row_sums finds the two means of every row first, and
// blocks of 256 columns need no sums across a row (x and dy are read twice).
// Bound: HBM.
#include <cfloat>

#include "vgc_rowpass.cuh"

namespace vgc {
namespace {

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}

// Sums over the `warps` warps of a row, in every thread of them.  Two slots in turn: a warp writes a slot again only behind the
// barrier of the sum after, when all have read it.
struct RowSum {
    float2 *slots;                   // [2][32] of this group
    int warps, warp, lane, barrier, turn;
    __device__ float2 operator()(float a, float b)
    {
        a = warp_sum(a);
        b = warp_sum(b);
        if (warps == 1) return make_float2(a, b);
        float2 *const s = slots + 32 * turn;
        turn ^= 1;
        if (lane == 0) s[warp] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(32 * warps) : "memory");
        const float2 v = lane < warps ? s[lane] : make_float2(0.f, 0.f);
        return make_float2(warp_sum(v.x), warp_sum(v.y));
    }
};

// ---- forward ------------------------------------------------------------------------------------------------------------------
template <class T>
struct Forward {
    const T *x;
    const float *gamma, *beta;
    T *y;
    float *mean, *rstd;
    int rows, features, warps, groups;      // warps of a row, rows a block takes at a time
    float eps;
    Checkpoint c;
};

// kParts: segments of 256 features a warp takes
template <class T, bool kVec, int kParts, bool kCheckpoint>
__global__ void __launch_bounds__(1024, 1) norm_forward(const Forward<T> p)
{
    __shared__ float2 slots[8][64];
    const int lane = threadIdx.x & 31, all = threadIdx.x >> 5, group = all / p.warps, warp = all - group * p.warps;
    RowSum sum = {slots[group], p.warps, warp, lane, 1 + group, 0};
    grid_release();
    grid_wait();
    const int C = p.features, first = warp * kParts * kSeg;
    constexpr bool kKept = kParts == 1;      // gain and bias in registers
    float gain[kKept ? 8 : 1], bias[kKept ? 8 : 1];
    if constexpr (kKept) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = first + seg_col<T, kVec>(i, lane);
            gain[i] = p.gamma && c < C ? ld_f(p.gamma + c) : 1.f;
            bias[i] = p.beta && c < C ? ld_f(p.beta + c) : 0.f;
        }
    }
    if (kCheckpoint && blockIdx.x == gridDim.x - 1) clear_row_padding(p.c, p.rows, threadIdx.x, blockDim.x);
    const float per = 1.f / (float)C;
    const int step = gridDim.x * p.groups;
    Raw<T> next[kParts];
    long long row = (long long)blockIdx.x * p.groups + group;
    auto load = [&](long long r) {
#pragma unroll
        for (int k = 0; k < kParts; ++k)
            if (r < p.rows) load_seg<kVec>(p.x + (size_t)r * C + first + k * kSeg, C - first - k * kSeg, lane, next[k]);
    };
    load(row);
    for (; row < p.rows; row += step) {
        Raw<T> cur[kParts];
#pragma unroll
        for (int k = 0; k < kParts; ++k) cur[k] = next[k];
        load(row + step);
        float a = 0.f;
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) a += value(cur[k], i);
        const float mean = sum(a, 0.f).x * per;
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = value(cur[k], i) - mean;
                if (first + k * kSeg + seg_col<T, kVec>(i, lane) < C) q = fmaf(d, d, q);
            }
        const float rstd = 1.f / sqrtf(sum(q, 0.f).x * per + p.eps);
        if (threadIdx.x % (32 * p.warps) == 0) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            const int at = first + k * kSeg;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float g, b;
                if constexpr (kKept) {
                    g = gain[i];
                    b = bias[i];
                } else {
                    const int c = at + seg_col<T, kVec>(i, lane);
                    g = p.gamma && c < C ? ld_f(p.gamma + c) : 1.f;
                    b = p.beta && c < C ? ld_f(p.beta + c) : 0.f;
                }
                v[i] = fmaf((value(cur[k], i) - mean) * rstd, g, b);
                if (kCheckpoint && at + seg_col<T, kVec>(i, lane) >= C) v[i] = 0.f;
            }
            const Raw<T> out = to_raw(v, T());
            store_seg<kVec>(p.y + (size_t)row * C + at, C - at, lane, out);
            if (kCheckpoint && at < p.c.wide) store_blocks<T, kVec>(p.c, (int)row, at, lane, out);
        }
    }
}

template <class T>
vgc_status forward_as(const void *x, const float *gamma, const float *beta, int rows, int features, float eps, void *y, float *mean,
                      float *rstd, void *checkpoint, cudaStream_t st)
{
    Forward<T> p;
    p.x = static_cast<const T *>(x);
    p.y = static_cast<T *>(y);
    p.gamma = gamma; p.beta = beta; p.mean = mean; p.rstd = rstd;
    p.rows = rows; p.features = features; p.eps = eps;
    p.c = {};
    if (checkpoint) p.c = checkpoint_at(checkpoint, rows, features);
    const int parts = features > 32 * kSeg ? 2 : 1;
    p.warps = (features + parts * kSeg - 1) / (parts * kSeg);
    // eight warps a block where rows are short, but no fewer blocks than SMs
    p.groups = p.warps <= 8 ? 8 / p.warps : 1;
    const int spread = (rows + kSmCount - 1) / kSmCount;
    if (p.groups > spread) p.groups = spread;
    const int threads = 32 * p.warps * p.groups, resident = kSmCount * (1024 / threads);
    const int need = (int)(((long long)rows + p.groups - 1) / p.groups);
    const bool vec = (size_t)features * sizeof(T) % 16 == 0;
    auto pick = [&](auto part) {
        constexpr int kParts = decltype(part)::value;
        return checkpoint ? (vec ? norm_forward<T, true, kParts, true> : norm_forward<T, false, kParts, true>)
                          : (vec ? norm_forward<T, true, kParts, false> : norm_forward<T, false, kParts, false>);
    };
    auto fn = parts == 2 ? pick(std::integral_constant<int, 2>()) : pick(std::integral_constant<int, 1>());
    VGC_CUDA_OK(launch_kernel(fn, dim3((unsigned)(need < resident ? need : resident)), dim3((unsigned)threads), 0, st, true, p));
    count_launch();
    return VGC_OK;
}

// ---- backward -----------------------------------------------------------------------------------------------------------------
enum { kRows = 0, kSamples = 1, kPieces = 2 };

struct Plan {
    bool wide;                       // the rows' two means come from norm_row_sums
    int mode, parts, warps, groups, blocks, pieces, length;      // kPieces: pieces of a sample, rows of a piece
    int sums;                        // columns sums that a block leaves
    size_t row_sums_bytes, bytes;
};
Plan plan_backward(int rows, int features, int per_example)
{
    Plan p;
    p.wide = features > 32 * kSeg;
    p.parts = !p.wide && features > 16 * kSeg ? 2 : 1;
    p.warps = p.wide ? 1 : (features + p.parts * kSeg - 1) / (p.parts * kSeg);
    p.groups = p.wide ? 8 : p.warps <= 8 ? 8 / p.warps : 1;
    const int slabs = p.wide ? (features + kSeg - 1) / kSeg : 1, threads = 32 * p.warps * p.groups;
    // blocks that an SM holds, next to one another: by registers
    const int resident = kSmCount * (threads <= 256 ? 2 : 1);
    const int target = (resident + slabs - 1) / slabs, samples = rows / per_example;
    p.pieces = 1;
    p.length = per_example;
    if (per_example == 1) {
        p.mode = kRows;
        p.blocks = (int)(((long long)rows + p.groups - 1) / p.groups);
        if (p.blocks > target) p.blocks = target;
    } else if ((long long)samples >= (long long)target * p.groups) {
        p.mode = kSamples;
        p.blocks = target;
    } else {
        p.mode = kPieces;
        p.pieces = (target + samples - 1) / samples;
        const int most = (per_example + p.groups - 1) / p.groups;
        if (p.pieces > most) p.pieces = most;
        p.length = (per_example + p.pieces - 1) / p.pieces;
        p.pieces = (per_example + p.length - 1) / p.length;
        p.blocks = samples * p.pieces;
    }
    p.sums = p.mode == kPieces ? 2 : 4;
    p.row_sums_bytes = p.wide ? round_up((size_t)rows * sizeof(float2), 256) : 0;
    p.bytes = p.row_sums_bytes + (size_t)p.blocks * p.sums * features * sizeof(float);
    return p;
}

template <class T>
struct Backward {
    const T *x, *dy;
    T *dx;
    const float *gamma, *mean, *rstd;
    const float2 *row_sums;          // wide: mean(w), mean(w xh) of every row
    float *partial;                  // [blocks][sums][features]
    int rows, features, warps, groups;
    int per_example, pieces, length;
};

template <class T, bool kVec, int kParts, int kMode, bool kWide>
__global__ void __launch_bounds__(512, 1) norm_backward(const Backward<T> p)
{
    __shared__ float2 slots[8][64];
    __shared__ float joined[kParts == 1 ? 8 * kSeg : 1];      // column sums of a block's groups: groups * warps <= 8
    const int lane = threadIdx.x & 31, all = threadIdx.x >> 5, group = all / p.warps, warp = all - group * p.warps;
    RowSum sum = {slots[group], p.warps, warp, lane, 1 + group, 0};
    grid_release();
    grid_wait();
    const int C = p.features, first = (kWide ? blockIdx.y * kSeg : 0) + warp * kParts * kSeg;
    float gain[kParts][8];
    float xh_dy[kParts][8] = {}, dy_sum[kParts][8] = {};                       // of all rows, or of the running sample
    constexpr int kKept = kMode == kSamples ? 2 : 0, kSquares = kMode == kPieces ? 0 : 2;
    float kept[kKept ? 2 : 1][kParts][8] = {}, squares[kSquares ? 2 : 1][kParts][8] = {};
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = first + k * kSeg + seg_col<T, kVec>(i, lane);
            gain[k][i] = c >= C ? 0.f : p.gamma ? ld_f(p.gamma + c) : 1.f;
        }

    // the rows of this group: from `row` on in steps, up to `end`; whole samples in steps of samples
    long long row, end, step;
    int left = 0;                                             // rows of the sample behind this one
    if constexpr (kMode == kPieces) {
        const int sample = blockIdx.x / p.pieces, piece = blockIdx.x - sample * p.pieces;
        const long long start = (long long)sample * p.per_example;
        row = start + (long long)piece * p.length + group;
        end = min(start + p.per_example, start + (long long)(piece + 1) * p.length);
        step = p.groups;
    } else {
        row = ((long long)blockIdx.x * p.groups + group) * p.per_example;
        step = (long long)gridDim.x * p.groups * p.per_example;
        end = p.rows;
        left = p.per_example - 1;
    }
    auto after = [&](long long r) {                           // the row behind row r
        if constexpr (kMode == kSamples) return left > 0 ? r + 1 : r + step - (p.per_example - 1);
        else return r + step;
    };
    const float per = 1.f / (float)C;
    Raw<T> next_x[kParts], next_d[kParts];
    float next_mean = 0.f, next_rstd = 0.f;
    float2 next_sums = make_float2(0.f, 0.f);
    auto load = [&](long long r) {
        if (r >= end) return;
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            load_seg<kVec>(p.x + (size_t)r * C + first + k * kSeg, C - first - k * kSeg, lane, next_x[k]);
            load_seg<kVec>(p.dy + (size_t)r * C + first + k * kSeg, C - first - k * kSeg, lane, next_d[k]);
        }
        next_mean = ld_f(p.mean + r);
        next_rstd = ld_f(p.rstd + r);
        if (kWide) next_sums = make_float2(ld_f(&p.row_sums[r].x), ld_f(&p.row_sums[r].y));
    };
    load(row);
    while (row < end) {
        Raw<T> x[kParts], d[kParts];
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            x[k] = next_x[k];
            d[k] = next_d[k];
        }
        const float mean = next_mean, rstd = next_rstd;
        float2 means = next_sums;
        const long long behind = after(row);
        load(behind);
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = (value(x[k], i) - mean) * rstd, dy = value(d[k], i), t = dy * xh, w = dy * gain[k][i];
                xh_dy[k][i] += t;
                dy_sum[k][i] += dy;
                if constexpr (kMode == kRows) {
                    squares[0][k][i] = fmaf(t, t, squares[0][k][i]);
                    squares[1][k][i] = fmaf(dy, dy, squares[1][k][i]);
                }
                a += w;
                b = fmaf(w, xh, b);
            }
        if constexpr (!kWide) {
            means = sum(a, b);
            means.x *= per;
            means.y *= per;
        }
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = (value(x[k], i) - mean) * rstd, w = value(d[k], i) * gain[k][i];
                v[i] = rstd * (w - means.x - xh * means.y);
            }
            store_seg<kVec>(p.dx + (size_t)row * C + first + k * kSeg, C - first - k * kSeg, lane, to_raw(v, T()));
        }
        if constexpr (kMode == kSamples) {
            if (left == 0) {
#pragma unroll
                for (int k = 0; k < kParts; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        kept[0][k][i] += xh_dy[k][i];
                        kept[1][k][i] += dy_sum[k][i];
                        squares[0][k][i] = fmaf(xh_dy[k][i], xh_dy[k][i], squares[0][k][i]);
                        squares[1][k][i] = fmaf(dy_sum[k][i], dy_sum[k][i], squares[1][k][i]);
                        xh_dy[k][i] = dy_sum[k][i] = 0.f;
                    }
            }
            left = left == 0 ? p.per_example - 1 : left - 1;
        }
        row = behind;
    }

    // the groups' sums in the groups' order, then the block's row of partial sums
    float *const out = p.partial + (size_t)blockIdx.x * (kSquares ? 4 : 2) * C;
#pragma unroll
    for (int q = 0; q < (kSquares ? 4 : 2); ++q) {
        float v[kParts][8];
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[k][i] = q >= 2 ? squares[kSquares ? q - 2 : 0][k][i] : kMode == kSamples ? kept[kKept ? q : 0][k][i] : q == 0 ? xh_dy[k][i] : dy_sum[k][i];
        if constexpr (kParts == 1) {
            if (p.groups > 1) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 8; ++i) joined[all * kSeg + 32 * i + lane] = v[0][i];
                __syncthreads();
                if (group > 0) continue;
                for (int g = 1; g < p.groups; ++g)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[0][i] += joined[(g * p.warps + warp) * kSeg + 32 * i + lane];
            }
        }
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = first + k * kSeg + seg_col<T, kVec>(i, lane);
                if (c < C) out[(size_t)q * C + c] = v[k][i];
            }
    }
}

// mean(w) and mean(w xh) of every row, a block a row
template <class T, bool kVec>
__global__ void __launch_bounds__(512) norm_row_sums(const Backward<T> p, float2 *out)
{
    __shared__ float2 slots[64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, C = p.features;
    RowSum sum = {slots, warps, warp, lane, 1, 0};
    grid_release();
    grid_wait();
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const float mean = ld_f(p.mean + row), rstd = ld_f(p.rstd + row);
        float a = 0.f, b = 0.f;
        for (int first = warp * kSeg; first < C; first += warps * kSeg) {
            Raw<T> x, d;
            load_seg<kVec>(p.x + (size_t)row * C + first, C - first, lane, x);
            load_seg<kVec>(p.dy + (size_t)row * C + first, C - first, lane, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = first + seg_col<T, kVec>(i, lane);
                const float w = c >= C ? 0.f : value(d, i) * (p.gamma ? ld_f(p.gamma + c) : 1.f);
                a += w;
                b = fmaf(w, (value(x, i) - mean) * rstd, b);
            }
        }
        const float2 s = sum(a, b);
        if (threadIdx.x == 0) out[row] = make_float2(s.x / (float)C, s.y / (float)C);
    }
}

// The blocks' partial sums of 32 features, each of eight warps an eighth of them, added in order.
// samples == 0: partial [n][4][C].  Otherwise [samples][pieces][2][C]: a sample's pieces are added, then squared.
struct Combine {
    const float *partial;
    int n, samples, pieces, features;
    float scale_g, scale_s;
    int accumulate_g, accumulate_s;
    float *out[4];                   // g_gamma, g_beta, s_gamma, s_beta
};
__global__ void __launch_bounds__(256) norm_combine(const Combine p)
{
    __shared__ float part[4][8][32];
    grid_release();
    grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const size_t C = (size_t)p.features;
    float v[4] = {};
    if (c < p.features) {
        if (p.samples == 0) {
            const int each = (p.n + 7) / 8, last = min(p.n, (warp + 1) * each);
#pragma unroll 4
            for (int b = warp * each; b < last; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] += ld_f(p.partial + ((size_t)b * 4 + q) * C + c);
        } else {
            const int each = (p.samples + 7) / 8, last = min(p.samples, (warp + 1) * each);
            for (int s = warp * each; s < last; ++s) {
                float a = 0.f, b = 0.f;
#pragma unroll 4
                for (int i = 0; i < p.pieces; ++i) {
                    const float *const at = p.partial + ((size_t)s * p.pieces + i) * 2 * C + c;
                    a += ld_f(at);
                    b += ld_f(at + C);
                }
                v[0] += a;
                v[1] += b;
                v[2] = fmaf(a, a, v[2]);
                v[3] = fmaf(b, b, v[3]);
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) part[q][warp][lane] = v[q];
    __syncthreads();
    float *const to = warp == 0 ? p.out[0] : warp == 1 ? p.out[1] : warp == 2 ? p.out[2] : p.out[3];
    if (warp >= 4 || c >= p.features || !to) return;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[warp][w][lane];
    s *= warp < 2 ? p.scale_g : p.scale_s;
    to[c] = (warp < 2 ? p.accumulate_g : p.accumulate_s) ? ld_f(to + c) + s : s;
}

template <class T>
vgc_status backward_as(const void *x, const void *dy, const float *gamma, const float *mean, const float *rstd, int rows,
                       int features, int per_example, void *dx, const Plan &plan, void *ws, cudaStream_t st)
{
    Backward<T> p;
    p.x = static_cast<const T *>(x);
    p.dy = static_cast<const T *>(dy);
    p.dx = static_cast<T *>(dx);
    p.gamma = gamma; p.mean = mean; p.rstd = rstd;
    float2 *const row_sums = static_cast<float2 *>(ws);
    p.row_sums = row_sums;
    p.partial = reinterpret_cast<float *>(static_cast<char *>(ws) + plan.row_sums_bytes);
    p.rows = rows; p.features = features; p.warps = plan.warps; p.groups = plan.groups;
    p.per_example = per_example; p.pieces = plan.pieces; p.length = plan.length;
    const bool vec = (size_t)features * sizeof(T) % 16 == 0;
    if (plan.wide) {
        const int most = kSmCount * 4;
        VGC_CUDA_OK(launch_kernel(vec ? norm_row_sums<T, true> : norm_row_sums<T, false>, dim3((unsigned)(rows < most ? rows : most)),
                                  dim3(512), 0, st, true, p, row_sums));
        count_launch();
    }
    auto pick = [&](auto mode) {
        constexpr int kMode = decltype(mode)::value;
        if (plan.wide) return vec ? norm_backward<T, true, 1, kMode, true> : norm_backward<T, false, 1, kMode, true>;
        if (plan.parts == 2) return vec ? norm_backward<T, true, 2, kMode, false> : norm_backward<T, false, 2, kMode, false>;
        return vec ? norm_backward<T, true, 1, kMode, false> : norm_backward<T, false, 1, kMode, false>;
    };
    auto fn = plan.mode == kRows ? pick(std::integral_constant<int, kRows>())
              : plan.mode == kSamples ? pick(std::integral_constant<int, kSamples>()) : pick(std::integral_constant<int, kPieces>());
    VGC_CUDA_OK(launch_kernel(fn, dim3((unsigned)plan.blocks, plan.wide ? (unsigned)((features + kSeg - 1) / kSeg) : 1u),
                              dim3((unsigned)(32 * plan.warps * plan.groups)), 0, st, true, p));
    count_launch();
    return VGC_OK;
}

bool type_ok(vgc_type type) { return type == VGC_FP32 || type == VGC_BF16; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace
}  // namespace vgc

using namespace vgc;

extern "C" vgc_status vgc_layernorm(const void *x, vgc_type type, const float *gamma, const float *beta, int rows, int features,
                                    float eps, void *y, float *mean, float *rstd, void *checkpoint, vgc_stream_t stream)
{
    if (rows < 0 || rows > kMaxRows || features < 0 || !type_ok(type) || !(eps >= 0.f && eps <= FLT_MAX)) return VGC_ERR_INVALID_ARG;
    if (rows == 0 || features == 0) return VGC_OK;
    if (features > VGC_NORM_MAX_FEATURES) return VGC_ERR_UNSUPPORTED;
    if (!x || !y || !mean || !rstd || !aligned16(x) || !aligned16(y) || !aligned16(checkpoint)) return VGC_ERR_INVALID_ARG;
    if (!aligned4(gamma) || !aligned4(beta) || !aligned4(mean) || !aligned4(rstd)) return VGC_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return type == VGC_FP32 ? forward_as<float>(x, gamma, beta, rows, features, eps, y, mean, rstd, checkpoint, st)
                            : forward_as<__nv_bfloat16>(x, gamma, beta, rows, features, eps, y, mean, rstd, checkpoint, st);
}

extern "C" size_t vgc_layernorm_backward_workspace_bytes(int rows, int features, int rows_per_example)
{
    if (rows <= 0 || rows > kMaxRows || features <= 0 || features > VGC_NORM_MAX_FEATURES || rows_per_example < 1 ||
        rows % rows_per_example)
        return 0;
    return round_up(plan_backward(rows, features, rows_per_example).bytes, 256);
}

extern "C" vgc_status vgc_layernorm_backward(const void *x, const void *dy, vgc_type type, const float *gamma, const float *mean,
                                             const float *rstd, int rows, int features, int rows_per_example, float scale_g,
                                             float scale_s, int accumulate_g, int accumulate_s, void *dx, float *g_gamma,
                                             float *g_beta, float *s_gamma, float *s_beta, void *ws, size_t ws_bytes,
                                             vgc_stream_t stream)
{
    if (rows < 0 || rows > kMaxRows || features < 0 || !type_ok(type) || rows_per_example < 1 || rows % rows_per_example)
        return VGC_ERR_INVALID_ARG;
    if (!(scale_g == scale_g) || !(scale_s == scale_s)) return VGC_ERR_INVALID_ARG;
    if (features == 0) return VGC_OK;
    if (features > VGC_NORM_MAX_FEATURES) return VGC_ERR_UNSUPPORTED;
    if (!aligned4(g_gamma) || !aligned4(g_beta) || !aligned4(s_gamma) || !aligned4(s_beta)) return VGC_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    Combine c;
    c.out[0] = g_gamma; c.out[1] = g_beta; c.out[2] = s_gamma; c.out[3] = s_beta;
    c.accumulate_g = accumulate_g; c.accumulate_s = accumulate_s;
    if (rows == 0) {                                          // empty sums
        for (int q = 0; q < 4; ++q)
            if (c.out[q] && !(q < 2 ? accumulate_g : accumulate_s))
                VGC_CUDA_OK(cudaMemsetAsync(c.out[q], 0, (size_t)features * sizeof(float), st));
        return VGC_OK;
    }
    if (!x || !dy || !dx || !mean || !rstd || !aligned16(x) || !aligned16(dy) || !aligned16(dx)) return VGC_ERR_INVALID_ARG;
    if (!aligned4(gamma) || !aligned4(mean) || !aligned4(rstd)) return VGC_ERR_INVALID_ARG;
    const Plan plan = plan_backward(rows, features, rows_per_example);
    if (!ws || !aligned16(ws) || ws_bytes < plan.bytes) return VGC_ERR_WORKSPACE;
    const vgc_status rc = type == VGC_FP32
        ? backward_as<float>(x, dy, gamma, mean, rstd, rows, features, rows_per_example, dx, plan, ws, st)
        : backward_as<__nv_bfloat16>(x, dy, gamma, mean, rstd, rows, features, rows_per_example, dx, plan, ws, st);
    if (rc != VGC_OK) return rc;
    if (!g_gamma && !g_beta && !s_gamma && !s_beta) return VGC_OK;
    c.partial = reinterpret_cast<const float *>(static_cast<const char *>(ws) + plan.row_sums_bytes);
    c.n = plan.blocks;
    c.samples = plan.mode == kPieces ? rows / rows_per_example : 0;
    c.pieces = plan.pieces;
    c.features = features; c.scale_g = scale_g; c.scale_s = scale_s;
    VGC_CUDA_OK(launch_kernel(norm_combine, dim3((unsigned)((features + 31) / 32)), dim3(256), 0, st, true, c));
    count_launch();
    return VGC_OK;
}
