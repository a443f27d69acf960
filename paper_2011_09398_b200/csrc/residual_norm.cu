// The boundary between two blocks of a residual stream in one pass: the norm behind a block, its gate and residual scale, the
// shortcut add, the norm in front of the next block and that block's LceQuantize.
//
// What bounds it is reading x, the block's output and the gate and writing y and the result once each: a row stays in the
// registers of the threads that loaded it, eight channels to a thread and vector, through up to four sums over the row (both
// norms, variances from the differences to the mean), all in fp32.
//
// Sign bits want more: a bit is the sign of a difference of rounded numbers, and next to zero fp32 gets it wrong.  So with them a
// bound on every result's error is worked out beside it, and a row in which some result is not clear of zero by it (7% of rows of
// 4000 channels) goes through once more in fp64.  (Everything in fp64 at once: 188 us for 8000 x 4000 fp32, most of it conversions.)
#include "kv_common.cuh"

#include <math.h>

namespace lce {
namespace {

constexpr int kMaxChannels = 16384;

struct NormParams {
    int64_t rows;
    int32_t channels, vectors;         // vectors of eight channels, whole words of 32
    int32_t post_norm, pre_norm, sigmoid, row_threads;
    float eps, residual_scale;
    int64_t x_stride, branch_stride, gate_stride, y_stride, normed_stride;
    const float *post_weight, *post_bias, *pre_weight, *pre_bias;
    uint8_t *packed;
};

__device__ __forceinline__ float sigmoid_of(float g) { return 1.0f / (1.0f + expf(-g)); }
__device__ __forceinline__ double sigmoid_of(double g) { return 1.0 / (1.0 + exp(-g)); }
__device__ __forceinline__ float inverse_root(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double inverse_root(double v) { return 1.0 / sqrt(v); }

// Sums over the threads of a row, in every one of them.
template <typename A, int M>
__device__ __forceinline__ void row_sums(A (&v)[M], int row_threads, A (*warps)[32])
{
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] += __shfl_xor_sync(0xffffffffu, v[m], d);
    if (row_threads == 32) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();  // the last sums have been read
    if (lane == 0)
#pragma unroll
        for (int m = 0; m < M; ++m) warps[m][warp] = v[m];
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = lane < row_threads / 32 ? warps[m][lane] : A(0);
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] += __shfl_xor_sync(0xffffffffu, v[m], d);
}

// Sum of a thread's values, in pairs: few roundings deep
template <typename A, int N>
__device__ __forceinline__ A sum_of(const A (&v)[N][8])
{
    A s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = ((v[k][0] + v[k][1]) + (v[k][2] + v[k][3])) + ((v[k][4] + v[k][5]) + (v[k][6] + v[k][7]));
    return N == 2 ? s[0] + s[N - 1] : s[0];
}
template <typename A, int N>
__device__ __forceinline__ A squares_of(const A (&v)[N][8])
{
    A q[N][8];
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) q[k][i] = v[k][i] * v[k][i];
    return sum_of(q);
}

template <typename A>
struct RowNorm {
    A mean, factor;  // (v - mean) * factor
};

// v := v - mean (LAYER), and the factor that norms it.  `more` is summed over the row along the way.
template <typename A, int N>
__device__ __forceinline__ RowNorm<A> row_norm(A (&v)[N][8], int kind, const NormParams &p, const int (&channel)[N], A (*warps)[32], A *more = nullptr)
{
    const A each = A(1) / A(p.channels);
    RowNorm<A> n{A(0), A(1)};
    if (kind == LCE_NORM_LAYER) {
        A sum[1] = {sum_of(v)};  // 0 behind the last channel
        row_sums(sum, p.row_threads, warps);
        n.mean = sum[0] * each;
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = channel[k] + i < p.channels ? v[k][i] - n.mean : A(0);
    }
    if (more) {
        A sums[2] = {squares_of(v), *more};
        row_sums(sums, p.row_threads, warps);
        if (kind != LCE_NORM_NONE) n.factor = inverse_root(sums[0] * each + A(p.eps));
        *more = sums[1];
    } else if (kind != LCE_NORM_NONE) {
        A sums[1] = {squares_of(v)};
        row_sums(sums, p.row_threads, warps);
        n.factor = inverse_root(sums[0] * each + A(p.eps));
    }
    return n;
}

template <typename TS, typename TB>
struct NormRow {  // one row's tensors
    const TS *x;
    const TB *branch, *gate;
    TS *y;
    TB *normed;
    uint8_t *packed;
};

// Errors of the fp32 arithmetic are below kUnsure times the sizes that meet in a value: sums of 14 levels of roundings, twice
// (mean and variance), and a dozen roundings, of 2^-24 each.
constexpr float kUnsure = 0x1p-18f;

// The row in the arithmetic A.  CHECKED: writes nothing and returns false where a sign is in doubt.
template <typename TS, typename TB, typename A, int N, bool VEC, bool CHECKED>
__device__ __forceinline__ bool norm_row(const NormParams &p, const NormRow<TS, TB> &row, int thread, A (*warps)[32])
{
    A v[N][8];
    int channel[N];
#pragma unroll
    for (int k = 0; k < N; ++k) channel[k] = 8 * (thread + k * p.row_threads);
    float f[8];
    float size[CHECKED ? N : 1][8];  // of what meets in y
    if (row.branch) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            load8<TB, VEC>(row.branch + channel[k], p.channels - channel[k], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[k][i] = f[i];
                if (CHECKED) size[k][i] = fabsf(f[i]);
            }
        }
        RowNorm<A> n{A(0), A(1)};
        if (p.post_norm != LCE_NORM_NONE) n = row_norm(v, p.post_norm, p, channel, warps);
        const float mean_size = fabsf((float)n.mean);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int count = p.channels - channel[k];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[k][i] *= n.factor;
                if (CHECKED) size[k][i] = (size[k][i] + mean_size) * (float)n.factor;
            }
            if (p.post_weight) {
                load8<float, VEC>(p.post_weight + channel[k], count, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[k][i] *= A(f[i]);
                    if (CHECKED) size[k][i] *= fabsf(f[i]);
                }
            }
            if (p.post_bias) {
                load8<float, VEC>(p.post_bias + channel[k], count, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[k][i] += A(f[i]);
                    if (CHECKED) size[k][i] += fabsf(f[i]);
                }
            }
            float g[8];
            if (row.gate) {
                load8<TB, VEC>(row.gate + channel[k], count, g);
                load8<TS, VEC>(row.x + channel[k], count, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const A by = A(p.residual_scale) * (p.sigmoid ? sigmoid_of(A(g[i])) : A(g[i]));
                    v[k][i] = i < count ? A(f[i]) + by * v[k][i] : A(0);
                    if (CHECKED) size[k][i] = fabsf(f[i]) + fabsf((float)by) * size[k][i];
                }
            } else {
                load8<TS, VEC>(row.x + channel[k], count, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[k][i] = i < count ? A(f[i]) + A(p.residual_scale) * v[k][i] : A(0);
                    if (CHECKED) size[k][i] = fabsf(f[i]) + fabsf(p.residual_scale) * size[k][i];
                }
            }
            if (CHECKED) {
#pragma unroll
                for (int i = 0; i < 8; ++i) size[k][i] = i < count ? size[k][i] : 0.0f;
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            load8<TS, VEC>(row.x + channel[k], p.channels - channel[k], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[k][i] = f[i];
                if (CHECKED) size[k][i] = fabsf(f[i]);
            }
        }
    }
    if (!CHECKED && row.y) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)v[k][i];
            store8<TS, VEC>(row.y + channel[k], p.channels - channel[k], f);
        }
    }
    if (!row.normed && !row.packed) return true;
    float y[CHECKED ? N : 1][8];
    float row_size = 0.0f;  // root mean square of the sizes
    RowNorm<A> n{A(0), A(1)};
    if (CHECKED) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) y[CHECKED ? k : 0][i] = (float)v[k][i];
        A more = (A)squares_of(size);
        if (p.pre_norm != LCE_NORM_NONE) {
            n = row_norm(v, p.pre_norm, p, channel, warps, &more);
            row_size = sqrtf((float)more / (float)p.channels);
        }
    } else if (p.pre_norm != LCE_NORM_NONE) {
        n = row_norm(v, p.pre_norm, p, channel, warps);
    }
    bool sure = true;
    uint32_t bits[N];
    const float spread = (1.0f + (float)n.factor * row_size) * (float)n.factor;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int count = p.channels - channel[k];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[k][i] *= n.factor;
            if (CHECKED) size[k][i] = (size[k][i] + row_size) * spread;
        }
        if (p.pre_weight) {
            load8<float, VEC>(p.pre_weight + channel[k], count, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[k][i] *= A(f[i]);
                if (CHECKED) size[k][i] *= fabsf(f[i]);
            }
        }
        if (p.pre_bias) {
            load8<float, VEC>(p.pre_bias + channel[k], count, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[k][i] += A(f[i]);
                if (CHECKED) size[k][i] += fabsf(f[i]);
            }
        }
        if (!CHECKED && row.normed) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)v[k][i];
            store8<TB, VEC>(row.normed + channel[k], count, f);
        }
        bits[k] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            bits[k] |= (i < count && v[k][i] < A(0) ? 1u : 0u) << i;
            // a row with an infinity or a NaN is in doubt throughout; zeros of zeros are not
            if (CHECKED) sure = sure && (i >= count || fabsf((float)v[k][i]) > kUnsure * size[k][i] || size[k][i] == 0.0f);
        }
    }
    if (CHECKED) {
        sure = p.row_threads == 32 ? __all_sync(0xffffffffu, sure) : __syncthreads_and(sure);
        if (!sure) return false;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (row.y) store8<TS, VEC>(row.y + channel[k], p.channels - channel[k], y[CHECKED ? k : 0]);
            if (row.normed) {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = (float)v[k][i];
                store8<TB, VEC>(row.normed + channel[k], p.channels - channel[k], f);
            }
        }
    }
    // eight bits are a byte of their word: lowest channel lowest, the lowest byte first in memory
    if (row.packed) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (channel[k] < 8 * p.vectors) row.packed[channel[k] / 8] = (uint8_t)bits[k];
    }
    return true;
}

// TS, TB: elements of the stream and of the block; N vectors to a thread.
template <typename TS, typename TB, int N, bool VEC, bool BITS>
__global__ void __launch_bounds__(N == 1 ? 512 : 1024) residual_norm_kernel(const __grid_constant__ NormParams p, const TS *x, const TB *branch, const TB *gate,
                                                                            TS *y, TB *normed)
{
    __shared__ float warps[2][32];
    __shared__ double wide_warps[1][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t at = p.row_threads == 32 ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (at >= p.rows) return;
    const int thread = p.row_threads == 32 ? threadIdx.x & 31 : threadIdx.x;
    const NormRow<TS, TB> row{x + at * p.x_stride, branch ? branch + at * p.branch_stride : nullptr, gate ? gate + at * p.gate_stride : nullptr,
                              y ? y + at * p.y_stride : nullptr, normed ? normed + at * p.normed_stride : nullptr,
                              BITS ? p.packed + at * p.vectors : nullptr};
    if (!BITS) norm_row<TS, TB, float, N, VEC, false>(p, row, thread, warps);
    else if (!norm_row<TS, TB, float, N, VEC, true>(p, row, thread, warps)) norm_row<TS, TB, double, N, VEC, false>(p, row, thread, wide_warps);
}

struct NormBuffers {
    const void *x, *branch, *gate;
    void *y, *normed;
};

template <typename TS, typename TB, int N, bool VEC, bool BITS>
lce_status launch(NormParams p, const NormBuffers &b, cudaStream_t s)
{
    int64_t blocks = p.rows;
    int threads = p.row_threads;
    if (threads == 32) {
        threads = 128;
        blocks = (p.rows + 3) / 4;
    }
    if (blocks >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    return launch_dependent(residual_norm_kernel<TS, TB, N, VEC, BITS>, dim3((unsigned)blocks), threads, 0, s, p, static_cast<const TS *>(b.x),
                            static_cast<const TB *>(b.branch), static_cast<const TB *>(b.gate), static_cast<TS *>(b.y), static_cast<TB *>(b.normed));
}

template <typename TS, typename TB, bool VEC, bool BITS>
lce_status launch_vectors(NormParams p, const NormBuffers &b, cudaStream_t s)
{
    // a warp to a row of up to 1024 channels, otherwise a block
    const auto threads = [&](int n) { return (p.vectors + 32 * n - 1) / (32 * n) * 32; };
    const int n = p.vectors <= 32 ? 1 : p.vectors <= 64 ? 2 : p.vectors <= 512 ? 1 : 2;
    p.row_threads = threads(n);
    return n == 1 ? launch<TS, TB, 1, VEC, BITS>(p, b, s) : launch<TS, TB, 2, VEC, BITS>(p, b, s);
}

template <typename TS, typename TB>
lce_status launch_types(const NormParams &p, const NormBuffers &b, cudaStream_t s)
{
    const auto rows16 = [&](const void *q, int64_t stride, size_t size) { return !q || (aligned(q, 16) && stride * size % 16 == 0); };
    const bool vec = p.channels % 8 == 0 && rows16(b.x, p.x_stride, sizeof(TS)) && rows16(b.y, p.y_stride, sizeof(TS)) && rows16(b.branch, p.branch_stride, sizeof(TB)) &&
                     rows16(b.gate, p.gate_stride, sizeof(TB)) && rows16(b.normed, p.normed_stride, sizeof(TB)) && aligned(p.post_weight, 16) &&
                     aligned(p.post_bias, 16) && aligned(p.pre_weight, 16) && aligned(p.pre_bias, 16);
    if (p.packed) return vec ? launch_vectors<TS, TB, true, true>(p, b, s) : launch_vectors<TS, TB, false, true>(p, b, s);
    return vec ? launch_vectors<TS, TB, true, false>(p, b, s) : launch_vectors<TS, TB, false, false>(p, b, s);
}

}  // namespace
}  // namespace lce

extern "C" lce_status lce_residual_norm(const lce_residual_norm_desc *desc, const void *x, const void *branch, const void *gate, const float *post_weight,
                                        const float *post_bias, const float *pre_weight, const float *pre_bias, void *y, void *normed, uint32_t *packed,
                                        void *stream)
{
    using namespace lce;
    if (!desc) return LCE_ERR_INVALID_ARG;
    const auto norm_known = [](int32_t n) { return n >= LCE_NORM_NONE && n <= LCE_NORM_LAYER; };
    if (desc->rows < 0 || desc->channels <= 0 || !norm_known(desc->post_norm) || !norm_known(desc->pre_norm) || !type_known(desc->type) ||
        !type_known(desc->stream_type))
        return LCE_ERR_INVALID_ARG;
    if (desc->gate_activation != LCE_ACT_NONE && desc->gate_activation != LCE_ACT_SIGMOID) return LCE_ERR_INVALID_ARG;
    if (!(desc->eps >= 0.0f) || !isfinite(desc->eps) || !isfinite(desc->residual_scale)) return LCE_ERR_INVALID_ARG;
    for (const int64_t s : {desc->x_stride, desc->branch_stride, desc->gate_stride, desc->y_stride, desc->normed_stride})
        if (s < 0 || s >= (1ll << 40)) return LCE_ERR_INVALID_ARG;
    if (desc->channels > kMaxChannels) return LCE_ERR_UNSUPPORTED;
    if (desc->stream_type != desc->type && desc->stream_type != LCE_TYPE_FLOAT32) return LCE_ERR_UNSUPPORTED;
    if (desc->rows >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    if (desc->rows == 0) return LCE_OK;
    if (!y && !normed && !packed) return LCE_ERR_INVALID_ARG;
    if (!branch && (gate || desc->post_norm != LCE_NORM_NONE || post_weight || post_bias)) return LCE_ERR_INVALID_ARG;
    if (!x) return LCE_ERR_INVALID_ARG;
    // rows that are written do not run into one another
    if (desc->rows > 1 && ((y && desc->y_stride < desc->channels) || (normed && desc->normed_stride < desc->channels))) return LCE_ERR_INVALID_ARG;
    const size_t stream_size = type_size(desc->stream_type), size = type_size(desc->type);
    if (!aligned(x, stream_size) || !aligned(y, stream_size) || !aligned(branch, size) || !aligned(gate, size) || !aligned(normed, size) || !aligned(packed, 4) ||
        !aligned(post_weight, 4) || !aligned(post_bias, 4) || !aligned(pre_weight, 4) || !aligned(pre_bias, 4))
        return LCE_ERR_ALIGNMENT;
    NormParams p{};
    p.rows = desc->rows;
    p.channels = desc->channels;
    p.vectors = (desc->channels + 31) / 32 * 4;
    p.post_norm = desc->post_norm; p.pre_norm = desc->pre_norm;
    p.sigmoid = desc->gate_activation == LCE_ACT_SIGMOID;
    p.eps = desc->eps; p.residual_scale = desc->residual_scale;
    p.x_stride = desc->x_stride; p.branch_stride = desc->branch_stride; p.gate_stride = desc->gate_stride;
    p.y_stride = desc->y_stride; p.normed_stride = desc->normed_stride;
    p.post_weight = post_weight; p.post_bias = post_bias; p.pre_weight = pre_weight; p.pre_bias = pre_bias;
    p.packed = reinterpret_cast<uint8_t *>(packed);
    const NormBuffers b{x, branch, gate, y, normed};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (desc->type) {
        case LCE_TYPE_FLOAT32: return launch_types<float, float>(p, b, s);
        case LCE_TYPE_FLOAT16: return desc->stream_type == LCE_TYPE_FLOAT32 ? launch_types<float, __half>(p, b, s) : launch_types<__half, __half>(p, b, s);
        default: return desc->stream_type == LCE_TYPE_FLOAT32 ? launch_types<float, __nv_bfloat16>(p, b, s) : launch_types<__nv_bfloat16, __nv_bfloat16>(p, b, s);
    }
}
