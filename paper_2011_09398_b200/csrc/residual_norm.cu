// The boundary between two blocks of a residual stream in one pass: the norm behind a block, its gate and residual scale, the
// shortcut add, the norm in front of the next block and that block's LceQuantize.
//
// What bounds it is reading x, the block's output and the gate and writing y and the result once each: a row stays in the
// registers of the threads that loaded it, eight channels to a thread and vector, through up to four sums over the row (both
// norms, variances from the differences to the mean).  Sums are fp32, or fp64 with everything behind them where sign bits are asked
// for: a bit is the sign of a difference of rounded numbers, and next to zero only a far finer arithmetic gets it right.
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

// Sum over the threads of a row, in every one of them.
template <typename A>
__device__ __forceinline__ A row_sum(A v, int row_threads, A *warps)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (row_threads == 32) return v;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();  // the last sum has been read
    if (lane == 0) warps[warp] = v;
    __syncthreads();
    v = lane < row_threads / 32 ? warps[lane] : A(0);
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// v := (v - mean) and the factor that norms it
template <typename A, int N>
__device__ __forceinline__ A norm_factor(A (&v)[N][8], int kind, const NormParams &p, const int (&channel)[N], A *warps)
{
    const A each = A(1) / A(p.channels);
    if (kind == LCE_NORM_LAYER) {
        A sum = 0;
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[k][i];  // 0 behind the last channel
        const A mean = row_sum(sum, p.row_threads, warps) * each;
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = channel[k] + i < p.channels ? v[k][i] - mean : A(0);
    }
    A squares = 0;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) squares += v[k][i] * v[k][i];
    return inverse_root(row_sum(squares, p.row_threads, warps) * each + A(p.eps));
}

// TS, TB: elements of the stream and of the block; A: the arithmetic; N vectors to a thread.
template <typename TS, typename TB, typename A, int N, bool VEC>
__global__ void __launch_bounds__(N == 1 ? 512 : 1024) residual_norm_kernel(const __grid_constant__ NormParams p, const TS *x, const TB *branch, const TB *gate,
                                                                            TS *y, TB *normed)
{
    __shared__ A warps[32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t row = p.row_threads == 32 ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= p.rows) return;
    const int thread = p.row_threads == 32 ? threadIdx.x & 31 : threadIdx.x;
    A v[N][8];
    int channel[N];
#pragma unroll
    for (int k = 0; k < N; ++k) channel[k] = 8 * (thread + k * p.row_threads);
    float f[8];
    if (branch) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            load8<TB, VEC>(branch + row * p.branch_stride + channel[k], p.channels - channel[k], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = f[i];
        }
        const A factor = p.post_norm == LCE_NORM_NONE ? A(1) : norm_factor(v, p.post_norm, p, channel, warps);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int count = p.channels - channel[k];
            if (p.post_norm != LCE_NORM_NONE) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] *= factor;
            }
            if (p.post_weight) {
                load8<float, VEC>(p.post_weight + channel[k], count, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] *= A(f[i]);
            }
            if (p.post_bias) {
                load8<float, VEC>(p.post_bias + channel[k], count, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] += A(f[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] *= A(p.residual_scale);
            if (gate) {
                load8<TB, VEC>(gate + row * p.gate_stride + channel[k], count, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] *= p.sigmoid ? sigmoid_of(A(f[i])) : A(f[i]);
            }
            load8<TS, VEC>(x + row * p.x_stride + channel[k], count, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = i < count ? v[k][i] + A(f[i]) : A(0);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            load8<TS, VEC>(x + row * p.x_stride + channel[k], p.channels - channel[k], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = f[i];
        }
    }
    if (y) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)v[k][i];
            store8<TS, VEC>(y + row * p.y_stride + channel[k], p.channels - channel[k], f);
        }
    }
    if (!normed && !p.packed) return;
    const A factor = p.pre_norm == LCE_NORM_NONE ? A(1) : norm_factor(v, p.pre_norm, p, channel, warps);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int count = p.channels - channel[k];
        if (p.pre_norm != LCE_NORM_NONE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] *= factor;
        }
        if (p.pre_weight) {
            load8<float, VEC>(p.pre_weight + channel[k], count, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] *= A(f[i]);
        }
        if (p.pre_bias) {
            load8<float, VEC>(p.pre_bias + channel[k], count, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] += A(f[i]);
        }
        if (normed) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)v[k][i];
            store8<TB, VEC>(normed + row * p.normed_stride + channel[k], count, f);
        }
        // eight bits are a byte of their word: lowest channel lowest, the lowest byte first in memory
        if (p.packed && channel[k] < 8 * p.vectors) {
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) bits |= (i < count && v[k][i] < A(0) ? 1u : 0u) << i;
            p.packed[row * p.vectors + channel[k] / 8] = (uint8_t)bits;
        }
    }
}

struct NormBuffers {
    const void *x, *branch, *gate;
    void *y, *normed;
};

template <typename TS, typename TB, typename A, int N, bool VEC>
lce_status launch(NormParams p, const NormBuffers &b, cudaStream_t s)
{
    int64_t blocks = p.rows;
    int threads = p.row_threads;
    if (threads == 32) {
        threads = 128;
        blocks = (p.rows + 3) / 4;
    }
    if (blocks >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    return launch_dependent(residual_norm_kernel<TS, TB, A, N, VEC>, dim3((unsigned)blocks), threads, 0, s, p, static_cast<const TS *>(b.x),
                            static_cast<const TB *>(b.branch), static_cast<const TB *>(b.gate), static_cast<TS *>(b.y), static_cast<TB *>(b.normed));
}

template <typename TS, typename TB, typename A, bool VEC>
lce_status launch_vectors(NormParams p, const NormBuffers &b, cudaStream_t s)
{
    // a warp to a row of up to 1024 channels, otherwise a block
    const auto threads = [&](int n) { return (p.vectors + 32 * n - 1) / (32 * n) * 32; };
    const int n = p.vectors <= 32 ? 1 : p.vectors <= 64 ? 2 : p.vectors <= 512 ? 1 : 2;
    p.row_threads = threads(n);
    return n == 1 ? launch<TS, TB, A, 1, VEC>(p, b, s) : launch<TS, TB, A, 2, VEC>(p, b, s);
}

template <typename TS, typename TB>
lce_status launch_types(const NormParams &p, const NormBuffers &b, cudaStream_t s)
{
    const auto rows16 = [&](const void *q, int64_t stride, size_t size) { return !q || (aligned(q, 16) && stride * size % 16 == 0); };
    const bool vec = p.channels % 8 == 0 && rows16(b.x, p.x_stride, sizeof(TS)) && rows16(b.y, p.y_stride, sizeof(TS)) && rows16(b.branch, p.branch_stride, sizeof(TB)) &&
                     rows16(b.gate, p.gate_stride, sizeof(TB)) && rows16(b.normed, p.normed_stride, sizeof(TB)) && aligned(p.post_weight, 16) &&
                     aligned(p.post_bias, 16) && aligned(p.pre_weight, 16) && aligned(p.pre_bias, 16);
    if (p.packed) return vec ? launch_vectors<TS, TB, double, true>(p, b, s) : launch_vectors<TS, TB, double, false>(p, b, s);
    return vec ? launch_vectors<TS, TB, float, true>(p, b, s) : launch_vectors<TS, TB, float, false>(p, b, s);
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
