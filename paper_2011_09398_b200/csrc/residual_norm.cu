// The boundary between two blocks of a residual stream in one pass: the norm behind a block, its gate and residual scale, the
// shortcut add, the norm in front of the next block and that block's LceQuantize.
//
// What bounds it is reading x, the block's output and the gate and writing y and the result once each: a row stays in the
// registers of its threads, eight channels to a thread and vector, through up to four sums over the row (both norms, variances from the
// differences to the mean).  A block takes row after row, and while it works on one the next one is on its way to shared memory.
//
// The arithmetic is fp32, or fp64 where sign bits are asked for: a bit is the sign of a difference of rounded numbers, and next to zero
// only a far finer arithmetic gets it right.  (fp32 with a bound on its error, and fp64 for the rows in doubt, was slower: 6% of rows
// of 4000 channels are, and each holds its block up.)
#include "kv_common.cuh"

#include <math.h>

#include <algorithm>

namespace lce {
namespace {

constexpr int kMaxChannels = 16384;

struct NormParams {
    int64_t rows;
    int32_t channels, vectors;         // vectors of eight channels, whole words of 32
    int32_t post_norm, pre_norm, sigmoid, row_threads;
    int32_t stages, stage_places;      // rows in shared memory at a time; pieces of 16 bytes to a row of the block
    float eps, residual_scale;
    int64_t x_stride, branch_stride, gate_stride, y_stride, normed_stride;
    const float *post_weight, *post_bias, *pre_weight, *pre_bias;
    uint8_t *packed;
};

__device__ __forceinline__ float sigmoid_of(float g) { return 1.0f / (1.0f + expf(-g)); }
__device__ __forceinline__ double sigmoid_of(double g) { return 1.0 / (1.0 + exp(-g)); }
__device__ __forceinline__ float inverse_root(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double inverse_root(double v) { return 1.0 / sqrt(v); }

// Sum over the threads of a row, in every one of them.  `warps`: shared memory of this sum alone, so that one barrier does.
template <typename A>
__device__ __forceinline__ A row_sum(A v, int row_threads, A *warps)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (row_threads == 32) return v;
    const int lane = threadIdx.x & 31, row_warps = row_threads / 32;
    if (lane == 0) warps[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < row_warps ? warps[lane] : A(0);
    // at most sixteen warps: lanes 0 .. 15 hold all there is
#pragma unroll
    for (int d = 8; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return __shfl_sync(0xffffffffu, v, 0);
}

// Sum of a thread's values, in pairs: few roundings deep
template <typename A, int N>
__device__ __forceinline__ A sum_of(const A (&v)[N][8])
{
    A s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = ((v[k][0] + v[k][1]) + (v[k][2] + v[k][3])) + ((v[k][4] + v[k][5]) + (v[k][6] + v[k][7]));
#pragma unroll
    for (int d = 1; d < N; d *= 2)
#pragma unroll
        for (int k = 0; k + d < N; k += 2 * d) s[k] += s[k + d];
    return s[0];
}
template <typename A, int N>
__device__ __forceinline__ A squares_of(const A (&v)[N][8])
{
    A s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        A q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = v[k][2 * i] * v[k][2 * i] + v[k][2 * i + 1] * v[k][2 * i + 1];
        s[k] = (q[0] + q[1]) + (q[2] + q[3]);
    }
#pragma unroll
    for (int d = 1; d < N; d *= 2)
#pragma unroll
        for (int k = 0; k + d < N; k += 2 * d) s[k] += s[k + d];
    return s[0];
}

// v := v - mean (LAYER); returns the factor that norms it.  Squares are of the differences to the mean.
template <typename A, int N>
__device__ __forceinline__ A row_norm(A (&v)[N][8], int kind, const NormParams &p, const int (&channel)[N], A (*warps)[32])
{
    const A each = A(1) / A(p.channels);
    if (kind == LCE_NORM_LAYER) {
        const A mean = row_sum(sum_of(v), p.row_threads, warps[0]) * each;  // 0 behind the last channel
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = channel[k] + i < p.channels ? v[k][i] - mean : A(0);
    }
    return inverse_root(row_sum(squares_of(v), p.row_threads, warps[1]) * each + A(p.eps));
}

// Results of the arithmetic rounded to an output's type, once: fp64 to 16 bits by way of fp32 would round twice.
template <typename T>
__device__ __forceinline__ T rounded(float v) { return from_float<T>(v); }
template <typename T>
__device__ __forceinline__ T rounded(double v);
template <>
__device__ __forceinline__ float rounded<float>(double v) { return (float)v; }
template <>
__device__ __forceinline__ __half rounded<__half>(double v) { return __double2half(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(double v) { return __double2bfloat16(v); }

template <typename T, bool VEC, typename A>
__device__ __forceinline__ void store_rounded(T *p, int count, const A (&v)[8])
{
    if (VEC) {
        if (count <= 0) return;
        Eight<T> r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.e[i] = rounded<T>(v[i]);
        store_eight(p, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = rounded<T>(v[i]);
    }
}

template <typename TS, typename TB>
struct NormRow {  // one row's tensors
    const TS *x;
    const TB *branch, *gate;
    TS *y;
    TB *normed;
    uint8_t *packed;
};

// A row comes by asynchronous copies to shared memory.  A warp's vectors of a tensor are one run of memory, which its lanes copy 16 bytes
// next to 16 bytes and read as they need them: what a warp copies is its own, so no other barrier is needed.
template <typename T>
__device__ __forceinline__ void fetch_run(const T *row, int channels, int channel0, uint4 *to)
{
    constexpr int W = sizeof(T) / 2, PIECE = 16 / sizeof(T);
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int channel = channel0 + (i * 32 + lane) * PIECE;
        const bool there = channel < channels;  // whole pieces: channels is a multiple of eight
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to + i * 32 + lane)), "l"(row + (there ? channel : 0)),
                     "r"(there ? 16 : 0)
                     : "memory");
    }
}
template <typename T>
__device__ __forceinline__ Eight<T> take(const uint4 *from)
{
    constexpr int W = sizeof(T) / 2;
    const int lane = threadIdx.x & 31;
    Eight<T> to;
#pragma unroll
    for (int i = 0; i < W; ++i) reinterpret_cast<uint4 *>(to.e)[i] = from[lane * W + i];
    return to;
}
// `places`: a warp's, 32 N (2 sizeof(TB) + sizeof(TS)) / 2 pieces of 16 bytes: of each vector the branch's, the gate's, the stream's.
template <typename TS, typename TB, int N>
__device__ __forceinline__ void fetch_share(const NormParams &p, const NormRow<TS, TB> &row, int thread, uint4 *places)
{
    constexpr int WB = 32 * sizeof(TB) / 2, WS = 32 * sizeof(TS) / 2;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int channel0 = 8 * ((thread & ~31) + k * p.row_threads);
        uint4 *const at = places + k * (2 * WB + WS);
        if (row.branch) fetch_run(row.branch, p.channels, channel0, at);
        if (row.gate) fetch_run(row.gate, p.channels, channel0, at + WB);
        fetch_run(row.x, p.channels, channel0, at + 2 * WB);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
// The row in the arithmetic A.  VEC: it lies in `places`.
template <typename TS, typename TB, typename A, int N, bool VEC>
__device__ __forceinline__ void norm_row(const NormParams &p, const NormRow<TS, TB> &row, const uint4 *places, int thread, A (*warps)[32])
{
    constexpr int WB = 32 * sizeof(TB) / 2, WS = 32 * sizeof(TS) / 2;
    A v[N][8];
    int channel[N];
#pragma unroll
    for (int k = 0; k < N; ++k) channel[k] = 8 * (thread + k * p.row_threads);
    float f[8];
    const auto block_values = [&](int k, const TB *from, int place) {
        const Eight<TB> e = VEC ? take<TB>(places + k * (2 * WB + WS) + place) : load_eight<TB, false>(from + channel[k], p.channels - channel[k]);
        e.expand(f);
    };
    const auto stream_values = [&](int k) {
        const Eight<TS> e = VEC ? take<TS>(places + k * (2 * WB + WS) + 2 * WB) : load_eight<TS, false>(row.x + channel[k], p.channels - channel[k]);
        e.expand(f);
    };
    const auto affine = [&](int k, const float *w, const float *b) {
        Eight<float> weight, bias;
        weight = load_eight<float, VEC>(w + channel[k], w ? p.channels - channel[k] : 0);
        bias = load_eight<float, VEC>(b + channel[k], b ? p.channels - channel[k] : 0);
        if (w) {
            weight.expand(f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] *= A(f[i]);
        }
        if (b) {
            bias.expand(f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] += A(f[i]);
        }
    };
    if (row.branch) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            block_values(k, row.branch, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = A(f[i]);
        }
        const A factor = p.post_norm != LCE_NORM_NONE ? row_norm(v, p.post_norm, p, channel, warps) : A(1);
#pragma unroll
        for (int k = 0; k < N; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] *= factor;
            affine(k, p.post_weight, p.post_bias);
            if (row.gate) {
                block_values(k, row.gate, WB);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] *= p.sigmoid ? sigmoid_of(A(f[i])) : A(f[i]);
            }
            stream_values(k);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = channel[k] + i < p.channels ? A(f[i]) + A(p.residual_scale) * v[k][i] : A(0);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            stream_values(k);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = A(f[i]);
        }
    }
    if (row.y) {
#pragma unroll
        for (int k = 0; k < N; ++k) store_rounded<TS, VEC>(row.y + channel[k], p.channels - channel[k], v[k]);
    }
    if (!row.normed && !row.packed) return;
    const A factor = p.pre_norm != LCE_NORM_NONE ? row_norm(v, p.pre_norm, p, channel, warps + 2) : A(1);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int count = p.channels - channel[k];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] *= factor;
        affine(k, p.pre_weight, p.pre_bias);
        if (row.normed) store_rounded<TB, VEC>(row.normed + channel[k], count, v[k]);
        // eight bits are a byte of their word: lowest channel lowest, the lowest byte first in memory
        if (row.packed && channel[k] < 8 * p.vectors) {
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) bits |= (i < count && v[k][i] < A(0) ? 1u : 0u) << i;
            row.packed[channel[k] / 8] = (uint8_t)bits;
        }
    }
}

// TS, TB: elements of the stream and of the block; A: the arithmetic; N vectors to a thread.  A block (a warp, for short rows) takes row
// after row.
template <typename TS, typename TB, typename A, int N, bool VEC>
__global__ void __launch_bounds__(sizeof(A) == 8 && N == 2 ? 256 : 512, sizeof(A) == 8 && N == 2 ? 2 : N == 1 ? 2 : 1) residual_norm_kernel(const __grid_constant__ NormParams p, const TS *x, const TB *branch, const TB *gate, TS *y,
                                                                            TB *normed)
{
    extern __shared__ __align__(16) uint4 shared_places[];
    // of each sum over the row, mean and squares of either norm; rows take the two sets in turn, so that one barrier to a sum does
    __shared__ A warps[2][4][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const bool warp_rows = p.row_threads == 32;
    const int64_t first = warp_rows ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    const int64_t step = warp_rows ? (int64_t)gridDim.x * (blockDim.x >> 5) : gridDim.x;
    const int thread = warp_rows ? threadIdx.x & 31 : threadIdx.x;
    uint4 *const places = shared_places + (threadIdx.x >> 5) * (32 * N * (2 * sizeof(TB) + sizeof(TS)) / 2);
    const auto row_at = [&](int64_t at) {
        return NormRow<TS, TB>{x + at * p.x_stride, branch ? branch + at * p.branch_stride : nullptr, gate ? gate + at * p.gate_stride : nullptr,
                               y ? y + at * p.y_stride : nullptr, normed ? normed + at * p.normed_stride : nullptr,
                               sizeof(A) == 8 ? p.packed + at * p.vectors : nullptr};
    };
    if (VEC && first < p.rows) fetch_share<TS, TB, N>(p, row_at(first), thread, places);
    int set = 0;
    for (int64_t at = first; at < p.rows; at += step, set ^= 1) {
        const NormRow<TS, TB> row = row_at(at);
        const uint4 *here = places;
        if (VEC && p.stages == 2) {
            // the other half of the places was read a row ago
            here = places + set * p.stage_places;
            __syncwarp();
            if (at + step < p.rows) fetch_share<TS, TB, N>(p, row_at(at + step), thread, places + (set ^ 1) * p.stage_places);
            else asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
        } else if (VEC) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
        }
        norm_row<TS, TB, A, N, VEC>(p, row, here, thread, warps[set]);
        if (VEC && p.stages == 1) {
            __syncwarp();
            if (at + step < p.rows) fetch_share<TS, TB, N>(p, row_at(at + step), thread, places);
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
    p.row_threads = (p.vectors + 32 * N - 1) / (32 * N) * 32;
    int64_t blocks = p.rows;
    int threads = p.row_threads;
    if (threads == 32) {
        threads = 128;
        blocks = (p.rows + 3) / 4;
    }
    const size_t stage = VEC ? (size_t)threads * N * 8 * (2 * sizeof(TB) + sizeof(TS)) : 0;
    p.stages = 2 * stage <= 200 * 1024 ? 2 : 1;
    p.stage_places = (int32_t)(stage / 16);
    const size_t smem = p.stages * stage;
    static SmemOptIn opt_in;
    const auto kernel = residual_norm_kernel<TS, TB, A, N, VEC>;
    // (the kernel's own 2 KB count towards the 48 KB that need no opt-in)
    if (!opt_in.ensure(kernel, smem > 40 * 1024 ? std::max<size_t>(smem, 48 * 1024 + 16) : smem)) return LCE_ERR_CUDA;
    // as many blocks as the GPU holds: by registers (64 a thread, or 128 where it has more vectors), by shared memory
    const int64_t by_threads = (N == 1 ? 1024 : 512) / threads, by_memory = smem ? (int64_t)(220 * 1024 / (smem + 4096)) : 16;
    const int64_t most = 148 * std::max<int64_t>(1, std::min<int64_t>({by_threads, by_memory, 16}));
    return launch_dependent(kernel, dim3((unsigned)std::min(blocks, most)), threads, smem, s, p, static_cast<const TS *>(b.x), static_cast<const TB *>(b.branch),
                            static_cast<const TB *>(b.gate), static_cast<TS *>(b.y), static_cast<TB *>(b.normed));
}

template <typename TS, typename TB, typename A, bool VEC>
lce_status launch_vectors(const NormParams &p, const NormBuffers &b, cudaStream_t s)
{
    // A warp to a row of up to 256 or 512 channels, otherwise a block.  One vector to a thread as far as it goes in fp32; fp64 does better with
    // two (8000 rows of 4000 channels in fp32, layer norms and a gate: 119 us with one, 133 with two; with sign bits 175 and 161).
    const int vectors = p.vectors;
    if (sizeof(A) == 8) {
        if (vectors <= 32) return launch<TS, TB, A, 1, VEC>(p, b, s);
        return vectors <= 512 ? launch<TS, TB, A, 2, VEC>(p, b, s) : launch<TS, TB, A, 4, VEC>(p, b, s);
    }
    if (vectors <= 32 || (vectors > 64 && vectors <= 512)) return launch<TS, TB, A, 1, VEC>(p, b, s);
    return vectors <= 1024 ? launch<TS, TB, A, 2, VEC>(p, b, s) : launch<TS, TB, A, 4, VEC>(p, b, s);
}

template <typename TS, typename TB>
lce_status launch_types(const NormParams &p, const NormBuffers &b, cudaStream_t s)
{
    const auto rows = [&](const void *q, int64_t stride, size_t size) { return !q || (aligned(q, 8 * size) && stride % 8 == 0); };
    const bool vec = p.channels % 8 == 0 && rows(b.x, p.x_stride, sizeof(TS)) && rows(b.y, p.y_stride, sizeof(TS)) && rows(b.branch, p.branch_stride, sizeof(TB)) &&
                     rows(b.gate, p.gate_stride, sizeof(TB)) && rows(b.normed, p.normed_stride, sizeof(TB)) && aligned(p.post_weight, 32) &&
                     aligned(p.post_bias, 32) && aligned(p.pre_weight, 32) && aligned(p.pre_bias, 32);
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
