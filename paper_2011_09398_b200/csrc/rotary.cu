// Rotary positions of queries and keys, in one launch for both.
//
// The kernel moves memory: every element is read and written once, three operations each.  A thread has eight pairs of one token and
// takes them through several heads, so that their sines and cosines are worked out once for all of these; its sixteen channels are two
// vectors, of either half of the head or next to one another.  An angle is the product of position and step in 64 bits, whose upper half is
// a part of a turn: no reduction, and nothing is lost far out.
//
// Measured: 16384 tokens of 32 and 8 heads of 128 channels in bf16 (336 MB) 56 us, 6.0 TB/s; 1777 tokens of 20 and 5 heads of 80 in fp32, 32
// channels turned (28 MB), 6.5 us; one token 5 us, launch and call.
#include "kv_common.cuh"
#include "row_overlap.cuh"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

constexpr int kThreads = 256;
constexpr int kMostHeads = 8;   // of a thread

struct RotaryRows {
    const void *in;
    void *out;
    int64_t in_token, in_head, out_token, out_head;
};

struct RotaryParams {
    int64_t tokens, items;         // items: (token, eight pairs)
    int32_t dim, rotary_dim, heads, q_heads;
    int32_t turning, units;        // units of sixteen channels that turn; of a head in all
    int32_t per_thread;            // heads
    float amplitude;
    FastDiv by_units;
    const int32_t *positions;
    const uint64_t *steps;
    RotaryRows rows[2];            // q, k
};

// amplitude * cos and sin of a part of a turn, in units of 2^-32: to the nearest quarter turn in whole numbers, then Taylor's sums up to
// x^9 and x^10, below 2^-28 for the eighth of a turn that is left.
__device__ __forceinline__ void turn_of(uint32_t part, float amplitude, float &c, float &s)
{
    const uint32_t quarter = (part + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(part - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
    const float z = x * x;
    const float sine = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
    const float cosine = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    c = amplitude * (quarter & 1 ? sine : cosine);
    s = amplitude * (quarter & 1 ? cosine : sine);
    if ((quarter + 1) & 2) c = -c;
    if (quarter & 2) s = -s;
}

// kTogether heads' loads are on their way at once: four heads of 16 bits by three blocks an SM (two blocks: 61 us for 16384 tokens, two heads 58).
template <typename T, bool PAIRS, int kTogether>
__global__ void __launch_bounds__(kThreads, 3) rotary_kernel(const __grid_constant__ RotaryParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (item >= p.items) return;
    const int token = p.by_units((int)item), unit = (int)item - token * p.units;
    // the two vectors' channels; the second one may not be there
    int a, b;
    bool both = true;
    float cosine[8], sine[8];
    const bool turns = unit < p.turning;
    if (turns) {
        const int pairs = p.rotary_dim / 2, pair0 = 8 * unit;
        if (PAIRS) {
            a = 2 * pair0;
            b = a + 8;
        } else {
            a = pair0;
            b = a + pairs;
        }
        const int64_t position = __ldg(p.positions + token);
        uint64_t step[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) step[i] = __ldg(reinterpret_cast<const unsigned long long *>(p.steps) + pair0 + i);
#pragma unroll
        for (int i = 0; i < 8; ++i) turn_of((uint32_t)(((uint64_t)position * step[i] + 0x80000000u) >> 32), p.amplitude, cosine[i], sine[i]);
    } else {
        a = p.rotary_dim + 16 * (unit - p.turning);
        b = a + 8;
        both = b < p.dim;
    }
    const int first = blockIdx.y * p.per_thread, last = min(first + p.per_thread, p.heads);
    for (int h0 = first; h0 < last; h0 += kTogether) {
        Eight<T> va[kTogether], vb[kTogether];
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            const int h = min(h0 + i, last - 1);
            const bool key = h >= p.q_heads;
            const RotaryRows &r = p.rows[key];
            const T *const from = static_cast<const T *>(r.in) + token * r.in_token + (key ? h - p.q_heads : h) * r.in_head;
            va[i] = load_eight<T, true>(from + a, h0 + i < last ? 8 : 0);
            vb[i] = load_eight<T, true>(from + b, both && h0 + i < last ? 8 : 0);
        }
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            const int h = h0 + i;
            if (h >= last) break;
            const bool key = h >= p.q_heads;
            const RotaryRows &r = p.rows[key];
            T *const to = static_cast<T *>(r.out) + token * r.out_token + (key ? h - p.q_heads : h) * r.out_head;
            if (turns) {
                float x[8], y[8];
                va[i].expand(x);
                vb[i].expand(y);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    // the pair: (x[j], y[j]), or neighbours of x, then of y
                    float &u = PAIRS ? (j < 4 ? x[2 * j & 7] : y[2 * j & 7]) : x[j];
                    float &v = PAIRS ? (j < 4 ? x[(2 * j + 1) & 7] : y[(2 * j + 1) & 7]) : y[j];
                    const float s = u * sine[j];
                    u = fmaf(u, cosine[j], -(v * sine[j]));
                    v = fmaf(v, cosine[j], s);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    va[i].e[j] = from_float<T>(x[j]);
                    vb[i].e[j] = from_float<T>(y[j]);
                }
            }
            store_eight(to + a, va[i]);
            if (both) store_eight(to + b, vb[i]);
        }
    }
}

// Heads that are not cut into whole vectors: a warp to a token and some of its heads, a lane to every 32nd pair, element by element.  (31333 tokens
// of 5 heads of 192 channels in bf16, 106 of them turned: 54 us, with eight elements one by one to a thread 139.)
constexpr int kRowWarps = 8, kMostPairs = kKvMaxDim / 64, kMostRest = kKvMaxDim / 32;

template <typename T, bool PAIRS>
__global__ void __launch_bounds__(32 * kRowWarps) rotary_rows_kernel(const __grid_constant__ RotaryParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t token = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    if (token >= p.tokens) return;
    const int pairs = p.rotary_dim / 2;
    const int64_t position = __ldg(p.positions + token);
    float cosine[kMostPairs], sine[kMostPairs];
#pragma unroll
    for (int j = 0; j < kMostPairs; ++j) {
        const int i = lane + 32 * j;
        cosine[j] = sine[j] = 0.0f;
        if (i < pairs) turn_of((uint32_t)(((uint64_t)position * __ldg(reinterpret_cast<const unsigned long long *>(p.steps) + i) + 0x80000000u) >> 32), p.amplitude, cosine[j], sine[j]);
    }
    const int first = blockIdx.y * p.per_thread, last = min(first + p.per_thread, p.heads);
#pragma unroll 2
    for (int h = first; h < last; ++h) {
        const bool key = h >= p.q_heads;
        const RotaryRows &r = p.rows[key];
        const T *const from = static_cast<const T *>(r.in) + token * r.in_token + (key ? h - p.q_heads : h) * r.in_head;
        T *const to = static_cast<T *>(r.out) + token * r.out_token + (key ? h - p.q_heads : h) * r.out_head;
        T x[kMostPairs], y[kMostPairs], rest[kMostRest];
#pragma unroll
        for (int j = 0; j < kMostPairs; ++j) {
            const int i = lane + 32 * j;
            if (i < pairs) {
                x[j] = from[PAIRS ? 2 * i : i];
                y[j] = from[PAIRS ? 2 * i + 1 : i + pairs];
            }
        }
#pragma unroll
        for (int j = 0; j < kMostRest; ++j)
            if (p.rotary_dim + lane + 32 * j < p.dim) rest[j] = from[p.rotary_dim + lane + 32 * j];
#pragma unroll
        for (int j = 0; j < kMostPairs; ++j) {
            const int i = lane + 32 * j;
            if (i < pairs) {
                const float u = to_float(x[j]), v = to_float(y[j]), s = u * sine[j];
                to[PAIRS ? 2 * i : i] = from_float<T>(fmaf(u, cosine[j], -(v * sine[j])));
                to[PAIRS ? 2 * i + 1 : i + pairs] = from_float<T>(fmaf(v, cosine[j], s));
            }
        }
#pragma unroll
        for (int j = 0; j < kMostRest; ++j)
            if (p.rotary_dim + lane + 32 * j < p.dim) to[p.rotary_dim + lane + 32 * j] = rest[j];
    }
}

template <typename T>
lce_status launch(const RotaryParams &p, bool pairs, cudaStream_t s)
{
    // whole vectors: sixteen channels that turn at a time, rows on the vectors' boundaries
    bool vec = p.dim % 8 == 0 && p.rotary_dim % 16 == 0;
    for (const RotaryRows &r : p.rows) {
        if (!r.in) continue;
        vec = vec && aligned(r.in, 8 * sizeof(T)) && aligned(r.out, 8 * sizeof(T));
        for (const int64_t stride : {r.in_token, r.in_head, r.out_token, r.out_head}) vec = vec && stride % 8 == 0;
    }
    const unsigned parts = (unsigned)((p.heads + p.per_thread - 1) / p.per_thread);
    if (!vec)
        return launch_dependent(pairs ? rotary_rows_kernel<T, true> : rotary_rows_kernel<T, false>, dim3((unsigned)((p.tokens + kRowWarps - 1) / kRowWarps), parts), 32 * kRowWarps, 0, s, p);
    const auto go = [&](auto together) {
        constexpr int N = decltype(together)::value;
        return launch_dependent(pairs ? rotary_kernel<T, true, N> : rotary_kernel<T, false, N>, dim3((unsigned)((p.items + kThreads - 1) / kThreads), parts), kThreads, 0, s, p);
    };
    return p.per_thread == 1 ? go(std::integral_constant<int, 1>()) : go(std::integral_constant<int, sizeof(T) == 2 ? 4 : 2>());
}

bool stride_ok(int64_t s) { return s >= 0 && s < (1ll << 40); }

}  // namespace
}  // namespace lce

extern "C" lce_status lce_rotary_steps(int32_t rotary_dim, int32_t scaling, double base, double factor, double original_length, double low_turns,
                                       double high_turns, uint64_t *steps)
{
    using namespace lce;
    if (rotary_dim < 0 || rotary_dim % 2 != 0 || scaling < LCE_ROTARY_PLAIN || scaling > LCE_ROTARY_PARTS || !steps) return LCE_ERR_INVALID_ARG;
    if (rotary_dim > kKvMaxDim) return LCE_ERR_UNSUPPORTED;
    // frequencies stay at most one radian: bases and factors below 1 would be no scaling for longer contexts
    if (!(base >= 1.0) || !isfinite(base) || (scaling != LCE_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor)))) return LCE_ERR_INVALID_ARG;
    if (scaling == LCE_ROTARY_PARTS && (!(original_length > 0.0) || !isfinite(original_length) || !(low_turns >= 0.0) || !(high_turns > low_turns) || !isfinite(high_turns)))
        return LCE_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    if (scaling == LCE_ROTARY_BASE && rotary_dim > 2) base *= pow(factor, rotary_dim / (rotary_dim - 2.0));
    if (!isfinite(base)) return LCE_ERR_INVALID_ARG;
    for (int32_t i = 0; i < rotary_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rotary_dim);
        if (scaling == LCE_ROTARY_LINEAR) f /= factor;
        if (scaling == LCE_ROTARY_PARTS) {
            const double g = std::min(1.0, std::max(0.0, (original_length * f / two_pi - low_turns) / (high_turns - low_turns)));
            f *= g + (1.0 - g) / factor;
        }
        steps[i] = (uint64_t)rint(ldexp(f / two_pi, 64));
    }
    return LCE_OK;
}

extern "C" lce_status lce_rotary(const lce_rotary_desc *desc, const void *q, const void *k, const int32_t *positions, const uint64_t *steps, void *q_out,
                                 void *k_out, void *stream)
{
    using namespace lce;
    if (!desc) return LCE_ERR_INVALID_ARG;
    const lce_rotary_desc &d = *desc;
    if (d.head_dim <= 0 || d.rotary_dim < 0 || d.rotary_dim % 2 != 0 || d.rotary_dim > d.head_dim || d.q_heads <= 0 || d.k_heads < 0 || d.tokens < 0)
        return LCE_ERR_INVALID_ARG;
    if (d.layout < LCE_ROTARY_HALVES || d.layout > LCE_ROTARY_PAIRS || !type_known(d.type) || !isfinite(d.amplitude)) return LCE_ERR_INVALID_ARG;
    for (const int64_t s : {d.q_token_stride, d.q_head_stride, d.k_token_stride, d.k_head_stride, d.q_out_token_stride, d.q_out_head_stride, d.k_out_token_stride,
                            d.k_out_head_stride})
        if (!stride_ok(s)) return LCE_ERR_INVALID_ARG;
    RotaryParams p{};
    p.turning = (d.rotary_dim + 15) / 16;
    p.units = p.turning + (d.head_dim - d.rotary_dim + 15) / 16;
    if (d.head_dim > kKvMaxDim || d.q_heads > 32767 || d.k_heads > 32767 || d.tokens >= (1ll << 31) || d.tokens * p.units >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    if (d.tokens == 0) return LCE_OK;
    if (!q || !q_out || !positions || (d.rotary_dim > 0 && !steps) || (d.k_heads > 0 && (!k || !k_out))) return LCE_ERR_INVALID_ARG;
    const size_t size = type_size(d.type);
    if (!aligned(q, size) || !aligned(q_out, size) || !aligned(positions, 4) || !aligned(steps, 8)) return LCE_ERR_ALIGNMENT;
    if (d.k_heads > 0 && (!aligned(k, size) || !aligned(k_out, size))) return LCE_ERR_ALIGNMENT;
    // Threads read some heads and write them while others are at other heads: in place, but over no other row that is read or written.
    const auto row_set = [&](const void *data, int32_t heads, int64_t token_stride, int64_t head_stride) {
        return RowSet{data, d.tokens, heads, token_stride, head_stride, d.head_dim, (int64_t)size};
    };
    const RowSet in[2] = {row_set(q, d.q_heads, d.q_token_stride, d.q_head_stride), row_set(k, d.k_heads, d.k_token_stride, d.k_head_stride)};
    const RowSet out[2] = {row_set(q_out, d.q_heads, d.q_out_token_stride, d.q_out_head_stride), row_set(k_out, d.k_heads, d.k_out_token_stride, d.k_out_head_stride)};
    for (int i = 0; i < 2; ++i) {
        const bool in_place = in[i].data == out[i].data && (d.tokens == 1 || in[i].outer_stride == out[i].outer_stride) && (in[i].inner <= 1 || in[i].inner_stride == out[i].inner_stride);
        if (!rows_apart(out[i]) || (!in_place && rows_meet(in[i], out[i])) || rows_meet(in[1 - i], out[i])) return LCE_ERR_INVALID_ARG;
    }
    if (rows_meet(out[0], out[1])) return LCE_ERR_INVALID_ARG;
    p.tokens = d.tokens;
    p.items = d.tokens * p.units;
    p.dim = d.head_dim; p.rotary_dim = d.rotary_dim; p.q_heads = d.q_heads; p.heads = d.q_heads + d.k_heads;
    p.amplitude = d.amplitude;
    fast_div_constants((uint32_t)p.units, &p.by_units.mul, &p.by_units.sh);
    p.positions = positions; p.steps = steps;
    p.rows[0] = {q, q_out, d.q_token_stride, d.q_head_stride, d.q_out_token_stride, d.q_out_head_stride};
    if (d.k_heads > 0) p.rows[1] = {k, k_out, d.k_token_stride, d.k_head_stride, d.k_out_token_stride, d.k_out_head_stride};
    // as many heads to a thread as leave every SM its threads
    p.per_thread = kMostHeads;
    while (p.per_thread > 1 && p.items * p.heads < (int64_t)p.per_thread * 148 * 1024) p.per_thread /= 2;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool pairs = d.layout == LCE_ROTARY_PAIRS;
    switch (d.type) {
        case LCE_TYPE_FLOAT32: return launch<float>(p, pairs, s);
        case LCE_TYPE_FLOAT16: return launch<__half>(p, pairs, s);
        default: return launch<__nv_bfloat16>(p, pairs, s);
    }
}
