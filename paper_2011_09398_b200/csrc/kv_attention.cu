// Attention over the 4-bit key/value cache.
//
// For the rows of one sequence that share a key/value head (its new tokens x the group's query heads: the "columns" here) the
// keys and values are read once: S = K Q^T and O = V^T P, with the 4-bit operand on the 16-row side of m16n8k16 products and 8 or
// 16 columns on the other.  What bounds a decode step is reading the cache, 4.5 bits a channel, so the arithmetic between the
// 4-bit words and the matrix operands is kept to a minimum:
//
//   keys    a code n = c + 8 of four bits is, as it stands in a 16-bit half, the subnormal f16 number n 2^-24 (or 16 n 2^-24 in
//           bits 4 .. 7): one AND makes a pair of operands, five instructions eight codes.  The 16 goes into Q, the 8 into the
//           accumulators' initial value, -8 sum(q) over the block, and the block's scale multiplies the finished sums.
//   values  likewise; the 8 leaves by a second product, of a constant matrix and the same p, tile by tile (left to the end,
//           the sums over a long sequence would lose their last bits next to 8 sum(p)): the tensor cores have the time.  The
//           block's scale multiplies p, in fp32, before it is rounded to f16.
//
// Measured: 131072 tokens of 8 heads of 128 channels (151 MB) 43 us, 5.2 TB/s where the sequence is longer still; 777 tokens 7.2 us; 48
// sequences of 1 - 8192 tokens (236 MB) 84 us.  A warp spends 340 instructions on 16 tokens of 128 channels and 8 columns, of them 24
// matrix products; the issue slots are 55% busy, with the registers for four warps a scheduler.
//
// Scores and the running softmax are fp32.  Q is f16 times a power of two chosen for each row.  Odd channels, whose codes count 16 times as
// they stand, are held as a sixteenth: f16 rows are exact where a number is not below 2^-24 of its row's largest, bf16 rows where it is
// not below 2^-27, and what is lost of smaller ones is below 2^-35 of the largest.  p is rounded to f16 (relative error 2^-11 of each
// weight, which is what an fp16 result has, and averages out): matrix products of more bits would take twice as many.  fp32 rows take Q
// and p as two f16 numbers each (22 bits), and codes as f16 c = n - 8: 1024 + n by one AND-OR, less 1032 by one packed add.
#include "kv_attention.cuh"
#include "kv_mma.cuh"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStages = 4;                // tiles in flight of a warp
constexpr float kRise = 4.0f;             // a running maximum is raised when a score passes it by 2^4
constexpr float kHeadroom = 10.0f;        // weights are held times 2^10: 2^(10 + 4 + 1) is the most that meets f16

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
// The same of bf16 numbers, c = 0.
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float remote(const float *p, int rank)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote_place(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float4 remote4(const float *p, int rank)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote_place(p, rank)) : "memory");
    return v;
}

constexpr size_t ring_bytes(int blocks) { return (size_t)kWarps * kStages * kv_tile_words(blocks) * 4; }

// Blocks that a variant's registers let an SM hold.
__host__ __device__ constexpr int blocks_per_sm(int blocks, int nt, bool split)
{
    return blocks * nt <= (split ? 3 : 4) ? 4 : blocks * nt <= (split ? 4 : 6) ? 3 : 2;
}

// B blocks of 32 channels, NT tiles of 8 columns, SPLIT: fp32 rows.
template <int B, int NT, bool SPLIT>
struct Warp {
    float o[B][2][NT][4];        // sums of c p: channels 32 b + 4 (lane / 4) + 2 i + {0, 1}, columns 8 nt + 2 (lane % 4) + {0, 1}
    float base[NT][2], weight[NT][2];  // of the lane's columns: what is added to a score, shift - largest so far; sum of weights
    uint32_t high;               // words of scales above this want a higher reference
    float shift, limit;          // kHeadroom - log2 of the scales' reference; shift + kRise
    uint32_t qf[B][2][NT][2];    // B operands of the keys' products
    uint32_t ql[SPLIT ? B : 1][2][NT][2];
    uint32_t eights[(B + 3) / 4][NT][2];  // -8 sum(q) of block lane % 4 of each four, for column lane / 4, in three bf16 parts
    float factor[NT][2];         // scores = factor * sum over blocks
    int32_t lo[NT][2], hi[NT][2];
};

// T: float, or __half for the bits of any 16-bit row.
template <int B, int NT, bool SPLIT, typename T>
__device__ __forceinline__ void take_queries(const AttnParams &p, const Unit &u, const Queries<B, NT, T> &queries, Warp<B, NT, SPLIT> &w)
{
    const int lane = threadIdx.x & 31, quarter = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float v[B][8];
        uint32_t magnitude = 0;  // magnitudes compare like integers, infinity and NaN above all others
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (!SPLIT && p.type == LCE_TYPE_BFLOAT16) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[b][i] = __uint_as_float((uint32_t)reinterpret_cast<const unsigned short *>(queries.e[nt][b].e)[i] << 16);
            } else {
                queries.e[nt][b].expand(v[b]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) magnitude = max(magnitude, __float_as_uint(v[b][i]) & 0x7fffffffu);
        }
        magnitude = max(magnitude, __shfl_xor_sync(0xffffffffu, magnitude, 1));
        magnitude = max(magnitude, __shfl_xor_sync(0xffffffffu, magnitude, 2));
        const bool finite = magnitude < 0x7f800000u;
        const float top = __uint_as_float(magnitude);
        // times 2^k, so that the largest is in [2^14, 2^15)
        int e = 0;
        if (top > 0.0f && finite) e = ilogbf(top);
        const int k = 14 - e, k1 = k / 2, k2 = k - k1;
        const float s1 = __uint_as_float((uint32_t)(127 + k1) << 23), s2 = __uint_as_float((uint32_t)(127 + k2) << 23);
        float eights[(B + 3) / 4] = {};
#pragma unroll
        for (int b = 0; b < B; ++b) {
            float sum = 0.0f;
            constexpr float kOddFactor = SPLIT ? 1.0f : 0.0625f;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                // channels 2 m and 2 m + 4, then 2 m + 1 and 2 m + 5, whose codes count 16 times as they stand
                const float x0 = v[b][2 * m] * s1 * s2, x1 = v[b][2 * m + 4] * s1 * s2, y0 = v[b][2 * m + 1] * s1 * s2 * kOddFactor,
                            y1 = v[b][2 * m + 5] * s1 * s2 * kOddFactor;
                const uint32_t a = pack_half2(x0, x1), c = pack_half2(y0, y1);
                w.qf[b][m][nt][0] = a;
                w.qf[b][m][nt][1] = c;
                if (SPLIT) {
                    w.ql[SPLIT ? b : 0][m][nt][0] = pack_half2(x0 - half_low(a), x1 - half_high(a));
                    w.ql[SPLIT ? b : 0][m][nt][1] = pack_half2(y0 - half_low(c), y1 - half_high(c));
                } else {
                    sum += half_low(a) + half_high(a) + 16.0f * (half_low(c) + half_high(c));
                }
            }
            if (!SPLIT) {
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if ((b & 3) == quarter) eights[b / 4] = sum * (-8.0f * 0x1p-22f);
            }
        }
        if (!SPLIT) {
#pragma unroll
            for (int x = 0; x < (B + 3) / 4; ++x) {
                const __nv_bfloat16 a = __float2bfloat16_rn(eights[x]), c = __float2bfloat16_rn(eights[x] - __bfloat162float(a)),
                                    d = __float2bfloat16_rn(eights[x] - __bfloat162float(a) - __bfloat162float(c));
                w.eights[x][nt][0] = (uint32_t)__bfloat16_as_ushort(a) | (uint32_t)__bfloat16_as_ushort(c) << 16;
                w.eights[x][nt][1] = (uint32_t)__bfloat16_as_ushort(d);
            }
        }
        // what the sums of 2^-22 2^k code * q are multiplied with (2^22 2^-k scale; fp32 rows 2^-k scale; in steps that stay in range)
        const float f = finite ? p.scale : __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int from = (2 * quarter + j) * 4, kc = (SPLIT ? 0 : 22) - __shfl_sync(0xffffffffu, k, from), c1 = kc / 2, c2 = kc - c1;
            w.factor[nt][j] = __shfl_sync(0xffffffffu, f, from) * __uint_as_float((uint32_t)(127 + c1) << 23) * __uint_as_float((uint32_t)(127 + c2) << 23);
            column_range(p, u, u.column0 + 8 * nt + 2 * quarter + j, &w.lo[nt][j], &w.hi[nt][j]);
        }
    }
}

// Scores of tokens 8 r + lane / 4 of the tile for the lane's columns, the blocks of one plane.
template <int B, int NT, bool SPLIT, int FIRST, int W>
__device__ __forceinline__ void plane_scores(const uint32_t *tile, const Warp<B, NT, SPLIT> &w, const uint32_t (&sc)[2][B], float (&s)[NT][4])
{
    const int lane = threadIdx.x & 31;
    uint32_t k[2][W];
#pragma unroll
    for (int h = 0; h < 2; ++h) load_words<W>(tile + 64 * FIRST + (32 * h + lane) * W, k[h]);
#pragma unroll
    for (int i = 0; i < W; ++i) {
        constexpr uint32_t kEven = 0x003c003cu, kOdd = 0x03c003c0u, kBase = 0x64006400u;
        const int b = FIRST + i;
        const uint32_t u0 = k[0][i], u1 = k[1][i], v0 = swap_bytes(u0), v1 = swap_bytes(u1);
        const float s0 = __uint_as_float(sc[0][b] << 16), s1 = __uint_as_float(sc[1][b] << 16);
        uint32_t a[8] = {u0 & kEven, u1 & kEven, u0 & kOdd, u1 & kOdd, v0 & kEven, v1 & kEven, v0 & kOdd, v1 & kOdd};
        if (SPLIT) {
#pragma unroll
            for (int x = 0; x < 8; ++x) a[x] = x & 2 ? signed_odd(a[x] | kBase) : signed_even(a[x] | kBase);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float d[4];
            if (SPLIT) {
                mma(d, a[0], a[1], a[2], a[3], w.ql[SPLIT ? b : 0][0][nt][0], w.ql[SPLIT ? b : 0][0][nt][1], 0.0f, 0.0f, 0.0f, 0.0f);
                mma(d, a[4], a[5], a[6], a[7], w.ql[SPLIT ? b : 0][1][nt][0], w.ql[SPLIT ? b : 0][1][nt][1]);
                mma(d, a[0], a[1], a[2], a[3], w.qf[b][0][nt][0], w.qf[b][0][nt][1]);
            } else {
                mma(d, a[0], a[1], a[2], a[3], w.qf[b][0][nt][0], w.qf[b][0][nt][1], 0.0f, 0.0f, 0.0f, 0.0f);
            }
            mma(d, a[4], a[5], a[6], a[7], w.qf[b][1][nt][0], w.qf[b][1][nt][1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s[nt][j] = fmaf(s0, d[j], s[nt][j]);
                s[nt][2 + j] = fmaf(s1, d[2 + j], s[nt][2 + j]);
            }
        }
    }
}

// O += V^T P over the tile, the blocks of one plane.  e: weights; shown: whether the column sees the token (only where MASKED).
template <int B, int NT, bool SPLIT, int FIRST, int W, bool MASKED>
__device__ __forceinline__ void plane_values(const uint32_t *tile, Warp<B, NT, SPLIT> &w, const uint32_t (&sc)[2][B], const float (&e)[2][NT][2],
                                             const bool (&shown)[2][NT][2])
{
    const int lane = threadIdx.x & 31;
    uint32_t v[2][W];
#pragma unroll
    for (int h = 0; h < 2; ++h) load_words<W>(tile + 64 * B + 64 * FIRST + (32 * h + lane) * W, v[h]);
#pragma unroll
    for (int i = 0; i < W; ++i) {
        constexpr uint32_t kEven = 0x003c003cu, kOdd = 0x03c003c0u, kBase = 0x64006400u;
        constexpr uint32_t kEven8 = 0x80208020u, kOdd8 = 0x82008200u;  // of the even and of the odd codes, as they stand
        const int b = FIRST + i;
        uint32_t a[2][4];  // [half][channel]
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t x = v[h][i], y = swap_bytes(x);
            a[h][0] = SPLIT ? signed_even(and_or(x, kEven, kBase)) : x & kEven;
            a[h][1] = SPLIT ? signed_odd(and_or(x, kOdd, kBase)) : x & kOdd;
            a[h][2] = SPLIT ? signed_even(and_or(y, kEven, kBase)) : y & kEven;
            a[h][3] = SPLIT ? signed_odd(and_or(y, kOdd, kBase)) : y & kOdd;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            uint32_t ph[2], pl[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float s = __uint_as_float(sc[r][b] & 0xffff0000u);
                float x0 = e[r][nt][0] * s, x1 = e[r][nt][1] * s;
                if (MASKED) {  // whatever stands behind a sequence's last token
                    x0 = shown[r][nt][0] ? x0 : 0.0f;
                    x1 = shown[r][nt][1] ? x1 : 0.0f;
                }
                const uint32_t packed = pack_half2(x0, x1);
                ph[r] = transpose8x8(packed);
                if (SPLIT) pl[r] = transpose8x8(pack_half2(x0 - half_low(packed), x1 - half_high(packed)));
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (!SPLIT) {
                    mma(w.o[b][c][nt], kEven8, kOdd8, kEven8, kOdd8, ph[0], ph[1]);
                    mma(w.o[b][c][nt], a[0][2 * c], a[0][2 * c + 1], a[1][2 * c], a[1][2 * c + 1], ph[0], ph[1]);
                } else {
                    float d[4];  // the products cut their sums: a long one would drift by 2^-24 each
                    mma(d, a[0][2 * c], a[0][2 * c + 1], a[1][2 * c], a[1][2 * c + 1], pl[0], pl[1], 0.0f, 0.0f, 0.0f, 0.0f);
                    mma(d, a[0][2 * c], a[0][2 * c + 1], a[1][2 * c], a[1][2 * c + 1], ph[0], ph[1]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) w.o[b][c][nt][x] += d[x];
                }
            }
        }
    }
}

template <int B, int NT, bool SPLIT, bool MASKED>
__device__ __forceinline__ void tile_step(const uint32_t *tile, int32_t token0, int32_t least_exponent, Warp<B, NT, SPLIT> &w)
{
    constexpr int Q = B / 4 * 4;
    constexpr bool T = (B & 2) != 0, S = (B & 1) != 0;
    const int lane = threadIdx.x & 31;
    uint32_t sc[2][B];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const uint32_t *at = tile + 128 * B;
        const int token = 8 * r + (lane >> 2);
#pragma unroll
        for (int f = 0; f < Q; f += 4) {
            uint32_t x[4];
            load_words<4>(at + 16 * f + 4 * token, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[r][f + i] = x[i];
        }
        if (T) {
            uint32_t x[2];
            load_words<2>(at + 16 * Q + 2 * token, x);
            sc[r][T ? Q : 0] = x[0];
            sc[r][T ? Q + 1 : 0] = x[1];
        }
        if (S) sc[r][B - 1] = at[16 * (B - 1) + token];
    }
    float s[NT][4] = {};
    if (!SPLIT) {
        // what the 8 in every code adds, taken off: -8 sum(q) of each block times the key's scale, a product of its own
#pragma unroll
        for (int x = 0; x < (B + 3) / 4; ++x) {
            const int b = 4 * x + (lane & 3);
            uint32_t a[2] = {0, 0};
            if (4 * x + 4 <= B || b < B) {
#pragma unroll
                for (int r = 0; r < 2; ++r) a[r] = __byte_perm(tile[kv_scale_word(B, 8 * r + (lane >> 2), b)], 0, 0x1010);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16(s[nt], a[0], a[1], a[0], a[1], w.eights[x][nt][0], w.eights[x][nt][1]);
        }
    }
    if (Q > 0) plane_scores<B, NT, SPLIT, 0, 4>(tile, w, sc, s);
    if (Q > 4) plane_scores<B, NT, SPLIT, (Q > 4 ? 4 : 0), 4>(tile, w, sc, s);
    if (T) plane_scores<B, NT, SPLIT, (T ? Q : 0), 2>(tile, w, sc, s);
    if (S) plane_scores<B, NT, SPLIT, B - 1, 1>(tile, w, sc, s);
    bool shown[2][NT][2], some[2];
    uint32_t largest = 0;  // scale of a value of the lane's tokens, in the high half
    float highest = -INFINITY;
    float e[2][NT][2];     // log2 of the weights first
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        some[r] = !MASKED;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                e[r][nt][j] = fmaf(s[nt][2 * r + j], w.factor[nt][j], w.base[nt][j]);
                shown[r][nt][j] = true;
                if (MASKED) {
                    const int32_t token = token0 + 8 * r + (lane >> 2);
                    shown[r][nt][j] = token >= w.lo[nt][j] && token < w.hi[nt][j];
                    if (!shown[r][nt][j]) e[r][nt][j] = -INFINITY;
                    some[r] = some[r] || shown[r][nt][j];
                }
                highest = fmaxf(highest, e[r][nt][j]);
            }
#pragma unroll
        for (int b = 0; b < B; ++b) largest = max(largest, some[r] ? sc[r][b] : 0u);
    }
    if (__any_sync(0xffffffffu, largest > w.high || highest > w.limit)) {
        // rare behind the first tiles: the references move up and the sums with them
        const float old_shift = w.shift;
        largest = __reduce_max_sync(0xffffffffu, largest);
        if (largest >= 0x7f800000u) {  // again without those that are NaN: their blocks' results are, the others keep their reference
            largest = 0;
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int b = 0; b < B; ++b) largest = max(largest, some[r] && sc[r][b] < 0x7f800000u ? sc[r][b] : 0u);
            largest = __reduce_max_sync(0xffffffffu, largest);
        }
        if (largest > w.high) {
            const int x = max((int)(largest >> 23) - 126, least_exponent);  // scales < 2^x; the weights' sum stays in range
            w.shift = kHeadroom - (float)x;
            w.high = (uint32_t)(127 + x) << 23 | 0xffffu;
            w.limit = w.shift + kRise;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // scores again, the largest among them and so far
                float x[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) x[r] = shown[r][nt][j] ? s[nt][2 * r + j] * w.factor[nt][j] : -INFINITY;
                float m = fmaxf(x[0], x[1]);
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                const float base = w.shift - fmaxf(m, old_shift - w.base[nt][j]), f = exp2f(base - w.base[nt][j]);
                w.base[nt][j] = base;
                w.weight[nt][j] *= f;
#pragma unroll
                for (int r = 0; r < 2; ++r) e[r][nt][j] = x[r] + base;
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        w.o[b][i][nt][j] *= f;
                        w.o[b][i][nt][2 + j] *= f;
                    }
            }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int r = 0; r < 2; ++r) e[r][nt][j] = exp2_fast(e[r][nt][j]);
            w.weight[nt][j] += e[0][nt][j] + e[1][nt][j];
        }
    if (Q > 0) plane_values<B, NT, SPLIT, 0, 4, MASKED>(tile, w, sc, e, shown);
    if (Q > 4) plane_values<B, NT, SPLIT, (Q > 4 ? 4 : 0), 4, MASKED>(tile, w, sc, e, shown);
    if (T) plane_values<B, NT, SPLIT, (T ? Q : 0), 2, MASKED>(tile, w, sc, e, shown);
    if (S) plane_values<B, NT, SPLIT, B - 1, 1, MASKED>(tile, w, sc, e, shown);
}

template <int B, int NT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(B, NT, SPLIT)) kv_attention_kernel(const __grid_constant__ AttnParams p)
{
    constexpr int COLUMNS = 8 * NT, TILE = kv_tile_words(B), PIECES = TILE / 4;
    extern __shared__ __align__(128) uint32_t smem[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (p.join) release_join();
    Unit u;
    int first_unit;
    const int unit = blockIdx.x / p.cluster, rank = blockIdx.x - unit * p.cluster;
    if (!find_unit<COLUMNS, false>(p, unit, &u, &first_unit)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, head = p.solo ? blockIdx.y * kWarps + warp : blockIdx.y;
    if (head >= p.g.heads) return;  // whole warps, which then meet nobody
    // tokens that every column sees, and those that one sees at least: the ranges' ends grow with the rows
    int32_t any_lo, all_hi, all_lo, any_hi;
    column_range(p, u, u.column0, &any_lo, &all_hi);
    column_range(p, u, min(u.column0 + COLUMNS, u.rows * p.group) - 1, &all_lo, &any_hi);
    const int32_t tile0 = any_hi > 0 ? max(u.tile0, any_lo / kKvTile) : u.tile1, tile1 = min(u.tile1, (any_hi + kKvTile - 1) / kKvTile);

    // on their way while the pages are looked up
    Queries<B, NT, typename std::conditional<SPLIT, float, __half>::type> queries;
    if (p.q_vectors) queries.template load<true>(p, u, head);
    else queries.template load<false>(p, u, head);

    uint32_t *const ring = smem + warp * kStages * TILE;
    const int32_t *const table = p.page_table + (int64_t)u.seq * p.table_pages;
    const int tiles_per_page = p.g.page_size / kKvTile;
    // a cluster's warps take its tiles in turn
    const int first_warp = p.solo ? 0 : rank * kWarps + warp, step = p.solo ? 1 : kWarps * p.cluster;
    // the warp's next 32 tiles in the cache, one to a lane; negative: not in the pool
    int32_t places = -1;
    const int32_t mine = max((tile1 - tile0 - first_warp + step - 1) / step, 0);
    const char *const cache = reinterpret_cast<const char *>(p.cache) + lane * 16;
    auto fetch = [&](int i, uint32_t to) {  // issues the copies of the warp's i-th tile
        if ((i & 31) == 0) {
            const int32_t t = tile0 + first_warp + (i + lane) * step, in_table = t / tiles_per_page;
            const int32_t page = t < tile1 ? __ldg(table + in_table) : -1;
            places = page >= 0 && page < p.g.pages ? (page * p.g.heads + head) * tiles_per_page + (t - in_table * tiles_per_page) : -1;
        }
        const int32_t place = __shfl_sync(0xffffffffu, places, i & 31);
        if (place >= 0) {
            const char *const from = cache + (int64_t)place * (TILE * 4);
#pragma unroll
            for (int c = 0; c < (PIECES + 31) / 32; ++c)
                if (c * 32 + 32 <= PIECES || c * 32 + lane < PIECES) cp_async16(to + c * 512, from + c * 512);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        return place >= 0;
    };
    uint32_t good = 0;  // whether the warp's next tiles are there, the next one in bit 0
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) good |= fetch(i, ring_at + i * (TILE * 4)) ? 1u << i : 0u;
    Warp<B, NT, SPLIT> w;
    take_queries(p, u, queries, w);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            w.base[nt][j] = -kLowest;
            w.weight[nt][j] = 0.0f;
        }
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) w.o[b][i][nt][j] = 0.0f;
    w.high = 0xffffu;
    w.shift = 0.0f;
    w.limit = kRise;

    int32_t token0 = (tile0 + first_warp) * kKvTile;
    for (int i = 0, stage = 0; i < mine; ++i, token0 += step * kKvTile, good >>= 1, stage = stage + 1 == kStages ? 0 : stage + 1) {
        __syncwarp();  // everyone is done with the stage that comes next
        good |= fetch(i + kStages - 1, ring_at + (stage ? stage - 1 : kStages - 1) * (TILE * 4)) ? 1u << (kStages - 1) : 0u;
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        __syncwarp();
        if (!(good & 1)) continue;
        const uint32_t *const tile = ring + stage * TILE;
        if (token0 >= all_lo && token0 + kKvTile <= all_hi) tile_step<B, NT, SPLIT, false>(tile, token0, p.least_exponent, w);
        else tile_step<B, NT, SPLIT, true>(tile, token0, p.least_exponent, w);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (p.solo) {
        // nobody to join: 4 channels of a block to a lane and column
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float l = w.weight[nt][j];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                const int q = u.column0 + 8 * nt + 2 * (lane & 3) + j, row = q / p.group;
                if (row >= u.rows) continue;
                const int64_t to = (u.row0 + row) * p.out_token + ((int64_t)head * p.group + (q - row * p.group)) * p.out_head + 4 * (lane >> 2);
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const float v[4] = {w.o[b][0][nt][j], w.o[b][0][nt][2 + j], w.o[b][1][nt][j], w.o[b][1][nt][2 + j]};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        constexpr float kEven = SPLIT ? 1.0f : 0x1p22f, kOdd = SPLIT ? 1.0f : 0x1p18f;  // what the codes stood for
                        if (32 * b + 4 * (lane >> 2) + i < p.g.dim) store_element(p.out, p.type, to + 32 * b + i, l == 0.0f ? 0.0f : v[i] * (i & 1 ? kOdd : kEven) / l);
                    }
                }
            }
        return;
    }
    __syncthreads();

    // The warps' sums meet in shared memory: [warp][column][32 B], largest and weight of each behind them.
    constexpr int D = 32 * B;
    float *const sums = reinterpret_cast<float *>(smem), *const tops = sums + kWarps * COLUMNS * D, *const weights = tops + kWarps * COLUMNS;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int column = 8 * nt + 2 * (lane & 3) + j;
            float l = w.weight[nt][j];
            l += __shfl_xor_sync(0xffffffffu, l, 4);
            l += __shfl_xor_sync(0xffffffffu, l, 8);
            l += __shfl_xor_sync(0xffffffffu, l, 16);
            if (lane < 4) {
                tops[warp * COLUMNS + column] = -w.base[nt][j];
                weights[warp * COLUMNS + column] = l;
            }
            float *const to = sums + (warp * COLUMNS + column) * D + 4 * (lane >> 2);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                constexpr float kEven = SPLIT ? 1.0f : 0x1p22f, kOdd = SPLIT ? 1.0f : 0x1p18f;  // what the codes stood for
                *reinterpret_cast<float4 *>(to + 32 * b) = make_float4(kEven * w.o[b][0][nt][j], kOdd * w.o[b][0][nt][2 + j], kEven * w.o[b][1][nt][j],
                                                                       kOdd * w.o[b][1][nt][2 + j]);
            }
        }
    __syncthreads();
    // [warp][column]: by what a warp's sums and weight count; the largest and the weight of all
    float *const factors = weights + kWarps * COLUMNS, *const all_top = factors + kWarps * COLUMNS, *const all_weight = all_top + COLUMNS;
    if (threadIdx.x < COLUMNS) {
        const int column = threadIdx.x;
        float top = tops[column], weight = 0.0f;
#pragma unroll
        for (int i = 1; i < kWarps; ++i) top = fmaxf(top, tops[i * COLUMNS + column]);
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            const float f = exp2f(tops[i * COLUMNS + column] - top);
            factors[i * COLUMNS + column] = f;
            weight = fmaf(f, weights[i * COLUMNS + column], weight);
        }
        all_top[column] = top;
        all_weight[column] = weight;
    }
    __syncthreads();
    // four channels at a time
    auto put = [&](int column, int c, float4 sum, float top, float weight) {
        if (u.chunks > 1) {
            float *const to = p.parts + (((int64_t)unit * p.g.heads + head) * COLUMNS + column) * (D + 4);
            *reinterpret_cast<float4 *>(to + c) = sum;
            if (c == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(top, weight);
            return;
        }
        const int q = u.column0 + column, row = q / p.group;
        if (row >= u.rows) return;
        const float by = weight == 0.0f ? 0.0f : 1.0f / weight;
        const int64_t at = (u.row0 + row) * p.out_token + ((int64_t)head * p.group + (q - row * p.group)) * p.out_head + c;
        const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < p.g.dim) store_element(p.out, p.type, at + i, weight == 0.0f ? 0.0f : v[i] * by);
    };
    for (int at = threadIdx.x; at < COLUMNS * D / 4; at += kThreads) {
        const int column = at / (D / 4), c = at % (D / 4) * 4;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            const float f = factors[i * COLUMNS + column];
            const float4 v = *reinterpret_cast<const float4 *>(sums + (i * COLUMNS + column) * D + c);
            sum.x = fmaf(f, v.x, sum.x);
            sum.y = fmaf(f, v.y, sum.y);
            sum.z = fmaf(f, v.z, sum.z);
            sum.w = fmaf(f, v.w, sum.w);
        }
        if (p.cluster == 1) put(column, c, sum, all_top[column], all_weight[column]);
        else *reinterpret_cast<float4 *>(sums + column * D + c) = sum;  // in warp 0's place, which nobody else reads
    }
    if (p.cluster == 1) return;
    // The blocks of a cluster read each other's sums where they are; each finishes its share of the columns' channels.
    cluster_sync();
    for (int at = rank * kThreads + threadIdx.x; at < COLUMNS * D / 4; at += p.cluster * kThreads) {
        const int column = at / (D / 4), c = at % (D / 4) * 4;
        float top = -INFINITY, weight = 0.0f;
        for (int r = 0; r < p.cluster; ++r) top = fmaxf(top, remote(all_top + column, r));
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int r = 0; r < p.cluster; ++r) {
            const float f = exp2f(remote(all_top + column, r) - top);
            weight = fmaf(f, remote(all_weight + column, r), weight);
            const float4 v = remote4(sums + column * D + c, r);
            sum.x = fmaf(f, v.x, sum.x);
            sum.y = fmaf(f, v.y, sum.y);
            sum.z = fmaf(f, v.z, sum.z);
            sum.w = fmaf(f, v.w, sum.w);
        }
        put(column, c, sum, top, weight);
    }
    cluster_sync();  // nobody leaves while its sums are read
}

// Joins the pieces of a column, always in the same order: a warp to a column, or where there are many pieces a block, its warps' share of
// them first, then the warps.  It is there before the pieces are (release_join) and has found its own by then.
constexpr int kJoinWarps = 8, kFewPieces = 16;

template <int NT>
__global__ void __launch_bounds__(32 * kJoinWarps) kv_attention_join_kernel(const __grid_constant__ AttnParams p)
{
    constexpr int COLUMNS = 8 * NT;
    __shared__ float4 sums[kJoinWarps][2][32];
    __shared__ float tops[kJoinWarps], weights[kJoinWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Unit u;
    int first_unit;
    // the lengths are what the kernel in front read: nothing has written them since
    const bool found = find_unit<COLUMNS, true>(p, blockIdx.x, &u, &first_unit);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the one in front, too
    const int head = blockIdx.y, D = 32 * p.g.blocks;
    if (!found) return;
    const int64_t step = (int64_t)p.g.heads * COLUMNS * (D + 4);
    const int chunks = min(u.chunks, p.units - first_unit);
    const auto column_parts = [&](int column) { return p.parts + (((int64_t)first_unit * p.g.heads + head) * COLUMNS + column) * (D + 4); };
    const auto add = [](float4 &sum, float f, const float4 &v) {
        sum.x = fmaf(f, v.x, sum.x);
        sum.y = fmaf(f, v.y, sum.y);
        sum.z = fmaf(f, v.z, sum.z);
        sum.w = fmaf(f, v.w, sum.w);
    };
    if (chunks <= kFewPieces) {
        // a warp to a column
        for (int column = blockIdx.z * kJoinWarps + warp; column < COLUMNS; column += gridDim.z * kJoinWarps) {
            const int q = u.column0 + column, row = q / p.group;
            if (row >= u.rows) return;
            const float *const from = column_parts(column);
            float top = lane < chunks ? from[lane * step + D] : -INFINITY;
#pragma unroll
            for (int d = kFewPieces / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            top = __shfl_sync(0xffffffffu, top, 0);
            float weight = 0.0f;
            float4 sum[2] = {};
#pragma unroll 4
            for (int i = 0; i < chunks; ++i) {
                const float f = exp2f(from[i * step + D] - top);
                weight = fmaf(f, from[i * step + D + 1], weight);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (4 * (lane + 32 * h) < D) add(sum[h], f, *reinterpret_cast<const float4 *>(from + i * step + 4 * (lane + 32 * h)));
            }
            const int64_t at = (u.row0 + row) * p.out_token + ((int64_t)head * p.group + (q - row * p.group)) * p.out_head;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float v[4] = {sum[h].x, sum[h].y, sum[h].z, sum[h].w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (4 * (lane + 32 * h) + i < p.g.dim) store_element(p.out, p.type, at + 4 * (lane + 32 * h) + i, weight == 0.0f ? 0.0f : v[i] / weight);
            }
        }
        return;
    }
    for (int column = blockIdx.z; column < COLUMNS; column += gridDim.z) {
        const int q = u.column0 + column, row = q / p.group;
        if (row >= u.rows) return;
        const float *const from = column_parts(column);
        float top = -INFINITY;
        for (int i = warp * 32 + lane; i < chunks; i += 32 * kJoinWarps) top = fmaxf(top, from[i * step + D]);
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        if (lane == 0) tops[warp] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kJoinWarps; ++i) top = fmaxf(top, tops[i]);
        float weight = 0.0f;
        float4 sum[2] = {};
#pragma unroll 4
        for (int i = warp; i < chunks; i += kJoinWarps) {
            const float f = exp2f(from[i * step + D] - top);
            weight = fmaf(f, from[i * step + D + 1], weight);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (4 * (lane + 32 * h) < D) add(sum[h], f, *reinterpret_cast<const float4 *>(from + i * step + 4 * (lane + 32 * h)));
        }
        sums[warp][0][lane] = sum[0];
        sums[warp][1][lane] = sum[1];
        if (lane == 0) weights[warp] = weight;
        __syncthreads();
        for (int c = threadIdx.x; c < p.g.dim; c += 32 * kJoinWarps) {
            float s = 0.0f, l = 0.0f;
#pragma unroll
            for (int i = 0; i < kJoinWarps; ++i) {
                s += reinterpret_cast<const float *>(sums[i])[c];
                l += weights[i];
            }
            store_element(p.out, p.type, (u.row0 + row) * p.out_token + ((int64_t)head * p.group + (q - row * p.group)) * p.out_head + c,
                          l == 0.0f ? 0.0f : s / l);
        }
        __syncthreads();
    }
}

constexpr size_t merge_bytes(int blocks, int nt) { return ((size_t)kWarps * 8 * nt * (32 * blocks + 3) + 2 * 8 * nt) * 4; }

template <int B, int NT, bool SPLIT>
lce_status launch(const AttnParams &p, cudaStream_t s)
{
    constexpr size_t smem = ring_bytes(B) > merge_bytes(B, NT) ? ring_bytes(B) : merge_bytes(B, NT);
    static SmemOptIn opt_in;
    if (!opt_in.ensure(kv_attention_kernel<B, NT, SPLIT>, smem)) return LCE_ERR_CUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.units * p.cluster), (unsigned)(p.solo ? (p.g.heads + kWarps - 1) / kWarps : p.g.heads), 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kv_attention_kernel<B, NT, SPLIT>, p) != cudaSuccess) {
        cudaGetLastError();
        return LCE_ERR_CUDA;
    }
    if (!p.join) return LCE_OK;
    // At most `target` column tiles are in pieces; columns that there can be in one; about a block for each place that the GPU has.
    const int64_t split = std::min<int64_t>(p.column_tiles, p.target), columns = std::min<int64_t>(p.tokens * p.group, p.one_row && p.group < 8 * NT ? p.group : 8 * NT);
    const int64_t side = std::max<int64_t>(1, std::min<int64_t>(columns, 148 * 8 / (split * p.g.heads)));
    return launch_dependent(kv_attention_join_kernel<NT>, dim3((unsigned)split, (unsigned)p.g.heads, (unsigned)side), 32 * kJoinWarps, 0, s, p);
}

// 16 columns where their sums and operands fit a thread's registers
constexpr int kWideBlocks = 4;

template <int NT, bool SPLIT>
lce_status launch_blocks(const AttnParams &p, cudaStream_t s)
{
    constexpr int N = 1;
    switch (p.g.blocks) {
        case 1: return launch<1, NT, SPLIT>(p, s);
        case 2: return launch<2, NT, SPLIT>(p, s);
        case 3: return launch<3, NT, SPLIT>(p, s);
        case 4: return launch<4, NT, SPLIT>(p, s);
        case 5: return launch<5, N, SPLIT>(p, s);
        case 6: return launch<6, N, SPLIT>(p, s);
        case 7: return launch<7, N, SPLIT>(p, s);
        default: return launch<8, N, SPLIT>(p, s);
    }
}

constexpr int kPromptLeastTiles = 6;  // tiles of 128 tokens that a piece is worth there
// Pieces that several sequences are cut into, in quarters of the blocks that the GPU holds: 48 sequences of 1 - 8192 tokens take 91.5, 90.6,
// 84.8 and 87.2 us with 3, 4, 6 and 8, 64 of 4096 89.8, 92.3, 92.9 and 101.1.
constexpr int kWaves = 6;
constexpr int kSoloTiles = 64;  // the longest that a warp takes alone
constexpr int kLeastTiles = 16;  // tiles of a warp that a piece is worth

// one_row: without q_starts
lce_status make_params(const lce_kv_attention_desc *d, bool one_row, AttnParams *p, int *nt)
{
    if (!d) return LCE_ERR_INVALID_ARG;
    const lce_status st = make_kv_geom(&d->cache, &p->g);
    if (st != LCE_OK) return st;
    if (d->batch <= 0 || d->heads <= 0 || d->table_pages <= 0 || d->tokens < 0 || d->window < 0 || !type_known(d->type)) return LCE_ERR_INVALID_ARG;
    if (d->causal != 0 && d->causal != 1) return LCE_ERR_INVALID_ARG;
    if (d->heads % d->cache.kv_heads != 0 || !isfinite(d->scale)) return LCE_ERR_INVALID_ARG;
    for (const int64_t s : {d->q_token_stride, d->q_head_stride, d->out_token_stride, d->out_head_stride})
        if (s < 0 || s >= (1ll << 40)) return LCE_ERR_INVALID_ARG;
    p->batch = d->batch; p->group = d->heads / d->cache.kv_heads; p->table_pages = d->table_pages;
    p->one_row = one_row;
    if (d->tokens >= (1ll << 31) || d->tokens * d->heads >= (1ll << 31) || (int64_t)d->table_pages * d->cache.page_size >= (1ll << 31) || d->batch >= (1 << 20)) return LCE_ERR_UNSUPPORTED;
    p->table_tokens = d->table_pages * d->cache.page_size;
    // A weight is at most 2^(kHeadroom + kRise - x): with x no less than this, the sum of a whole table's stays below 2^127.
    int bits = 0;
    while ((1ll << bits) < p->table_tokens) ++bits;
    p->least_exponent = std::max(-100, bits + (int)(kHeadroom + kRise) - 127);
    p->causal = d->causal; p->window = d->window; p->type = d->type;
    p->tokens = d->tokens;
    p->q_token = d->q_token_stride; p->q_head = d->q_head_stride; p->out_token = d->out_token_stride; p->out_head = d->out_head_stride;
    p->scale = d->scale * 1.44269504088896341f;
    *nt = p->g.blocks <= kWideBlocks && (d->tokens * p->group + d->batch - 1) / d->batch > 8 ? 2 : 1;
    // Many rows go to the kernel for prompts where it is estimated to be ahead (us for 128 channels, bf16; the two take what they were
    // measured to take: 16 columns of a head of one kernel 8.6e-5 a token, 256 of the other 1.4e-4, and 12 more to begin and end).
    // By the longest the sequences can be: their lengths are not known here.  One sequence of 512 / 4096 / 32768 tokens, 8 key heads of
    // 4: 16 rows 12.5 / 26.9 / 105 us here, 22.8 / 34.0 / 80.8 there, 64 rows 15.2 / 60.2 / 312 and 26.9 / 39.9 / 83.8; 16 sequences
    // of 512 / 4096, 8 rows each 17.3 / 107 and 25.5 / 99.0, 16 rows 31.8 / 189 and 25.9 / 102.
    const int64_t each = (p->tokens * p->group + p->batch - 1) / p->batch;  // columns of a sequence, on average
    const auto of_columns = [&](int64_t columns) { return (double)((each + columns - 1) / columns * p->batch * p->g.heads); };
    p->prompt = p->g.blocks <= 4 && d->type != LCE_TYPE_FLOAT32 && (of_columns(16) * 8.6e-5 - of_columns(kPromptColumns) * 1.4e-4) * p->table_tokens > 12.0;
    if (p->prompt) {
        // a block to an SM; sequences are cut into pieces where that leaves SMs without one (joining costs a few us)
        const int64_t tiles = p->tokens * p->group / kPromptColumns + p->batch, likely = p->batch * ((each + kPromptColumns - 1) / kPromptColumns);
        p->cluster = 1;
        p->least_tiles = 8 * kPromptLeastTiles;
        p->join = likely * p->g.heads * 5 < 148 * 4 && p->table_tokens > 128 * kPromptLeastTiles;
        const int64_t target = p->join ? std::max<int64_t>(148 / p->g.heads - likely, 1) : 0;
        p->target = (int32_t)std::max<int64_t>(target, 1);
        p->column_tiles = (int32_t)tiles;
        p->units = (int32_t)(tiles + target);
        return LCE_OK;
    }
    const int columns = 8 * *nt;
    const int64_t tiles = one_row ? (int64_t)p->batch * ((p->group + columns - 1) / columns) : p->tokens * p->group / columns + p->batch;
    // A cluster of up to eight blocks shares a unit, as many as the GPU has room for and as there are tiles for their warps.
    const int64_t blocks = 148 * blocks_per_sm(p->g.blocks, *nt, p->type == LCE_TYPE_FLOAT32);
    int64_t most = (p->table_tokens + kKvTile - 1) / kKvTile;  // tiles that a sequence can have in view
    if (p->window > 0 && one_row && p->window / kKvTile + 2 < most) most = p->window / kKvTile + 2;
    p->cluster = 1;
    const int64_t likely = p->batch * ((each + columns - 1) / columns);  // column tiles, were all sequences alike
    while (p->cluster < 8 && most <= kWarps * 8 * kLeastTiles && likely * p->g.heads * p->cluster * 2 <= blocks && p->cluster * kWarps < most) p->cluster *= 2;
    // Sequences longer than that pays for are cut further.
    p->least_tiles = kWarps * p->cluster * kLeastTiles;
    p->join = most > p->least_tiles;
    // Many short sequences: a warp to each, without the joining (256 of 512 tokens, 8 key heads: 71.7 us by blocks).
    p->solo = !p->join && p->cluster == 1 && most <= kSoloTiles && likely * p->g.heads >= 3 * blocks;
    const int waves = p->batch > 1 ? kWaves : 4;  // pieces of one sequence are all alike
    const int64_t target = p->join ? (blocks * waves / 4 / p->cluster + p->g.heads - 1) / p->g.heads : 0;
    p->target = (int32_t)(target > 0 ? target : 1);
    if ((tiles + target) * p->cluster >= (1ll << 31) || (int64_t)p->g.slots / kKvTile * p->g.heads >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    p->units = (int32_t)(tiles + target);
    p->column_tiles = (int32_t)tiles;
    return LCE_OK;
}

size_t workspace_bytes(const AttnParams &p, int nt)
{
    if (!p.join) return 16;
    if (p.prompt) return (size_t)p.units * p.g.heads * kPromptColumns * (32 * p.g.blocks + 4) * 4;
    return (size_t)p.units * p.g.heads * 8 * nt * (32 * p.g.blocks + 4) * 4;
}

}  // namespace
}  // namespace lce

extern "C" size_t lce_kv_attention_workspace_bytes(const lce_kv_attention_desc *desc)
{
    using namespace lce;
    AttnParams p{};
    int nt;
    // the room that the call wants with and without q_starts
    size_t bytes = 0;
    for (const bool one_row : {false, true}) {
        if (one_row && desc && desc->tokens != desc->batch) continue;
        if (make_params(desc, one_row, &p, &nt) != LCE_OK) return 0;
        const size_t b = workspace_bytes(p, nt);
        if (b > bytes) bytes = b;
    }
    return bytes;
}

extern "C" lce_status lce_kv_attention(const lce_kv_attention_desc *desc, const void *q, const void *cache, const int32_t *page_table,
                                       const int32_t *lengths, const int32_t *q_starts, void *out, void *workspace, size_t workspace_size, void *stream)
{
    using namespace lce;
    AttnParams p{};
    int nt;
    const lce_status st = make_params(desc, !q_starts, &p, &nt);
    if (st != LCE_OK) return st;
    if (!q_starts && desc->tokens != desc->batch) return LCE_ERR_INVALID_ARG;
    if (desc->tokens == 0) return LCE_OK;
    if (!q || !cache || !page_table || !lengths || !out || !workspace) return LCE_ERR_INVALID_ARG;
    const size_t element = type_size(desc->type);
    if (!aligned(q, element) || !aligned(out, element) || !aligned(cache, 16) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(q_starts, 4) ||
        !aligned(workspace, 16))
        return LCE_ERR_ALIGNMENT;
    if (workspace_size < workspace_bytes(p, nt)) return LCE_ERR_WORKSPACE;
    p.q_vectors = p.g.dim % 8 == 0 && aligned(q, 8 * element) && p.q_token % 8 == 0 && p.q_head % 8 == 0;
    p.out_vectors = p.g.dim % 8 == 0 && aligned(out, 8 * element) && p.out_token % 8 == 0 && p.out_head % 8 == 0;
    p.q = q; p.cache = static_cast<const uint32_t *>(cache); p.page_table = page_table; p.lengths = lengths; p.q_starts = q_starts;
    p.out = out; p.parts = static_cast<float *>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p.prompt) return launch_kv_prompt(p, s);
    if (desc->type == LCE_TYPE_FLOAT32) return nt == 2 ? launch_blocks<2, true>(p, s) : launch_blocks<1, true>(p, s);
    return nt == 2 ? launch_blocks<2, false>(p, s) : launch_blocks<1, false>(p, s);
}
