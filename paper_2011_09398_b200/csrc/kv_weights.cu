// How much attention every token of the 4-bit cache gets: sums of softmax weights over a sequence's newest rows.
//
// For the rows of one sequence that share a key/value head (its new tokens x the group's query heads: the "columns" here) the softmax needs
// the largest score and the sum of a whole column before the first weight is known.  So there are two kernels over pieces of the
// sequences: the first makes the scores, S = K Q^T with the 4-bit keys on the 16-row side of m16n8k16 products and 8 or 16 columns on the other,
// and each piece's largest and sum of every column; the second joins the pieces' (always in the same order) and adds a token's weights up
// over the columns.  Where there is room for them the second kernel reads the scores that the first one left, 4 bytes each, next to which the
// keys were 80 bytes for 128 channels; otherwise it makes them again.
//
// Keys are codes times a block's scale.  The codes c = n - 8 are exact f16 operands (1024 + n by one AND-OR, less 1032 by a packed
// multiply-add), the scale multiplies a block's finished sums in fp32; 16-bit rows of q are one f16 number times a power of two of the row,
// fp32 rows two of them.
//
// Measured (both kernels): 131072 tokens of 8 heads of 128 channels and 64 columns in all 39 us (84 MB of keys: 13 at the copy rate), 48 sequences
// of 1 - 8192 tokens 72 us, 777 tokens 7.5 us.  A warp of the first kernel spends 255 instructions on a tile of 16 tokens and 8 columns, of them 8 matrix
// products and 69 between the 4-bit words and their operands, with the issue slots 64 % busy at four warps a scheduler (127 registers).
#include "kv_mma.cuh"
#include "kv_weights.cuh"
#include "row_overlap.cuh"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

__host__ __device__ constexpr int key_words(int blocks) { return 80 * blocks; }  // of a tile: its keys and scales

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStages = 4;                  // tiles in flight of a warp
constexpr int kBlocksPerSm = 4;
// that a variant's registers let it hold
__host__ __device__ constexpr int blocks_per_sm(int blocks, int nt, bool split) { return blocks * nt * (split ? 2 : 1) < 8 ? kBlocksPerSm : 3; }
constexpr float kNothing = -3e38f;          // stands for the largest score where there is none
constexpr float kRise = 16.0f;              // the score that powers of two are relative to is raised when one passes it by this much
constexpr int64_t kMostScores = 256 << 20;  // bytes of workspace that scores may take
constexpr double kMostUnits = 1 << 21;      // (256 tokens, key head) that their list has room for
constexpr int64_t kMostStats = 64 << 20;

// B blocks of 32 channels, NT tiles of 8 columns, SPLIT: fp32 rows.
template <int B, int NT, bool SPLIT>
struct Columns {
    uint32_t qf[B][2][NT][2], ql[SPLIT ? B : 1][2][NT][2];  // B operands of the products
    float factor[NT][2];                                    // scores, as powers of two, are this times the sums over blocks
    int32_t lo[NT][2], hi[NT][2];                           // tokens that the lane's columns 8 nt + 2 (lane % 4) + {0, 1} see

    template <typename T>
    __device__ __forceinline__ void take(const WeightsParams &p, const Unit &u, const Queries<B, NT, T> &queries)
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
            // times 2^k, so that the largest is in [2^14, 2^15)
            const int k = 14 - (finite && magnitude > 0 ? ilogbf(__uint_as_float(magnitude)) : 0), k1 = k / 2, k2 = k - k1;
            const float s1 = __uint_as_float((uint32_t)(127 + k1) << 23), s2 = __uint_as_float((uint32_t)(127 + k2) << 23);
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int odd = 0; odd < 2; ++odd) {
                        // channels 2 m and 2 m + 4, then 2 m + 1 and 2 m + 5, in the order in which a word's codes come apart
                        const float x = v[b][2 * m + odd] * s1 * s2, y = v[b][2 * m + odd + 4] * s1 * s2;
                        const uint32_t a = pack_half2(x, y);
                        qf[b][m][nt][odd] = a;
                        if (SPLIT) ql[SPLIT ? b : 0][m][nt][odd] = pack_half2(x - half_low(a), y - half_high(a));
                    }
            const float f = finite ? p.scale : __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int from = (2 * quarter + j) * 4, kc = -__shfl_sync(0xffffffffu, k, from), c1 = kc / 2, c2 = kc - c1;
                factor[nt][j] = __shfl_sync(0xffffffffu, f, from) * __uint_as_float((uint32_t)(127 + c1) << 23) * __uint_as_float((uint32_t)(127 + c2) << 23);
                column_range(p, u, u.column0 + 8 * nt + 2 * quarter + j, &lo[nt][j], &hi[nt][j]);
            }
        }
    }
    __device__ __forceinline__ void load(const WeightsParams &p, const Unit &u, int head)
    {
        Queries<B, NT, typename std::conditional<SPLIT, float, __half>::type> queries;  // __half: the bits of any 16-bit row
        if (p.q_vectors) queries.template load<true>(p, u, head);
        else queries.template load<false>(p, u, head);
        take(p, u, queries);
    }

    // Sums over one plane's blocks for tokens 8 r + lane / 4 of the tile and the lane's columns: s[nt][2 r + j].
    template <int FIRST, int W>
    __device__ __forceinline__ void plane(const uint32_t *tile, float (&s)[NT][4]) const
    {
        constexpr uint32_t kEven = 0x003c003cu, kOdd = 0x03c003c0u, kBase = 0x64006400u;
        const int lane = threadIdx.x & 31;
        uint32_t k[2][W], sc[2][W];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            load_words<W>(tile + 64 * FIRST + (32 * h + lane) * W, k[h]);
            load_words<W>(tile + 64 * B + 16 * FIRST + (8 * h + (lane >> 2)) * W, sc[h]);
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int b = FIRST + i;
            const uint32_t u0 = k[0][i], u1 = k[1][i], v0 = swap_bytes(u0), v1 = swap_bytes(u1);
            const uint32_t a[8] = {signed_even(and_or(u0, kEven, kBase)), signed_even(and_or(u1, kEven, kBase)), signed_odd(and_or(u0, kOdd, kBase)),
                                   signed_odd(and_or(u1, kOdd, kBase)),   signed_even(and_or(v0, kEven, kBase)), signed_even(and_or(v1, kEven, kBase)),
                                   signed_odd(and_or(v0, kOdd, kBase)),   signed_odd(and_or(v1, kOdd, kBase))};
            const float s0 = __uint_as_float(sc[0][i] << 16), s1 = __uint_as_float(sc[1][i] << 16);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float d[4];
                if (SPLIT) {
                    mma(d, a[0], a[1], a[2], a[3], ql[SPLIT ? b : 0][0][nt][0], ql[SPLIT ? b : 0][0][nt][1], 0.0f, 0.0f, 0.0f, 0.0f);
                    mma(d, a[4], a[5], a[6], a[7], ql[SPLIT ? b : 0][1][nt][0], ql[SPLIT ? b : 0][1][nt][1]);
                    mma(d, a[0], a[1], a[2], a[3], qf[b][0][nt][0], qf[b][0][nt][1]);
                } else {
                    mma(d, a[0], a[1], a[2], a[3], qf[b][0][nt][0], qf[b][0][nt][1], 0.0f, 0.0f, 0.0f, 0.0f);
                }
                mma(d, a[4], a[5], a[6], a[7], qf[b][1][nt][0], qf[b][1][nt][1]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s[nt][j] = fmaf(s0, d[j], s[nt][j]);
                    s[nt][2 + j] = fmaf(s1, d[2 + j], s[nt][2 + j]);
                }
            }
        }
    }
    // Scores of a tile; minus infinity where a column does not see the token (only looked at where MASKED).
    template <bool MASKED>
    __device__ __forceinline__ void scores(const uint32_t *tile, int32_t token0, float (&s)[NT][4]) const
    {
        constexpr int Q = B / 4 * 4;
        constexpr bool T = (B & 2) != 0, S = (B & 1) != 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = 0.0f;
        if (Q > 0) plane<0, 4>(tile, s);
        if (Q > 4) plane<(Q > 4 ? 4 : 0), 4>(tile, s);
        if (T) plane<(T ? Q : 0), 2>(tile, s);
        if (S) plane<B - 1, 1>(tile, s);
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[nt][i] *= factor[nt][i & 1];
                if (MASKED) {
                    const int32_t token = token0 + 8 * (i >> 1) + (lane >> 2);
                    if (token < lo[nt][i & 1] || token >= hi[nt][i & 1]) s[nt][i] = -INFINITY;
                }
            }
    }
};

// The warp's tiles of a view, brought to shared memory one after the other: body(tile, its words or null where its page is outside the pool).
template <int B, typename Body>
__device__ __forceinline__ void each_tile(const WeightsParams &p, const Piece &piece, const View &v, int head, uint32_t *ring, Body body)
{
    constexpr int WORDS = key_words(B), PIECES = WORDS / 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t *const table = p.page_table + (int64_t)piece.u.seq * p.table_pages;
    const int tiles_per_page = p.g.page_size / kKvTile;
    const int32_t mine = max((v.tile1 - v.tile0 - warp + kWarps - 1) / kWarps, 0);
    const char *const cache = reinterpret_cast<const char *>(p.cache);
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    int32_t places = -1;  // the warp's next 32 tiles in the cache, one to a lane; negative: not in the pool
    const auto fetch = [&](int i, int stage) {
        if ((i & 31) == 0) {
            const int32_t t = v.tile0 + warp + (i + lane) * kWarps, in_table = t / tiles_per_page;
            const int32_t page = t < v.tile1 ? __ldg(table + in_table) : -1;
            places = page >= 0 && page < p.g.pages ? (page * p.g.heads + head) * tiles_per_page + (t - in_table * tiles_per_page) : -1;
        }
        const int32_t place = __shfl_sync(0xffffffffu, places, i & 31);
        if (place >= 0) {
            const char *const from = cache + (int64_t)place * (kv_tile_words(B) * 4);
#pragma unroll
            for (int c = 0; c < (PIECES + 31) / 32; ++c) {
                const int at = c * 32 + lane;
                if (c * 32 + 32 <= PIECES || at < PIECES) cp_async16(ring_at + (stage * WORDS + 4 * at) * 4, from + 16 * (at < 16 * B ? at : at + 16 * B));
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        return place >= 0;
    };
    uint32_t good = 0;  // whether the warp's next tiles are there, the next one in bit 0
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) good |= fetch(i, i) ? 1u << i : 0u;
    for (int i = 0, stage = 0; i < mine; ++i, good >>= 1, stage = stage + 1 == kStages ? 0 : stage + 1) {
        __syncwarp();  // everyone is done with the stage that comes next
        good |= fetch(i + kStages - 1, stage ? stage - 1 : kStages - 1) ? 1u << (kStages - 1) : 0u;
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        __syncwarp();
        body(v.tile0 + warp + i * kWarps, good & 1 ? ring + stage * WORDS : nullptr);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
}

// Scores of a tile's first token.
__device__ __forceinline__ float *scores_at(const WeightsParams &p, const Piece &piece, int head, int32_t tile)
{
    return p.scores + head * p.scores_head + piece.scores_before + (int64_t)tile * kKvTile * scores_stride(piece.columns);
}

// Sums of powers of two relative to `top` and to `other_top`, joined.
__device__ __forceinline__ void join_sums(float &top, float &sum, float other_top, float other_sum)
{
    const float high = fmaxf(top, other_top);
    sum = sum * exp2f(top - high) + other_sum * exp2f(other_top - high);
    top = high;
}

template <int B, int NT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(B, NT, SPLIT)) kv_weights_scores_kernel(const __grid_constant__ WeightsParams p)
{
    constexpr int COLUMNS = 8 * NT;
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ float tops[kWarps][COLUMNS], sums[kWarps][COLUMNS];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    release_join();
    Piece piece;
    if (!find_piece(p, blockIdx.x, &piece)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, head = blockIdx.y;
    const int64_t stride = scores_stride(piece.columns);
    for (piece.u.column0 = blockIdx.z * COLUMNS; piece.u.column0 < piece.columns; piece.u.column0 += gridDim.z * COLUMNS) {
        const View v = view(p, piece, COLUMNS);
        Columns<B, NT, SPLIT> c;
        c.load(p, piece.u, head);
        float top[NT][2], sum[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[nt][j] = kNothing;
                sum[nt][j] = 0.0f;
            }
        float *to = p.scores ? scores_at(p, piece, head, v.tile0 + warp) + (lane >> 2) * stride + piece.u.column0 + 2 * (lane & 3) : nullptr;
        const auto tile_step = [&](int32_t tile, const uint32_t *words, auto masked) {
            float s[NT][4];
            c.template scores<decltype(masked)::value>(words, tile * kKvTile, s);
            if (p.scores) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    if (piece.u.column0 + 8 * nt + 2 * (lane & 3) < stride) {
                        *reinterpret_cast<float2 *>(to + 8 * nt) = make_float2(s[nt][0], s[nt][1]);
                        *reinterpret_cast<float2 *>(to + 8 * nt + 8 * stride) = make_float2(s[nt][2], s[nt][3]);
                    }
            }
            float e[NT][4], highest = -INFINITY;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[nt][i] = s[nt][i] - top[nt][i & 1];
                    highest = fmaxf(highest, e[nt][i]);
                }
            if (__any_sync(0xffffffffu, highest > kRise)) {  // rare behind the first tiles: the lane's references move up
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float high = fmaxf(top[nt][j], fmaxf(s[nt][j], s[nt][2 + j]));
                        sum[nt][j] *= exp2f(top[nt][j] - high);
                        top[nt][j] = high;
                        e[nt][j] = s[nt][j] - high;
                        e[nt][2 + j] = s[nt][2 + j] - high;
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[nt][j] += exp2_fast(e[nt][j]) + exp2_fast(e[nt][2 + j]);
        };
        each_tile<B>(p, piece, v, head, smem + warp * kStages * key_words(B), [&](int32_t tile, const uint32_t *words) {
            if (!words) {
                if (p.scores)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        if (piece.u.column0 + 8 * nt + 2 * (lane & 3) < stride)
                            *reinterpret_cast<float2 *>(to + 8 * nt) = *reinterpret_cast<float2 *>(to + 8 * nt + 8 * stride) = make_float2(-INFINITY, -INFINITY);
            } else if (tile * kKvTile >= v.all_lo && tile * kKvTile + kKvTile <= v.all_hi) {
                tile_step(tile, words, std::false_type());
            } else {
                tile_step(tile, words, std::true_type());
            }
            to += (int64_t)kWarps * kKvTile * stride;
        });
        // eight lanes have a column's tokens, then the warps
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    const float t = __shfl_xor_sync(0xffffffffu, top[nt][j], d), s = __shfl_xor_sync(0xffffffffu, sum[nt][j], d);
                    join_sums(top[nt][j], sum[nt][j], t, s);
                }
                if (lane < 4) {
                    tops[warp][8 * nt + 2 * lane + j] = top[nt][j];
                    sums[warp][8 * nt + 2 * lane + j] = sum[nt][j];
                }
            }
        __syncthreads();
        if (threadIdx.x < COLUMNS && piece.u.column0 + (int)threadIdx.x < piece.columns) {
            float t = tops[0][threadIdx.x], s = sums[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) join_sums(t, s, tops[w][threadIdx.x], sums[w][threadIdx.x]);
            const int64_t column = (head * p.tokens + piece.u.row0) * p.group + piece.u.column0 + threadIdx.x;
            p.stats[column * p.pieces + piece.index] = make_float2(t, s);
        }
        __syncthreads();
    }
}

// The pieces' parts of `count` columns joined: a column's largest score and what its powers of two are multiplied with, 0 where it sees nothing or
// is none.  A warp to a column.
__device__ __forceinline__ void column_totals(const WeightsParams &p, const Piece &piece, int head, int count, float2 *totals)
{
    const int lane = threadIdx.x & 31;
    for (int in_tile = threadIdx.x >> 5; in_tile < count; in_tile += blockDim.x >> 5) {
        float top = kNothing, sum = 0.0f;
        if (piece.u.column0 + in_tile < piece.columns) {
            const float2 *const from = p.stats + ((head * p.tokens + piece.u.row0) * p.group + piece.u.column0 + in_tile) * p.pieces;
#pragma unroll 4
            for (int i = lane; i < piece.pieces; i += 32) {
                const float2 part = from[i];
                join_sums(top, sum, part.x, part.y);
            }
        }
        float high = top;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, d));
        sum *= exp2f(top - high);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) totals[in_tile] = sum == 0.0f ? make_float2(0.0f, 0.0f) : make_float2(high, 1.0f / sum);
    }
}

// Scores that were kept: LANES threads to a token (one for few columns, eight for many), kTogether tokens at a time.
constexpr int kKeptThreads = 256, kTogether = 4, kKeptColumns = 128;

template <int LANES>
__global__ void __launch_bounds__(kKeptThreads, 4) kv_weights_kept_kernel(const __grid_constant__ WeightsParams p)
{
    __shared__ alignas(16) float2 totals[kKeptColumns];
    __shared__ int2 ranges[kKeptColumns];  // tokens that a column sees: the others' places may never have been written
    Piece piece;
    // the lengths are what the kernel in front read: nothing has written them since
    const bool found = find_piece(p, blockIdx.x, &piece);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the one in front, too
    if (!found) return;
    const int head = blockIdx.y, sub = threadIdx.x % LANES;
    const int64_t stride = scores_stride(piece.columns);
    const int32_t first = piece.u.tile0 * kKvTile, last = min(piece.u.tile1 * kKvTile, tokens_held(p, piece.u.length));
    constexpr int32_t kOne = kKeptThreads / LANES, kStep = kOne * kTogether;
    const float *const scores = scores_at(p, piece, head, 0);
    // whole blocks go round together: the columns' totals are theirs
    for (int32_t t0 = first; t0 < last; t0 += kStep) {
        float w[kTogether] = {};
        for (piece.u.column0 = 0; piece.u.column0 < piece.columns; piece.u.column0 += kKeptColumns) {
            const int count = min(kKeptColumns, piece.columns - piece.u.column0);
            if (piece.columns > kKeptColumns || t0 == first) {
                __syncthreads();
                column_totals(p, piece, head, count, totals);
                if ((int)threadIdx.x < count) column_range(p, piece.u, piece.u.column0 + threadIdx.x, &ranges[threadIdx.x].x, &ranges[threadIdx.x].y);
                __syncthreads();
            }
            // tokens whose scores are there: those that some column sees; all of these columns see the step's
            const View v = view(p, piece, kKeptColumns);
            const bool all = t0 >= v.all_lo && min(t0 + kStep, last) <= v.all_hi;
            if (t0 >= v.tile1 * kKvTile || t0 + kStep <= v.tile0 * kKvTile) continue;
            const auto go = [&](auto vector, auto masked) {
                using V = decltype(vector);
                constexpr int N = sizeof(V) / 4;
                for (int c = N * sub; c < count; c += N * LANES) {
                    union Scores {
                        V v;
                        float e[N];
                    } s[kTogether];
#pragma unroll
                    for (int k = 0; k < kTogether; ++k) {
                        const int32_t t = t0 + k * kOne + threadIdx.x / LANES;
#pragma unroll
                        for (int i = 0; i < N; ++i) s[k].e[i] = -INFINITY;
                        if (t < last && t >= v.tile0 * kKvTile && t < v.tile1 * kKvTile) s[k].v = *reinterpret_cast<const V *>(scores + t * stride + piece.u.column0 + c);
                    }
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        if (N > 1 && c + i >= count) break;
                        const float2 total = totals[c + i];
                        int2 range = make_int2(0, 0x7fffffff);
                        if (decltype(masked)::value) range = ranges[c + i];
#pragma unroll
                        for (int k = 0; k < kTogether; ++k) {
                            const int32_t t = t0 + k * kOne + threadIdx.x / LANES;
                            if (!decltype(masked)::value || (s[k].e[i] != -INFINITY && t >= range.x && t < range.y)) w[k] = fmaf(exp2_fast(s[k].e[i] - total.x), total.y, w[k]);
                        }
                    }
                }
            };
            // 0 times what a column that is not finite has would not be 0
            bool finite = true;
            if (all)
                for (int c = threadIdx.x & 31; c < count; c += 32) finite = finite && totals[c].y == totals[c].y;
            const bool plain = __all_sync(0xffffffffu, all && finite);
            if (stride % 4 == 0) plain ? go(float4(), std::false_type()) : go(float4(), std::true_type());
            else plain ? go(float2(), std::false_type()) : go(float2(), std::true_type());
        }
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const int32_t t = t0 + k * kOne + threadIdx.x / LANES;
#pragma unroll
            for (int d = 1; d < LANES; d <<= 1) w[k] += __shfl_xor_sync(0xffffffffu, w[k], d);
            if (t < last && sub == 0) put_weight(p, piece.u, head, t, w[k]);
        }
    }
}

template <int B, int NT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(B, NT, SPLIT)) kv_weights_sum_kernel(const __grid_constant__ WeightsParams p)
{
    constexpr int COLUMNS = 8 * NT;
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ float2 totals[COLUMNS];
    float *const weights = reinterpret_cast<float *>(smem) + kWarps * kStages * key_words(B);  // of the piece's tokens
    Piece piece;
    // The lengths are what the kernel in front read, nothing has written them since; of a call without rows there is none in front, and who
    // has written them may still be at it.
    if (p.tokens == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
    const bool found = find_piece(p, blockIdx.x, &piece);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the one in front, too
    if (!found) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, head = blockIdx.y;
    const int tokens = (piece.u.tile1 - piece.u.tile0) * kKvTile;
    for (int i = threadIdx.x; i < tokens; i += kThreads) weights[i] = 0.0f;
    for (piece.u.column0 = 0; piece.u.column0 < piece.columns; piece.u.column0 += COLUMNS) {
        column_totals(p, piece, head, COLUMNS, totals);
        __syncthreads();
        const View v = view(p, piece, COLUMNS);
        {
            Columns<B, NT, SPLIT> c;
            c.load(p, piece.u, head);
            float top[NT][2], part[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    top[nt][j] = totals[8 * nt + 2 * (lane & 3) + j].x;
                    part[nt][j] = totals[8 * nt + 2 * (lane & 3) + j].y;
                }
            each_tile<B>(p, piece, v, head, smem + warp * kStages * key_words(B), [&](int32_t tile, const uint32_t *words) {
                if (!words) return;
                float s[NT][4], w[2] = {0.0f, 0.0f};
                const int32_t token0 = tile * kKvTile;
                if (token0 >= v.all_lo && token0 + kKvTile <= v.all_hi) c.template scores<false>(words, token0, s);
                else c.template scores<true>(words, token0, s);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i >> 1] += s[nt][i] == -INFINITY ? 0.0f : exp2_fast(s[nt][i] - top[nt][i & 1]) * part[nt][i & 1];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    w[r] += __shfl_xor_sync(0xffffffffu, w[r], 1);
                    w[r] += __shfl_xor_sync(0xffffffffu, w[r], 2);
                    if ((lane & 3) == 0) weights[(tile - piece.u.tile0) * kKvTile + 8 * r + (lane >> 2)] += w[r];
                }
            });
        }
        __syncthreads();
    }
    __syncthreads();
    const int32_t held = tokens_held(p, piece.u.length);
    for (int i = threadIdx.x; i < tokens && piece.u.tile0 * kKvTile + i < held; i += kThreads) put_weight(p, piece.u, head, piece.u.tile0 * kKvTile + i, weights[i]);
}

template <int B, int NT, bool SPLIT>
lce_status launch(const WeightsParams &p, cudaStream_t s)
{
    constexpr size_t ring = (size_t)kWarps * kStages * key_words(B) * 4, all = ring + (size_t)kMostTiles * kKvTile * 4;
    static SmemOptIn first_opt_in, second_opt_in;
    if (!first_opt_in.ensure(kv_weights_scores_kernel<B, NT, SPLIT>, ring) || !second_opt_in.ensure(kv_weights_sum_kernel<B, NT, SPLIT>, all)) return LCE_ERR_CUDA;
    const dim3 grid((unsigned)p.units, (unsigned)p.g.heads);
    if (p.tokens > 0) {
        // many columns of few tokens: blocks share the columns (579 rows on 579 tokens, 3 heads of 256 channels: 366 us without, 86 with)
        const int64_t each = (p.tokens * p.group + p.batch - 1) / p.batch;
        const int64_t side = std::min<int64_t>((each + 8 * NT - 1) / (8 * NT), std::max<int64_t>(148 * kBlocksPerSm / ((int64_t)p.units * p.g.heads), 1));
        const lce_status st = launch_dependent(kv_weights_scores_kernel<B, NT, SPLIT>, dim3(grid.x, grid.y, (unsigned)side), kThreads, ring, s, p);
        if (st != LCE_OK) return st;
    }
    if (p.scores) return launch_dependent(p.tokens * p.group > 32 * (int64_t)p.batch ? kv_weights_kept_kernel<8> : kv_weights_kept_kernel<1>, grid, kKeptThreads, 0, s, p);
    return launch_dependent(kv_weights_sum_kernel<B, NT, SPLIT>, grid, kThreads, all, s, p);
}

// 16 columns where their operands fit a thread's registers
constexpr int kWideBlocks = 4;

template <int NT, bool SPLIT>
lce_status launch_blocks(const WeightsParams &p, cudaStream_t s)
{
    switch (p.g.blocks) {
        case 1: return launch<1, NT, SPLIT>(p, s);
        case 2: return launch<2, NT, SPLIT>(p, s);
        case 3: return launch<3, NT, SPLIT>(p, s);
        case 4: return launch<4, NT, SPLIT>(p, s);
        case 5: return launch<5, 1, SPLIT>(p, s);
        case 6: return launch<6, 1, SPLIT>(p, s);
        case 7: return launch<7, 1, SPLIT>(p, s);
        default: return launch<8, 1, SPLIT>(p, s);
    }
}

bool stride_ok(int64_t s) { return s >= 0 && s < (1ll << 40); }

lce_status make_params(const lce_kv_attention_weights_desc *d, WeightsParams *p, int *nt)
{
    if (!d) return LCE_ERR_INVALID_ARG;
    const lce_status st = make_kv_geom(&d->cache, &p->g);
    if (st != LCE_OK) return st;
    if (d->batch <= 0 || d->heads <= 0 || d->table_pages <= 0 || d->tokens < 0 || d->window < 0 || !type_known(d->type)) return LCE_ERR_INVALID_ARG;
    if (d->causal != 0 && d->causal != 1) return LCE_ERR_INVALID_ARG;
    if (d->heads % d->cache.kv_heads != 0 || !isfinite(d->scale) || !isfinite(d->decay)) return LCE_ERR_INVALID_ARG;
    for (const int64_t s : {d->q_token_stride, d->q_head_stride, d->previous_seq_stride, d->previous_head_stride, d->out_seq_stride, d->out_head_stride})
        if (!stride_ok(s)) return LCE_ERR_INVALID_ARG;
    if (d->tokens >= (1ll << 31) || d->tokens * d->heads >= (1ll << 31) || (int64_t)d->table_pages * d->cache.page_size >= (1ll << 30) || d->batch >= (1 << 20) ||
        (int64_t)p->g.slots / kKvTile * p->g.heads >= (1ll << 31))
        return LCE_ERR_UNSUPPORTED;
    p->batch = d->batch; p->group = d->heads / d->cache.kv_heads; p->table_pages = d->table_pages;
    p->table_tokens = d->table_pages * d->cache.page_size;
    p->causal = d->causal; p->window = d->window; p->type = d->type;
    p->tokens = d->tokens;
    p->q_token = d->q_token_stride; p->q_head = d->q_head_stride;
    p->scale = d->scale * 1.44269504088896341f;
    p->decay = d->decay;
    p->previous_seq = d->previous_seq_stride; p->previous_head = d->previous_head_stride;
    p->out_seq = d->out_seq_stride; p->out_head = d->out_head_stride;
    *nt = p->g.blocks <= kWideBlocks && (d->tokens * p->group + d->batch - 1) / d->batch > 8 ? 2 : 1;
    // Many rows go to the kernels of kv_weights_prompt.cu where they are estimated to be ahead (us, by tokens times key heads; by the longest the
    // sequences can be: their lengths are not known here).  Measured with 128 channels in bf16 and used for fewer, too: those kernels' time hardly depends on
    // the channels (two chunks of 1024 rows on 5120 tokens: 32 channels 268 us, 64 279, 96 283, 128 291), that of the others falls with them.  One sequence of 512 / 4096 / 32768 tokens, 8 key heads: 20 columns
    // 16.2 / 28.3 / 46.1 here and 24.6 / 27.4 / 81.4 there, 64 columns 35.2 / 61.3 / 99.2 and 24.4 / 27.8 / 81.3; 16 sequences of 512 / 4096: 32 columns 38.0 / 86.1
    // and 38.6 / 132, 128 columns 132 / 415 and 37.1 / 106.
    const double each = (double)p->tokens * p->group / p->batch, read = (double)p->batch * p->g.heads * p->table_tokens;
    p->prompt = p->g.blocks <= 4 && d->type != LCE_TYPE_FLOAT32 && ceil(each / 16) * (11.0 + 6.5e-5 * read) > 24.0 + ceil(each / 256) * 1.65e-4 * read &&
                p->g.heads < 65535 && (double)p->g.heads * p->batch * (p->table_tokens / 256 + 1) < kMostUnits;
    // As many pieces as the GPU has places for, as a sequence has one more than its share (48 of 1 - 8192 tokens, 8 heads: 72 us, with a
    // piece for each place whatever the sequences 77, with two 72; 16 of up to 1500, 12 heads: 14.8, 19.3 and 24.2), but for many sequences half of
    // them at least; fewer where there are so many columns that their sums would take much room.
    const int64_t columns = std::max<int64_t>(p->tokens * d->heads, 1), places = 148 * kBlocksPerSm / p->g.heads;
    p->target = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(places - p->batch, places / 2), kMostStats / 8 / columns));
    const int64_t tiles = (p->table_tokens + kKvTile - 1) / kKvTile;
    const int64_t units = p->batch * ((tiles + kLeastTiles - 1) / kLeastTiles);
    p->pieces = (int32_t)std::min<int64_t>(tiles, std::max<int64_t>(p->target, (tiles + kMostTiles - 1) / kMostTiles) + 1);
    p->units = (int32_t)std::min<int64_t>(units, p->batch + std::max<int64_t>(p->target, (p->batch * tiles + kMostTiles - 1) / kMostTiles));
    // what sequences as long as the table would leave
    p->scores_head = (p->tokens * p->group + p->batch) * tiles * kKvTile;
    return LCE_OK;
}

size_t stats_bytes(const WeightsParams &p) { return ((size_t)p.tokens * p.group * p.g.heads * p.pieces * 8 + 15) / 16 * 16; }
// Scores are kept where there is room for them.
size_t scores_bytes(const WeightsParams &p)
{
    const double bytes = 4.0 * p.scores_head * p.g.heads;
    return p.tokens > 0 && bytes <= kMostScores ? (size_t)p.scores_head * p.g.heads * 4 : 0;
}

size_t workspace_bytes(const WeightsParams &p)
{
    return std::max<size_t>(p.prompt ? kv_weights_prompt_bytes(p) : stats_bytes(p) + scores_bytes(p), 16);
}

}  // namespace
}  // namespace lce

extern "C" size_t lce_kv_attention_weights_workspace_bytes(const lce_kv_attention_weights_desc *desc)
{
    using namespace lce;
    WeightsParams p{};
    int nt;
    if (make_params(desc, &p, &nt) != LCE_OK) return 0;
    return workspace_bytes(p);
}

extern "C" lce_status lce_kv_attention_weights(const lce_kv_attention_weights_desc *desc, const void *q, const void *cache, const int32_t *page_table,
                                               const int32_t *lengths, const int32_t *q_starts, const float *previous, float *out, void *workspace,
                                               size_t workspace_size, void *stream)
{
    using namespace lce;
    WeightsParams p{};
    int nt;
    const lce_status st = make_params(desc, &p, &nt);
    if (st != LCE_OK) return st;
    if (!q_starts && desc->tokens != desc->batch) return LCE_ERR_INVALID_ARG;
    if ((!q && desc->tokens > 0) || !cache || !page_table || !lengths || !out || !workspace) return LCE_ERR_INVALID_ARG;
    const size_t element = type_size(desc->type);
    if (!aligned(q, element) || !aligned(cache, 16) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(q_starts, 4) || !aligned(previous, 4) ||
        !aligned(out, 4) || !aligned(workspace, 16))
        return LCE_ERR_ALIGNMENT;
    if (workspace_size < workspace_bytes(p)) return LCE_ERR_WORKSPACE;
    // A weight is written by the thread that reads the previous one, so only in place may they be the same memory.  How long rows are follows from
    // the lengths, on the device: here every row is looked at by its first element.
    const RowSet new_sums{out, p.batch, p.g.heads, p.out_seq, p.out_head, 1, 4}, old_sums{previous, p.batch, p.g.heads, p.previous_seq, p.previous_head, 1, 4};
    if (!rows_apart(new_sums)) return LCE_ERR_INVALID_ARG;
    if (previous == out) {
        if (desc->decay != 0.0f && ((p.batch > 1 && p.previous_seq != p.out_seq) || (p.g.heads > 1 && p.previous_head != p.out_head))) return LCE_ERR_INVALID_ARG;
    } else if (previous && desc->decay != 0.0f && rows_meet(old_sums, new_sums)) {
        return LCE_ERR_INVALID_ARG;
    }
    p.q_vectors = p.g.dim % 8 == 0 && aligned(q, 8 * element) && p.q_token % 8 == 0 && p.q_head % 8 == 0;
    p.q = q; p.cache = static_cast<const uint32_t *>(cache); p.page_table = page_table; p.lengths = lengths; p.q_starts = q_starts;
    p.previous = desc->decay != 0.0f ? previous : nullptr;
    p.sums = out;
    if (p.prompt) return launch_kv_weights_prompt(p, workspace, static_cast<cudaStream_t>(stream));
    p.stats = static_cast<float2 *>(workspace);
    p.scores = scores_bytes(p) ? reinterpret_cast<float *>(static_cast<char *>(workspace) + stats_bytes(p)) : nullptr;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (desc->type == LCE_TYPE_FLOAT32) return nt == 2 ? launch_blocks<2, true>(p, s) : launch_blocks<1, true>(p, s);
    return nt == 2 ? launch_blocks<2, false>(p, s) : launch_blocks<1, false>(p, s);
}
