// Attention weights by token of many rows (a prompt, or its last rows), on the 5th-generation tensor cores.
//
// The softmax needs a column's largest score and sum before its first weight is known, so the scores are made twice, by two kernels of one
// shape: 256 rows of one operand stay in shared memory, tiles of 128 rows of the other one stream past them, and two threads
// have one of the 256 in TMEM, 64 of its 128 products a step each.
//   first     256 columns (rows of q that share a key/value head) stay, keys stream: threads have a column's scores, and keep their
//             largest and the sum of their powers of two
//   second    256 tokens stay, columns stream: threads have a token's scores, and add its weights up.  The logarithms of the columns' sums
//             lie in shared memory
// So no sum crosses threads before a unit's end.  Work is cut into units of a few steps: (256 columns, a piece of the sequence) and (256 tokens,
// a chunk of the columns), joined in a fixed order by small kernels.  The kernel that puts the rows of q in order as f16 lists them; 148
// blocks take them in turn, and their warps go from one to the next without meeting:
//   warps 0 - 15        the powers of two: two threads to each of the 256, for 64 of a step's 128 each; two accumulators of 128 x 128 for
//                       every 128 of the 256 in TMEM
//   warps 16 - 23       4-bit words to f16 keys, both in shared memory
//   warp 24             issues the products
//   warp 25             has the rows of q copied
//   warp 26             has the keys' words copied from the cache (loads of the warps that decode them do not stay in flight over the fence in
//                       front of the products: 143 instead of 125 us for the first kernel)
//
// Two sequences of 1024 rows of 4 columns on 5120 tokens, 8 key heads of 128 channels: 278 us, 125 and 135 of them in the two kernels.  Products (1024
// clocks for a step of 256 x 128 at the tensor cores' rate) and powers of two (2048 at 16 a clock) would allow 70 each; a step takes 3500.  Taken out one by
// one, the powers of two are 15 % of it, the products 5 %, reading TMEM 25 %: what is left is the way through shared memory that the warps hand each
// other a tile on.  More tiles streaming (four instead of two), one arrival a warp at the barriers, 128-byte swizzled operands and eight warps with twice
// the registers for the powers of two were all within 3 % of this.
//
// f16 holds a code times its scale exactly, relative to the largest scale of 128 tokens, down to 2^-28 of it; 16-bit rows of q,
// 128 of them times one power of two, are exact down to 2^-24 of their largest element at least, and what is lost of smaller ones is below 2^-39 of it.
// Scores and sums are fp32.
#include "kv_tensor.cuh"
#include "kv_weights.cuh"
#include "kv_weights_rings.cuh"

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

constexpr int kSoftmaxWarps = 16, kProducerWarps = 8, kIssuerWarp = kSoftmaxWarps + kProducerWarps, kCopyWarp = kIssuerWarp + 1, kWordsWarp = kCopyWarp + 1;
constexpr int kThreads = 32 * (kWordsWarp + 1);
constexpr float kNothing = -3e38f;   // stands for the largest score where there is none
constexpr float kRise = 16.0f;       // the score that powers of two are relative to is raised when one passes it by this much
constexpr int kBlocks = 148;         // one to an SM
constexpr int kSteps = kBlocks * 8;  // units are cut so that there are about as many
constexpr int kHeldUnits = 32;       // of a block, in shared memory

enum { BAR_STAY_FULL = 0, BAR_STAY_EMPTY = BAR_STAY_FULL + 2, BAR_STREAM_FULL = BAR_STAY_EMPTY + 2, BAR_STREAM_EMPTY = BAR_STREAM_FULL + 2,
       BAR_WORDS_FULL = BAR_STREAM_EMPTY + 2, BAR_WORDS_EMPTY = BAR_WORDS_FULL + 2, BAR_S_FULL = BAR_WORDS_EMPTY + 2, BAR_S_EMPTY = BAR_S_FULL + 4, BAR_DONE = BAR_S_EMPTY + 4, BAR_COUNT };

struct TileInfo {
    float unit;      // 2^e: scores count in it
    uint32_t valid;  // bit per 16 tokens: their page is in the pool
};

// A unit of work.
struct alignas(16) WorkUnit {
    int32_t seq, length, rows, held;  // tokens of the sequence, its rows of q, tokens that its pages hold
    int32_t columns, tiles_before;    // columns; tiles of columns of the sequences in front
    int32_t head, first;              // the first of the 256 columns, or tokens, that stay
    int32_t step0, step1;
    int32_t part;                     // second kernel: where its sums wait for the other chunks'; negative: it has no others
    int32_t unused;
};

struct Shared {
    uint64_t bars[BAR_COUNT];
    uint32_t tmem, largest[2][kProducerWarps], valid[2];  // valid: of a tile's words, as in TileInfo
    TileInfo info[kInfos];
    alignas(16) __half scales[2][kTokens][4];         // relative to the tile's largest; [turn]
    alignas(16) float columns[2][2][kTokens];         // [half][turn]: the logarithms of columns' sums, taken off
    float2 others[2][2][kTokens];                     // [half][turn]: what the second of two threads has at a unit's end
    WorkUnit units[kHeldUnits];                       // the block's first ones
};

constexpr int kMiscBytes = 12288;
static_assert(sizeof(Shared) <= kMiscBytes, "");
// Words of 128 tokens: the keys of eight tiles of the cache, then their scales.
__host__ __device__ constexpr int words_bytes(int blocks) { return kTokens / kKvTile * 320 * blocks; }
constexpr size_t weights_smem(int blocks) { return kMiscBytes + 6 * (size_t)(kTokens * 64 * blocks) + 2 * words_bytes(blocks); }

struct PromptParams : WeightsParams {
    WorkUnit *units[2];
    int32_t *unit_counts;
    int32_t most_tiles, most_units[2], most_parts;  // that there is room for
    uint8_t *images;      // [tile of 128 columns][kv head]: rows of q as f16, in the order in which they are an operand
    float *factors;       // [tile of columns][kv head][128]
    float2 *stats_units;  // [unit of the first kernel][256]: largest, sum
    float *tile_factors;  // [tile of columns][kv head]: the factor of all its rows that are finite
    float *constants;     // [tile of columns][kv head][128]: less the logarithm of the sum
    float *parts;         // [unit of the second kernel of sequences whose columns are cut][256]
};

__device__ __forceinline__ int32_t up(int32_t n, int32_t by) { return (n + by - 1) / by; }

// How a call is cut: steps of a unit of each kernel.
struct Cut {
    int32_t first, second;
};

// What a sequence has of everything that is counted through the batch.
struct Counts {
    int32_t tiles, units[2], parts;  // tiles of columns; units of each kernel; units of the second that are joined
};
__device__ __forceinline__ Counts counts(const PromptParams &p, const Sequence &s, const Cut &cut)
{
    const int32_t held = tokens_held(p, s.length), columns = s.rows * p.group, chunks = max(up(up(columns, 128), cut.second), 1);
    Counts c;
    c.tiles = up(columns, 128);
    c.units[0] = p.g.heads * up(columns, 256) * up(up(held, kTokens), cut.first);
    c.units[1] = p.g.heads * up(held, 256) * chunks;
    c.parts = chunks > 1 ? c.units[1] : 0;
    return c;
}

__device__ __forceinline__ Cut find_cut(const PromptParams &p)
{
    const int lane = threadIdx.x & 31;
    int64_t first = 0, second = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const Sequence s = sequence<8>(p, b0 + lane);
        const int64_t held = tokens_held(p, s.length), columns = (int64_t)s.rows * p.group;
        first += (columns + 255) / 256 * ((held + kTokens - 1) / kTokens);
        second += (held + 255) / 256 * ((columns + 127) / 128);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        first += __shfl_xor_sync(0xffffffffu, first, d);
        second += __shfl_xor_sync(0xffffffffu, second, d);
    }
    Cut cut;
    cut.first = (int32_t)max((first * p.g.heads + kSteps - 1) / kSteps, (int64_t)2);
    cut.second = (int32_t)max((second * p.g.heads + kSteps - 1) / kSteps, (int64_t)2);
    return cut;
}

// Finds the sequence that the `at`-th of what `count` counts belongs to, and what the sequences in front of it have.  By whole warps.
template <typename Count>
__device__ __forceinline__ int32_t find_sequence(const PromptParams &p, const Cut &cut, int at, Count count, Counts *before)
{
    const int lane = threadIdx.x & 31;
    *before = Counts{};
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const Counts c = counts(p, sequence<8>(p, b0 + lane), cut);
        Counts upto = c;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t t = __shfl_up_sync(0xffffffffu, upto.tiles, d), u0 = __shfl_up_sync(0xffffffffu, upto.units[0], d),
                          u1 = __shfl_up_sync(0xffffffffu, upto.units[1], d), q = __shfl_up_sync(0xffffffffu, upto.parts, d);
            if (lane >= d) {
                upto.tiles += t;
                upto.units[0] += u0;
                upto.units[1] += u1;
                upto.parts += q;
            }
        }
        const uint32_t has = __ballot_sync(0xffffffffu, count(*before) + count(upto) > at);
        const int from = has ? __ffs(has) - 1 : 31;
        const Counts mine = has ? c : Counts{};
        before->tiles += __shfl_sync(0xffffffffu, upto.tiles - mine.tiles, from);
        before->units[0] += __shfl_sync(0xffffffffu, upto.units[0] - mine.units[0], from);
        before->units[1] += __shfl_sync(0xffffffffu, upto.units[1] - mine.units[1], from);
        before->parts += __shfl_sync(0xffffffffu, upto.parts - mine.parts, from);
        if (has) return b0 + from;
    }
    return -1;
}
// What the sequences in front of sequence b have.
__device__ __forceinline__ void find_sequence(const PromptParams &p, const Cut &cut, int b, Counts *before)
{
    const int lane = threadIdx.x & 31;
    *before = Counts{};
    for (int b0 = 0; b0 < b; b0 += 32) {
        Counts c{};
        if (b0 + lane < b) c = counts(p, sequence<8>(p, b0 + lane), cut);
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            c.tiles += __shfl_xor_sync(0xffffffffu, c.tiles, d);
            c.units[0] += __shfl_xor_sync(0xffffffffu, c.units[0], d);
            c.units[1] += __shfl_xor_sync(0xffffffffu, c.units[1], d);
            c.parts += __shfl_xor_sync(0xffffffffu, c.parts, d);
        }
        before->tiles += c.tiles;
        before->units[0] += c.units[0];
        before->units[1] += c.units[1];
        before->parts += c.parts;
    }
}

// Columns [lo, hi) that see some of tokens [t0, t1): their ranges move up with the rows, so they are a run.
__device__ __forceinline__ void columns_of(const PromptParams &p, int32_t length, int32_t rows, int32_t t0, int32_t t1, int32_t *lo, int32_t *hi)
{
    const int64_t row0 = (int64_t)length - rows;  // position of the first row
    *lo = p.causal ? (int32_t)(min(max(t0 - row0, (int64_t)0), (int64_t)rows) * p.group) : 0;
    *hi = (p.window > 0 ? (int32_t)min(max((int64_t)t1 - 1 + p.window - row0, (int64_t)0), (int64_t)rows) : rows) * p.group;
}

// Writes one sequence's units of both kernels down, a thread to a unit; the last sequence says how many there are.
__device__ __forceinline__ void list_units(const PromptParams &p, int b)
{
    const Cut cut = find_cut(p);
    Counts before;
    const int seq = b < p.batch ? b : -1;
    find_sequence(p, cut, seq, &before);
    if (seq < 0) return;
    const Sequence s = sequence<8>(p, seq);
    const Counts mine = counts(p, s, cut);
    // more than there is room for: rows of q that are several sequences' (q_starts that decrease); nothing is done then
    Counts all;
    find_sequence(p, cut, p.batch, &all);
    if (all.tiles > p.most_tiles || all.units[0] > p.most_units[0] || all.units[1] > p.most_units[1] || all.parts > p.most_parts) {
        if (seq == p.batch - 1 && threadIdx.x < 2) p.unit_counts[threadIdx.x] = 0;
        return;
    }
    if (seq == p.batch - 1 && threadIdx.x < 2) p.unit_counts[threadIdx.x] = before.units[threadIdx.x] + mine.units[threadIdx.x];
    const int32_t held = tokens_held(p, s.length), columns = s.rows * p.group;
#pragma unroll
    for (int kernel = 0; kernel < 2; ++kernel) {
        const int32_t outer = kernel ? up(held, 256) : up(columns, 256), each = kernel ? cut.second : cut.first;
        const int32_t inner = kernel ? max(up(up(columns, 128), each), 1) : up(up(held, kTokens), each);
        for (int32_t local = threadIdx.x; local < mine.units[kernel]; local += blockDim.x) {
            const int32_t of_outer = local / inner, i = local - of_outer * inner, head = of_outer / outer, first = 256 * (of_outer - head * outer);
            int32_t lo, hi, unused;
            if (kernel) {
                columns_of(p, s.length, s.rows, first, min(first + 256, held), &lo, &hi);
            } else {
                Unit u{};
                u.length = s.length;
                u.rows = s.rows;
                column_range(p, u, first, &lo, &unused);
                column_range(p, u, min(first + 256, columns) - 1, &unused, &hi);
            }
            // equal shares of what is seen
            const int32_t seen0 = lo / 128, seen = hi > lo ? up(hi, 128) - seen0 : 0;
            const WorkUnit w{seq, s.length, s.rows, held, columns, before.tiles, head, first, seen0 + (int32_t)((int64_t)seen * i / inner),
                             seen0 + (int32_t)((int64_t)seen * (i + 1) / inner), kernel && inner > 1 ? before.parts + local : -1, 0};
            p.units[kernel][before.units[kernel] + local] = w;
        }
    }
}

// The block's k-th unit, which is unit `at`.
template <bool SUMS>
__device__ __forceinline__ WorkUnit load_unit(const PromptParams &p, const Shared &sh, int32_t k, int32_t at)
{
    return k < kHeldUnits ? sh.units[k] : p.units[SUMS][at];
}
__device__ __forceinline__ int64_t image_of(const PromptParams &p, const WorkUnit &w, int32_t tile) { return (int64_t)(w.tiles_before + tile) * p.g.heads + w.head; }
// Whether the second 128 of what stays exist.
template <bool SUMS>
__device__ __forceinline__ int halves_of(const WorkUnit &w) { return w.first + 128 < (SUMS ? w.held : w.columns) ? 2 : 1; }

// Rows of q as f16 operands and what their scores are multiplied with: a warp to eight rows, lane 8 c + r to every fourth group of eight channels
// of row r, which is how they lie in the operand; a block to 128 columns.  A last row of blocks lists the units of the kernels to come.
constexpr int kRowsThreads = 4 * kTokens;

template <int B>
__global__ void __launch_bounds__(kRowsThreads) kv_weights_rows_kernel(const __grid_constant__ PromptParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    release_join();
    constexpr int ROWS8 = 512 * B;
    __shared__ uint32_t largest[kRowsThreads / 32];
    if (blockIdx.y == p.g.heads) {
        for (int b = blockIdx.x; b < p.batch; b += gridDim.x) list_units(p, b);
        return;
    }
    Counts before;
    const Cut cut{1, 1};
    const int seq = find_sequence(p, cut, blockIdx.x, [](const Counts &c) { return c.tiles; }, &before), head = blockIdx.y;
    if (seq < 0) return;
    const Sequence s = sequence<8>(p, seq);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_tile = 8 * warp + (lane & 7), quarter = lane >> 3;
    const int column = (blockIdx.x - before.tiles) * 128 + in_tile, row = column / p.group;
    const int64_t at = (s.row0 + row) * p.q_token + ((int64_t)head * p.group + (column - row * p.group)) * p.q_head + 8 * quarter, image = (int64_t)blockIdx.x * p.g.heads + head;
    uint8_t *const to = p.images + image * (kTokens * 64 * B) + warp * ROWS8 + lane * 16;
    const auto take_rows = [&](auto element, auto vectors) {
        using T = decltype(element);
        Eight<T> e[B];
#pragma unroll
        for (int b = 0; b < B; ++b) e[b] = load_eight<T, decltype(vectors)::value>(static_cast<const T *>(p.q) + at + 32 * b, row < s.rows ? p.g.dim - 32 * b - 8 * quarter : 0);
        uint32_t magnitude = 0;  // magnitudes compare like integers, infinity and NaN above all others
        float v[8];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            e[b].expand(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) magnitude = max(magnitude, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        magnitude = max(magnitude, __shfl_xor_sync(0xffffffffu, magnitude, 8));
        magnitude = max(magnitude, __shfl_xor_sync(0xffffffffu, magnitude, 16));
        const bool finite = magnitude < 0x7f800000u;
        // all 128 rows times 2^k, so that the largest is in [2^14, 2^15); a scale below zero changes q's sign
        const uint32_t of_warp = __reduce_max_sync(0xffffffffu, finite ? magnitude : 0);
        if (lane == 0) largest[warp] = of_warp;
        __syncthreads();
        const uint32_t top = __reduce_max_sync(0xffffffffu, largest[lane % (kRowsThreads / 32)]);
        const int k = 14 - (top > 0 ? ilogbf(__uint_as_float(top)) : 0), k1 = k / 2, k2 = k - k1;
        const float s1 = __uint_as_float((uint32_t)(127 + k1) << 23) * (p.scale < 0.0f ? -1.0f : 1.0f), s2 = __uint_as_float((uint32_t)(127 + k2) << 23);
#pragma unroll
        for (int b = 0; b < B; ++b) {
            e[b].expand(v);
            // in the order in which a word's codes are decoded; a row that is not finite is one by its factor
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = finite ? v[i] * s1 * s2 : 0.0f;
            *reinterpret_cast<uint4 *>(to + b * 512) = make_uint4(pack_half2(v[0], v[4]), pack_half2(v[1], v[5]), pack_half2(v[2], v[6]), pack_half2(v[3], v[7]));
        }
        const int kc = -11 - k, c1 = kc / 2, c2 = kc - c1;
        const float factor = fabsf(p.scale) * __uint_as_float((uint32_t)(127 + c1) << 23) * __uint_as_float((uint32_t)(127 + c2) << 23);
        if (quarter == 0) p.factors[image * kTokens + in_tile] = finite ? factor : __uint_as_float(0x7fc00000u);
        if (threadIdx.x == 0) p.tile_factors[image] = factor;
    };
    if (p.type == LCE_TYPE_FLOAT16) {
        if (p.q_vectors) take_rows(__half(), std::true_type());
        else take_rows(__half(), std::false_type());
    } else {
        if (p.q_vectors) take_rows(__nv_bfloat16(), std::true_type());
        else take_rows(__nv_bfloat16(), std::false_type());
    }
}

// Eight tokens to a producer warp at a time, lane 8 q + t to channels 8 q .. of each block of token t.
constexpr int kKeyGroups = kTokens / 8 / kProducerWarps;

// The B words of a place (a lane's of 64 places, a token's of 16) in shared memory, plane by plane.
template <int B, int ROWS>
__device__ __forceinline__ void shared_planes(const uint32_t *base, int place, uint32_t (&w)[B])
{
    if (B == 4) {
        const uint4 v = reinterpret_cast<const uint4 *>(base)[place];
        w[0] = v.x; w[B > 1 ? 1 : 0] = v.y; w[B > 2 ? 2 : 0] = v.z; w[B > 3 ? 3 : 0] = v.w;
    } else {
        if (B & 2) {
            const uint2 v = reinterpret_cast<const uint2 *>(base)[place];
            w[0] = v.x; w[B > 1 ? 1 : 0] = v.y;
        }
        if (B & 1) w[B - 1] = base[ROWS * (B - 1) + place];
    }
}

// A wait of a whole warp.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bounded(bar, parity)); }
// Eight warps meet; whether all of them are well.
__device__ __forceinline__ bool half_sync_and(uint32_t barrier, bool ok)
{
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
        "bar.red.and.pred p, %2, 256, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)ok), "r"(barrier)
        : "memory");
    return all != 0;
}

// The tiles of keys that a block's units want, one after the other.
template <bool SUMS>
struct Tiles {
    WorkUnit w;
    int32_t k, unit, count, step;  // step: of the unit, or the half
    __device__ __forceinline__ void begin(const PromptParams &p, const Shared &sh, int32_t units)
    {
        k = 0;
        unit = blockIdx.x;
        count = units;
        settle(p, sh);
    }
    __device__ __forceinline__ bool there() const { return unit < count; }
    __device__ __forceinline__ void settle(const PromptParams &p, const Shared &sh)  // at the first tile of a unit that has one
    {
        for (; unit < count; unit += gridDim.x, ++k) {
            w = load_unit<SUMS>(p, sh, k, unit);
            if (w.step0 < w.step1) break;
        }
        step = SUMS ? 0 : w.step0;
    }
    __device__ __forceinline__ int32_t tile() const { return SUMS ? w.first / kTokens + step : step; }
    __device__ __forceinline__ bool last() const { return step + 1 == (SUMS ? halves_of<true>(w) : w.step1); }
    __device__ __forceinline__ void next(const PromptParams &p, const Shared &sh)
    {
        if (!last()) {
            ++step;
            return;
        }
        unit += gridDim.x;
        ++k;
        settle(p, sh);
    }
};

template <int B, bool SUMS>
__global__ void __launch_bounds__(kThreads, 1) kv_weights_prompt_kernel(const __grid_constant__ PromptParams p, const TimeoutReport report)
{
    constexpr uint32_t ROWS8 = 512 * B;  // bytes from eight rows to the next
    constexpr uint32_t TILE_BYTES = kTokens * 64 * B;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem);
    uint8_t *const stay_smem = smem + kMiscBytes, *const stream_smem = stay_smem + 4 * TILE_BYTES;  // two pairs of tiles; two tiles
    uint8_t *const words_smem = stream_smem + 2 * TILE_BYTES;
    constexpr uint32_t WORDS_BYTES = words_bytes(B), SCALES_AT = kTokens / kKvTile * 256 * B;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    release_join();
    const int32_t count = __ldg(p.unit_counts + SUMS);
    if ((int)blockIdx.x >= count) return;
    for (int i = threadIdx.x; i < 3 * kHeldUnits; i += kThreads) {
        const int32_t at = blockIdx.x + i / 3 * gridDim.x;
        if (at < count) reinterpret_cast<int4 *>(sh.units)[i] = reinterpret_cast<const int4 *>(p.units[SUMS] + at)[i % 3];
    }

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.bars[BAR_STAY_FULL + i], SUMS ? 32 * kProducerWarps : 1);
            mbar_init(&sh.bars[BAR_STAY_EMPTY + i], 1);
            mbar_init(&sh.bars[BAR_STREAM_FULL + i], SUMS ? 1 : 32 * kProducerWarps);
            mbar_init(&sh.bars[BAR_STREAM_EMPTY + i], 1);
            mbar_init(&sh.bars[BAR_WORDS_FULL + i], 1);
            mbar_init(&sh.bars[BAR_WORDS_EMPTY + i], 32 * kProducerWarps);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&sh.bars[BAR_S_FULL + i], 1);
            mbar_init(&sh.bars[BAR_S_EMPTY + i], 256);
        }
        mbar_init(&sh.bars[BAR_DONE], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuerWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh.tmem;
    bool ok = true;

    if (warp < kSoftmaxWarps) {
        // ---- powers of two: two threads to a column, or to a token ------------------------------------
        const int half = warp >> 2 & 1, side = warp >> 3, in_tile = threadIdx.x & 127;
        const uint32_t s_at = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 256 * half + 64 * side;
        uint32_t steps = 0, units = 0, units_here = 0, tiles = 0;  // steps of this half; units that have some; units of this half; tiles of keys so far
        // Brought ahead, also from one unit to the next: second kernel, of the next step's tile of columns its factor and what is taken off column
        // in_tile; first kernel, the factor of the next unit's column.
        float next_factor = 0.0f, next_constant = 0.0f;
        bool ahead = false;
        const auto bring = [&](const WorkUnit &w, int32_t step) {
            const int64_t image = image_of(p, w, SUMS ? step : w.first / kTokens + half);
            next_factor = SUMS ? p.tile_factors[image] : p.factors[image * kTokens + in_tile];
            if (SUMS && !side) next_constant = p.constants[image * kTokens + in_tile];
        };
        for (int32_t unit_at = blockIdx.x, k = 0; ok && unit_at < count; unit_at += gridDim.x, ++k) {
            const WorkUnit w = load_unit<SUMS>(p, sh, k, unit_at);
            if (half < halves_of<SUMS>(w)) {
                const int32_t own = w.first + 128 * half + in_tile;
                int32_t lo, hi;  // what it sees: of the tokens, or of the columns
                float factor = 0.0f, unit = 0.0f, top = kNothing;
                uint64_t sum[2] = {};  // pairs of fp32 sums
                const bool some = w.step0 < w.step1;
                if (SUMS) {
                    columns_of(p, w.length, w.rows, own, own + 1, &lo, &hi);
                } else {
                    Unit u{};
                    u.length = w.length;
                    u.rows = w.rows;
                    column_range(p, u, own, &lo, &hi);
                }
                if (some) {
                    if (!ahead) bring(w, w.step0);
                    factor = next_factor;
                    // the unit behind: if it is one without this half, or without steps, nobody uses what is brought for it
                    ahead = k + 1 < kHeldUnits && unit_at + (int32_t)gridDim.x < count;
                    if (!SUMS && ahead) {
                        const WorkUnit &behind = sh.units[k + 1];
                        ahead = behind.step0 < behind.step1 && half < halves_of<SUMS>(behind);
                        if (ahead) bring(behind, 0);
                    }
                }
                for (int32_t step = w.step0; ok && step < w.step1; ++step, ++steps) {
                    const uint32_t buffer = step_buffer(steps);
                    ok = warp_wait(&sh.bars[BAR_S_FULL + 2 * half + buffer], step_parity(steps));
                    if (!SUMS && !ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const int first = step * 128 + 64 * side;  // token, or column
                    uint32_t valid = 0xfu;
                    if (!SUMS || step == w.step0) {
                        const TileInfo info = sh.info[info_place(SUMS, tiles + (uint32_t)(step - w.step0), units, half)];
                        unit = info.unit;
                        if (SUMS) {
                            if (!(info.valid >> (in_tile >> 4) & 1)) hi = lo;  // its page is not in the pool
                        } else {
                            valid = info.valid >> (4 * side) & 0xfu;
                        }
                    }
                    if (SUMS) {
                        // the buffer before last is read by nobody any more
                        if (!side) sh.columns[half][buffer][in_tile] = next_constant;
                        factor = next_factor;
                        if (step + 1 < w.step1) {
                            bring(w, step + 1);
                        } else if (ahead) {
                            const WorkUnit &behind = sh.units[k + 1];
                            ahead = behind.step0 < behind.step1 && half < halves_of<SUMS>(behind);
                            if (ahead) bring(behind, behind.step0);
                        }
                        ok = half_sync_and(2 + half, ok);  // all eight warps leave together
                        if (!ok) break;
                    }
                    const bool all = __all_sync(0xffffffffu, valid == 0xfu && first >= lo && first + 64 <= hi);
                    const float f = factor * unit;
                    // 32 scores of the 64
                    const auto take = [&](const uint32_t (&r)[32], int c, uint32_t seen, auto masked) {
                        const uint64_t f2 = pair_of(f, f);
                        uint64_t plus = 0;
                        if (!SUMS) {
                            const auto score = [&](int i) { return decltype(masked)::value && !(seen >> i & 1) ? -INFINITY : __uint_as_float(r[i]); };
                            float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                            for (int i = 0; i < 32; ++i) tops[i & 3] = fmaxf(tops[i & 3], score(i));
                            float m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                            m = m == -INFINITY ? m : m * f;
                            if (m > top + kRise) {
                                const float by = exp2_fast(top - m);
                                sum[0] = mul_pair(sum[0], pair_of(by, by));
                                sum[1] = mul_pair(sum[1], pair_of(by, by));
                                top = m;
                            }
                            plus = pair_of(-top, -top);
                        }
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            if (SUMS) plus = *reinterpret_cast<const uint64_t *>(&sh.columns[half][buffer][64 * side + 32 * c + i]);
                            float x, y;
                            of_pair(fma_pair(pair_of(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), f2, plus), x, y);
                            if (decltype(masked)::value) {  // not 0, or what a column that is not finite has, times minus infinity
                                x = seen >> i & 1 ? x : -INFINITY;
                                y = seen >> (i + 1) & 1 ? y : -INFINITY;
                            }
                            sum[i >> 1 & 1] = add_pair(sum[i >> 1 & 1], pair_of(exp2_fast(x), exp2_fast(y)));
                        }
                    };
                    uint32_t r[32];
                    const auto load = [&](int c) {
                        tmem_begin32(s_at + 128 * buffer + 32 * c, r);
                        tmem_end32(r);
                        if (c == 0) return;
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        mbar_arrive(&sh.bars[BAR_S_EMPTY + 2 * half + buffer]);  // the buffer is free again
                    };
                    if (all) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            load(c);
                            take(r, c, 0xffffffffu, std::false_type());
                        }
                    } else {
#pragma unroll 1
                        for (int c = 0; c < 2; ++c) {
                            const int32_t at = first + 32 * c, from = min(max(lo - at, 0), 32), to = min(max(hi - at, 0), 32);
                            const uint32_t below = to >= 32 ? 0xffffffffu : (1u << to) - 1, above = from >= 32 ? 0u : 0xffffffffu << from, pages = valid >> (2 * c);
                            load(c);
                            take(r, c, below & above & ((pages & 1 ? 0xffffu : 0u) | (pages & 2 ? 0xffff0000u : 0u)), std::true_type());
                        }
                    }
                }
                // the two threads' sums meet
                float w0, w1, w2, w3;
                of_pair(sum[0], w0, w1);
                of_pair(sum[1], w2, w3);
                float total = (w0 + w1) + (w2 + w3);
                if (side) sh.others[half][units_here & 1][in_tile] = make_float2(top, total);
                ok = half_sync_and(2 + half, ok);
                if (!ok) break;
                if (!side) {
                    const float2 other = sh.others[half][units_here & 1][in_tile];
                    if (!SUMS) {
                        const float high = fmaxf(top, other.x);
                        total = total * exp2_fast(top - high) + other.y * exp2_fast(other.x - high);
                        p.stats_units[(int64_t)unit_at * 256 + 128 * half + in_tile] = make_float2(high, total);
                    } else if (w.part >= 0) {
                        p.parts[(int64_t)w.part * 256 + 128 * half + in_tile] = total + other.y;
                    } else if (own < w.held) {
                        Unit u{};
                        u.seq = w.seq;
                        u.length = w.length;
                        u.rows = w.rows;
                        put_weight(p, u, w.head, own, total + other.y);
                    }
                }
                ++units_here;
            } else {
                ahead = false;
            }
            if (w.step1 > w.step0) {
                ++units;
                tiles += (uint32_t)(w.step1 - w.step0);
            }
        }
    } else if (warp < kIssuerWarp) {
        // ---- keys: from 4 bits to f16 operands ------------------------------------------------------------
        const int thread = threadIdx.x - 32 * kSoftmaxWarps, producer = warp - kSoftmaxWarps;
        Tiles<SUMS> tile;
        tile.begin(p, sh, count);
        for (uint32_t n = 0, units = 0; tile.there(); ++n) {
            const uint32_t turn = n & 1;
            uint32_t scales[B], keys[kKeyGroups][B];
            ok = wait_bounded(&sh.bars[BAR_WORDS_FULL + turn], n >> 1 & 1);
            const uint32_t *const words = reinterpret_cast<const uint32_t *>(words_smem + turn * WORDS_BYTES);
            const uint32_t valid = sh.valid[turn];
            // a token that is none, or not in the pool, has keys of 0
            shared_planes<B, 16>(words + SCALES_AT / 4 + (thread >> 4 & 7) * 16 * B, thread & 15, scales);
            const bool there = (valid >> (thread >> 4 & 7) & 1) && tile.tile() * kTokens + (thread & 127) < tile.w.held;
#pragma unroll
            for (int b = 0; b < B; ++b) scales[b] = there ? key_scale(scales[b]) : 0;
#pragma unroll
            for (int i = 0; i < kKeyGroups; ++i) {
                const int eight = i * kProducerWarps + producer;
                shared_planes<B, 64>(words + (eight >> 1) * 64 * B, (eight & 1) * 32 + (lane & 7) * 4 + (lane >> 3), keys[i]);
            }
            mbar_arrive(&sh.bars[BAR_WORDS_EMPTY + turn]);
            // the largest scale of the tile (bits of bf16 numbers compare like integers; a NaN does not count)
            uint32_t top = 0;
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (scales[b] < 0x7f800000u) top = max(top, scales[b]);
            top = __reduce_max_sync(0xffffffffu, top);
            if (lane == 0) sh.largest[turn][producer] = top;
            ok = half_sync_and(1, ok);
            if (!ok) break;
#pragma unroll
            for (int i = 0; i < kTokens / 32; ++i) top = max(top, sh.largest[turn][i]);
            const int exponent = max((int)(top >> 23) - 127, -100);
            const float by = __uint_as_float((uint32_t)(127 + 11 - exponent) << 23);  // relative scales, below 2^12: 7 of them fit
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (thread < kTokens) sh.scales[turn][thread][b] = __float2half_rn(__uint_as_float(scales[b]) * by);
            // second kernel: a unit's tile i is its half i, whether there is a second one or not
            const uint32_t half = SUMS ? (uint32_t)tile.step : 0, slot = SUMS ? 2 * (units & 1) + half : n & 1;
            uint8_t *const to_tile = (SUMS ? stay_smem : stream_smem) + slot * TILE_BYTES;
            if (SUMS) {
                if (units >= 2 && half == 0) ok = wait_bounded(&sh.bars[BAR_STAY_EMPTY + (units & 1)], (units >> 1 & 1) ^ 1);
            } else if (n >= 2) {
                ok = wait_bounded(&sh.bars[BAR_STREAM_EMPTY + slot], (n >> 1 & 1) ^ 1);
            }
            ok = half_sync_and(1, ok);  // where the place did not get free for one of them, all leave: nothing is written there, and nobody told so
            if (!ok) break;
            if (thread == 0) sh.info[info_place(SUMS, n, units, half)] = TileInfo{__uint_as_float((uint32_t)(127 + exponent) << 23), valid};
#pragma unroll
            for (int i = 0; i < kKeyGroups; ++i) {
                const int eight = i * kProducerWarps + producer, token = eight * 8 + (lane & 7), quarter = lane >> 3;
                uint8_t *const to = to_tile + eight * ROWS8 + quarter * 128 + (lane & 7) * 16;
                const uint2 by_block = *reinterpret_cast<const uint2 *>(sh.scales[turn][token]);
#pragma unroll
                for (int b = 0; b < B; ++b)
                    *reinterpret_cast<uint4 *>(to + b * 512) = decode(keys[i][b], as_half2(__byte_perm(b & 2 ? by_block.y : by_block.x, 0, b & 1 ? 0x3232 : 0x1010)));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (!SUMS) {
                mbar_arrive(&sh.bars[BAR_STREAM_FULL + slot]);
            } else if (tile.last()) {
                mbar_arrive(&sh.bars[BAR_STAY_FULL + (units & 1)]);
                ++units;
            }
            tile.next(p, sh);
        }
    } else {
        if (warp == kIssuerWarp) {
            // ---- the products ---------------------------------------------------------------------------------
            constexpr uint32_t kIdesc = 1u << 4 | (uint32_t)(128 >> 4) << 24 | (uint32_t)(128 >> 3) << 17;  // fp32 sums of f16 products, both operands along k, 128 x 128
            const uint32_t stay_at = smem_u32(stay_smem), stream_at = smem_u32(stream_smem);
            uint32_t units = 0, streamed = 0, steps[2] = {0, 0};
            const auto read_out = [&](int half, uint32_t step) { return warp_wait(&sh.bars[BAR_S_EMPTY + 2 * half + step_buffer(step)], step_parity(step)); };
            for (int32_t unit_at = blockIdx.x, k = 0; ok && unit_at < count; unit_at += gridDim.x, ++k) {
                const WorkUnit w = load_unit<SUMS>(p, sh, k, unit_at);
                if (w.step0 == w.step1) continue;
                const uint32_t pair = units & 1;
                const int halves = halves_of<SUMS>(w);
                ok = before_unit(halves, steps, read_out) && warp_wait(&sh.bars[BAR_STAY_FULL + pair], units >> 1 & 1);
                for (int32_t step = w.step0; ok && step < w.step1; ++step, ++streamed) {
                    const uint32_t slot = streamed & 1;
                    ok = warp_wait(&sh.bars[BAR_STREAM_FULL + slot], streamed >> 1 & 1);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if (!ok || half >= halves) break;
                        const uint32_t buffer = step_buffer(steps[half]);
                        ok = before_step(half, steps, read_out);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        if (lane == 0) {
#pragma unroll
                            for (int k = 0; k < 2 * B; ++k)
                                mma_shared(tmem + 256 * half + 128 * buffer, operand(stay_at + (2 * pair + half) * TILE_BYTES + k * 256, ROWS8),
                                           operand(stream_at + slot * TILE_BYTES + k * 256, ROWS8), kIdesc, k > 0);
                            mma_commit(&sh.bars[BAR_S_FULL + 2 * half + buffer]);
                        }
                        __syncwarp();
                        ++steps[half];
                    }
                    if (ok && lane == 0) mma_commit(&sh.bars[BAR_STREAM_EMPTY + slot]);
                    __syncwarp();
                }
                if (ok && lane == 0) mma_commit(&sh.bars[BAR_STAY_EMPTY + pair]);
                __syncwarp();
                ++units;
            }
            // whatever happened: nothing is in flight when the tensor memory goes
            if (lane == 0) mma_commit(&sh.bars[BAR_DONE]);
            __syncwarp();
            if (!wait_bounded(&sh.bars[BAR_DONE], 0)) ok = false;
        } else if (warp == kWordsWarp) {
            // ---- the keys' words to shared memory: a lane to a tile of the cache -------------------------------
            Tiles<SUMS> tile;
            tile.begin(p, sh, count);
            const int32_t tiles_per_page = p.g.page_size / kKvTile;
            const auto find = [&]() { return tile.there() ? find_page(p, p.page_table + (int64_t)tile.w.seq * p.table_pages, tile.w.held, tile.tile(), lane) : -1; };
            int32_t page = find();  // a tile ahead
            uint32_t n = 0;
            for (; tile.there(); ++n) {
                const uint32_t slot = n & 1;
                const int32_t place = page >= 0 && page < p.g.pages ? (page * p.g.heads + tile.w.head) * tiles_per_page + (tile.tile() * 8 + lane) % tiles_per_page : -1;
                tile.next(p, sh);
                page = find();
                if (n >= 2) ok = warp_wait(&sh.bars[BAR_WORDS_EMPTY + slot], (n >> 1 & 1) ^ 1);
                if (!ok) break;
                const uint32_t valid = __ballot_sync(0xffffffffu, place >= 0);
                uint64_t *const bar = &sh.bars[BAR_WORDS_FULL + slot];
                if (lane == 0) {
                    sh.valid[slot] = valid;
                    mbar_expect_tx(bar, __popc(valid) * 320 * B);
                }
                __syncwarp();
                if (place >= 0) {
                    uint8_t *const to = words_smem + slot * WORDS_BYTES;
                    const uint32_t *const from = p.cache + (int64_t)place * kv_tile_words(B);
                    bulk_copy_g2s(to + lane * 256 * B, from, 256 * B, bar);
                    bulk_copy_g2s(to + SCALES_AT + lane * 64 * B, from + 128 * B, 64 * B, bar);
                }
            }
            // whatever happened: no copy is in flight when the block ends
            for (uint32_t i = n < 2 ? 0 : n - 2; i < n; ++i)
                if (!wait_bounded(&sh.bars[BAR_WORDS_FULL + (i & 1)], i >> 1 & 1)) ok = false;
        } else {
            // ---- rows of q: images to shared memory -------------------------------------------------------------
            uint32_t units = 0, streamed = 0;
            for (int32_t unit_at = blockIdx.x, k = 0; ok && unit_at < count; unit_at += gridDim.x, ++k) {
                const WorkUnit w = load_unit<SUMS>(p, sh, k, unit_at);
                const auto copy = [&](uint8_t *to, int32_t tile, uint64_t *bar) { bulk_copy_g2s(to, p.images + image_of(p, w, tile) * TILE_BYTES, TILE_BYTES, bar); };
                if (w.step0 == w.step1) continue;
                if (!SUMS) {
                    const uint32_t pair = units & 1;
                    if (units >= 2) ok = warp_wait(&sh.bars[BAR_STAY_EMPTY + pair], (units >> 1 & 1) ^ 1);
                    if (!ok) break;
                    if (lane == 0) {
                        const int halves = halves_of<SUMS>(w);
                        mbar_expect_tx(&sh.bars[BAR_STAY_FULL + pair], halves * TILE_BYTES);
                        for (int half = 0; half < halves; ++half) copy(stay_smem + (2 * pair + half) * TILE_BYTES, w.first / 128 + half, &sh.bars[BAR_STAY_FULL + pair]);
                    }
                    __syncwarp();
                    ++units;
                } else {
                    for (int32_t step = w.step0; step < w.step1; ++step, ++streamed) {
                        const uint32_t slot = streamed & 1;
                        if (streamed >= 2) ok = warp_wait(&sh.bars[BAR_STREAM_EMPTY + slot], (streamed >> 1 & 1) ^ 1);
                        if (!ok) break;
                        if (lane == 0) {
                            mbar_expect_tx(&sh.bars[BAR_STREAM_FULL + slot], TILE_BYTES);
                            copy(stream_smem + slot * TILE_BYTES, step, &sh.bars[BAR_STREAM_FULL + slot]);
                        }
                        __syncwarp();
                    }
                }
            }
            // whatever happened: no copy is in flight when the block ends
            const uint32_t copied = SUMS ? streamed : units;
            for (uint32_t i = copied < 2 ? 0 : copied - 2; i < copied; ++i)
                if (!wait_bounded(&sh.bars[(SUMS ? BAR_STREAM_FULL : BAR_STAY_FULL) + (i & 1)], i >> 1 & 1)) ok = false;
        }
    }
    if (!ok) {
        *report.device_word = 1;
        if (report.host_word) {
            *reinterpret_cast<volatile int *>(report.host_word) = 1;
            __threadfence_system();
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == kIssuerWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// The pieces' sums of a column joined, always in the same order: eight threads to a column, a block to 128.
constexpr int kJoining = 8;

__global__ void __launch_bounds__(kJoining * kTokens) kv_weights_columns_kernel(const __grid_constant__ PromptParams p)
{
    __shared__ float2 parts[kJoining][kTokens];
    Counts before;
    const Cut cut = find_cut(p);
    // the lengths are what the kernels in front read: nothing has written them since
    const int seq = find_sequence(p, cut, blockIdx.x, [](const Counts &c) { return c.tiles; }, &before), head = blockIdx.y;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the ones in front, too
    if (seq < 0 || p.unit_counts[0] == 0) return;
    const Sequence s = sequence<8>(p, seq);
    const int in_tile = threadIdx.x % kTokens, part = threadIdx.x / kTokens;
    const int tile = blockIdx.x - before.tiles, columns = s.rows * p.group, pieces = up(up(tokens_held(p, s.length), kTokens), cut.first);
    const auto add = [](float2 &sum, const float2 &other) {  // relative to their largest
        const float high = fmaxf(sum.x, other.x);
        sum = make_float2(high, sum.y * exp2_fast(sum.x - high) + other.y * exp2_fast(other.x - high));
    };
    float2 sum = make_float2(kNothing, 0.0f);
    if (tile * 128 + in_tile < columns) {
        const float2 *const from = p.stats_units + (before.units[0] + (int64_t)(head * up(columns, 256) + tile / 2) * pieces) * 256 + (tile & 1) * 128 + in_tile;
#pragma unroll 4
        for (int i = part; i < pieces; i += kJoining) add(sum, from[(int64_t)i * 256]);
    }
    parts[part][in_tile] = sum;
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int i = 1; i < kJoining; ++i) add(sum, parts[i][in_tile]);
    const int64_t at = ((int64_t)blockIdx.x * p.g.heads + head) * kTokens + in_tile;
    // nothing of a column that is none, or sees nothing
    p.constants[at] = sum.y == 0.0f ? -INFINITY : -(sum.x + log2f(sum.y));
}

// The chunks' weights of a token added up, always in the same order; a block to 256 tokens at a time.
__global__ void __launch_bounds__(256) kv_weights_chunks_kernel(const __grid_constant__ PromptParams p)
{
    const Cut cut = find_cut(p);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the ones in front, too
    if (p.unit_counts[1] == 0) return;
    for (int at = blockIdx.x;; at += gridDim.x) {
        Counts before;
        const int seq = find_sequence(p, cut, at, [](const Counts &c) { return c.parts; }, &before);
        if (seq < 0) return;
        const Sequence s = sequence<8>(p, seq);
        const int held = tokens_held(p, s.length), outer = up(held, 256), chunks = up(up(s.rows * p.group, 128), cut.second);
        const int local = at - before.parts, of_outer = local / chunks, head = of_outer / outer, t = (of_outer - head * outer) * 256 + threadIdx.x;
        if (local == of_outer * chunks && t < held) {  // the first of 256 tokens' chunks stands for them all
            const float *const from = p.parts + (int64_t)at * 256 + threadIdx.x;
            float w = 0.0f;
#pragma unroll 4
            for (int i = 0; i < chunks; ++i) w += from[(int64_t)i * 256];
            Unit u{};
            u.seq = seq;
            u.length = s.length;
            u.rows = s.rows;
            put_weight(p, u, head, t, w);
        }
    }
}

// Tiles of columns, units and parts that there can be.
struct Bounds {
    int64_t tiles, units, second_units, parts;
};
Bounds bounds(const WeightsParams &p)
{
    // at most kSteps units by the cut, and one more for every 256 columns, or tokens, of a head; parts: the chunks are at most twice the steps by the cut
    const int64_t columns = p.tokens * p.group;
    const int64_t tokens = (int64_t)p.batch * ((p.table_tokens + 255) / 256);
    return {columns / 128 + p.batch, kSteps + p.g.heads * (columns / 256 + p.batch), kSteps + p.g.heads * tokens, 2 * kSteps};
}

int64_t rounded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

template <int B>
lce_status launch(PromptParams &p, const TimeoutReport &report, cudaStream_t s)
{
    static SmemOptIn first_opt_in, second_opt_in;
    if (!first_opt_in.ensure(kv_weights_prompt_kernel<B, false>, weights_smem(B)) || !second_opt_in.ensure(kv_weights_prompt_kernel<B, true>, weights_smem(B))) return LCE_ERR_CUDA;
    const Bounds most = bounds(p);
    const dim3 tiles((unsigned)most.tiles, (unsigned)p.g.heads);
    lce_status st = launch_dependent(kv_weights_rows_kernel<B>, dim3(tiles.x, tiles.y + 1), kRowsThreads, 0, s, p);
    if (st == LCE_OK) st = launch_dependent(kv_weights_prompt_kernel<B, false>, dim3(kBlocks), kThreads, weights_smem(B), s, p, report);
    if (st == LCE_OK) st = launch_dependent(kv_weights_columns_kernel, tiles, kJoining * kTokens, 0, s, p);
    if (st == LCE_OK) st = launch_dependent(kv_weights_prompt_kernel<B, true>, dim3(kBlocks), kThreads, weights_smem(B), s, p, report);
    if (st == LCE_OK) st = launch_dependent(kv_weights_chunks_kernel, dim3(4 * kBlocks), 256, 0, s, p);
    return st;
}

}  // namespace

size_t kv_weights_prompt_bytes(const WeightsParams &p)
{
    const Bounds most = bounds(p);
    const int64_t columns = most.tiles * p.g.heads * kTokens;
    return (size_t)(rounded(most.units * sizeof(WorkUnit)) + rounded(most.second_units * sizeof(WorkUnit)) + rounded(8) + rounded(columns * 64 * p.g.blocks) + rounded(columns * 4) + rounded(columns / kTokens * 4) + rounded(columns * 4) + rounded(most.units * 256 * 8) + rounded(most.parts * 256 * 4));
}

lce_status launch_kv_weights_prompt(const WeightsParams &params, void *workspace, cudaStream_t s)
{
    if (tensor_timeout_flagged()) return LCE_ERR_DEVICE_TIMEOUT;
    const TimeoutReport report = tensor_timeout_report(s);
    if (!report.device_word) return LCE_ERR_CUDA;
    PromptParams p{};
    static_cast<WeightsParams &>(p) = params;
    const Bounds most = bounds(p);
    const int64_t columns = most.tiles * p.g.heads * kTokens;
    p.most_tiles = (int32_t)most.tiles;
    p.most_units[0] = (int32_t)most.units;
    p.most_units[1] = (int32_t)most.second_units;
    p.most_parts = (int32_t)most.parts;
    char *at = static_cast<char *>(workspace);
    const auto take = [&](int64_t bytes) {
        char *const here = at;
        at += rounded(bytes);
        return here;
    };
    p.units[0] = reinterpret_cast<WorkUnit *>(take(most.units * sizeof(WorkUnit)));
    p.units[1] = reinterpret_cast<WorkUnit *>(take(most.second_units * sizeof(WorkUnit)));
    p.unit_counts = reinterpret_cast<int32_t *>(take(8));
    p.images = reinterpret_cast<uint8_t *>(take(columns * 64 * p.g.blocks));
    p.factors = reinterpret_cast<float *>(take(columns * 4));
    p.tile_factors = reinterpret_cast<float *>(take(columns / kTokens * 4));
    p.constants = reinterpret_cast<float *>(take(columns * 4));
    p.stats_units = reinterpret_cast<float2 *>(take(most.units * 256 * 8));
    p.parts = reinterpret_cast<float *>(take(most.parts * 256 * 4));
    switch (p.g.blocks) {
        case 1: return launch<1>(p, report, s);
        case 2: return launch<2>(p, report, s);
        case 3: return launch<3>(p, report, s);
        default: return launch<4>(p, report, s);
    }
}

}  // namespace lce
