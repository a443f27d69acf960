// Attention weights by token of many rows (a prompt, or its last rows), on the 5th-generation tensor cores.
//
// The softmax needs a column's largest score and sum before its first weight is known, so the scores are made twice, by two kernels of one
// shape: 256 rows of one operand stay in shared memory, tiles of 128 rows of the other one stream past them, and every thread of eight warps
// has one of the 256 in TMEM, with its 128 products a step.
//   first     256 columns (rows of q that share a key/value head) stay, keys stream: a thread has a column's scores, and keeps their
//             largest and the sum of their powers of two
//   second    256 tokens stay, columns stream: a thread has a token's scores, and adds its weights up.  A column's factor and the logarithm of
//             its sum lie in shared memory
// So no sum crosses threads.  Work is cut into units of a few steps: (256 columns, a piece of the sequence) and (256 tokens, a chunk of the
// columns), joined in a fixed order by small kernels; 148 blocks take equal runs of units, and their warps go from one to the next
// without meeting:
//   warps 0 - 3, 4 - 7  the powers of two, 128 of the 256 each; two accumulators of 128 x 128 for each in TMEM
//   warps 8 - 11        4-bit words from the cache to f16 keys in shared memory
//   warp 12             issues the products
//   warp 13             has rows of q copied, which a kernel in front has put in order as f16
//
// f16 holds a code times its scale exactly, relative to the largest scale of 128 tokens, down to 2^-28 of it; 16-bit rows of q are exact
// down to 2^-24 of their largest element at least.  Scores and sums are fp32.
#include "kv_tensor.cuh"
#include "kv_weights.cuh"

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

constexpr int kSoftmaxWarps = 8, kProducerWarps = 4, kIssuerWarp = kSoftmaxWarps + kProducerWarps, kCopyWarp = kIssuerWarp + 1;
constexpr int kThreads = 32 * (kIssuerWarp + 4);  // whole warpgroups: registers are shared out between them
// Registers a thread: 128 at the launch, 512 * 128 in all = 256 * 144 + 128 * 112 + 128 * 112.
constexpr int kSoftmaxRegisters = 144, kProducerRegisters = 112, kIssuerRegisters = 112;
static_assert(256 * kSoftmaxRegisters + 128 * kProducerRegisters + 128 * kIssuerRegisters <= kThreads * 128, "more registers than the block has");
constexpr float kNothing = -3e38f;   // stands for the largest score where there is none
constexpr float kRise = 16.0f;       // the score that powers of two are relative to is raised when one passes it by this much
constexpr int kBlocks = 148;         // one to an SM
constexpr int kSteps = kBlocks * 8;  // units are cut so that there are about as many
constexpr int kInfos = 8;            // tiles of keys; the producers are less than four units, of two tiles, ahead of the softmax

enum { BAR_STAY_FULL = 0, BAR_STAY_EMPTY = BAR_STAY_FULL + 2, BAR_STREAM_FULL = BAR_STAY_EMPTY + 2, BAR_STREAM_EMPTY = BAR_STREAM_FULL + 2,
       BAR_S_FULL = BAR_STREAM_EMPTY + 2, BAR_S_EMPTY = BAR_S_FULL + 4, BAR_DONE = BAR_S_EMPTY + 4, BAR_COUNT };

struct TileInfo {
    float unit;      // 2^e: scores count in it
    uint32_t valid;  // bit per 16 tokens: their page is in the pool
};

struct Shared {
    uint64_t bars[BAR_COUNT];
    uint32_t tmem, largest[2][kProducerWarps];
    TileInfo info[kInfos];
    alignas(16) __half scales[2][kTokens][4];         // relative to the tile's largest; [turn]
    alignas(16) float columns[2][2][kTokens / 2][4];  // [half][turn][pair]: two factors, two logarithms taken off
};

constexpr int kMiscBytes = 8192;
static_assert(sizeof(Shared) <= kMiscBytes, "");
constexpr size_t weights_smem(int blocks) { return kMiscBytes + 6 * (size_t)(kTokens * 64 * blocks); }

struct PromptParams : WeightsParams {
    uint8_t *images;      // [tile of 128 columns][kv head]: rows of q as f16, in the order in which they are an operand
    float *factors;       // [tile of columns][kv head][128]
    float2 *stats_units;  // [unit of the first kernel][256]: largest, sum
    float2 *constants;    // [tile of columns][kv head][128]: factor, less the logarithm of the sum
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

// Finds the sequence that the `at`-th of what `count` counts belongs to, and what the sequences in front of it have; at < 0: all sequences'.
// By whole warps.
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
        const uint32_t has = __ballot_sync(0xffffffffu, at >= 0 && count(*before) + count(upto) > at);
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

// The unit that a role works on, of the first kernel (SUMS false) or the second.
template <bool SUMS>
struct Work {
    Cut cut;
    Counts before;     // the sequences in front
    int32_t unit, end; // this and one past the block's last
    Unit u;
    int32_t held, columns, outer, inner;  // of the sequence: tokens, columns; 256 of what stays there are; pieces or chunks
    int32_t head, o, i;
    int32_t step0, step1;

    __device__ __forceinline__ void take_sequence(const PromptParams &p, int b)
    {
        const Sequence s = sequence<8>(p, b);
        u.seq = b;
        u.length = s.length;
        u.rows = s.rows;
        u.row0 = s.row0;
        held = tokens_held(p, s.length);
        columns = s.rows * p.group;
        outer = SUMS ? up(held, 256) : up(columns, 256);
        inner = SUMS ? max(up(up(columns, 128), cut.second), 1) : up(up(held, kTokens), cut.first);
    }
    // Columns [lo, hi) that see some of tokens [t0, t1): their ranges move up with the rows, so they are a run.
    __device__ __forceinline__ void columns_of(const PromptParams &p, int32_t t0, int32_t t1, int32_t *lo, int32_t *hi) const
    {
        const int64_t row0 = (int64_t)u.length - u.rows;  // position of the first row
        *lo = p.causal ? (int32_t)(min(max(t0 - row0, (int64_t)0), (int64_t)u.rows) * p.group) : 0;
        *hi = p.window > 0 ? (int32_t)(min(max(t1 - 1 + p.window - row0, (int64_t)0), (int64_t)u.rows) * p.group) : columns;
    }
    __device__ __forceinline__ void find_steps(const PromptParams &p)
    {
        int32_t lo, hi, unused;
        if (SUMS) {
            columns_of(p, 256 * o, min(256 * o + 256, held), &lo, &hi);
        } else {
            column_range(p, u, 256 * o, &lo, &unused);
            column_range(p, u, min(256 * o + 256, columns) - 1, &unused, &hi);
        }
        const int32_t each = SUMS ? cut.second : cut.first;
        step0 = max(lo / 128, i * each);
        step1 = hi > lo ? min(up(hi, 128), (int32_t)min((int64_t)(i + 1) * each, (int64_t)0x7fffffff)) : step0;
        step1 = max(step1, step0);
    }
    // The block's first unit; false: there is none.  By whole warps.
    __device__ __forceinline__ bool begin(const PromptParams &p)
    {
        cut = find_cut(p);
        const auto count = [](const Counts &c) { return c.units[SUMS]; };
        find_sequence(p, cut, -1, count, &before);
        const int64_t total = before.units[SUMS];
        unit = (int32_t)(total * blockIdx.x / gridDim.x);
        end = (int32_t)(total * (blockIdx.x + 1) / gridDim.x);
        if (unit >= end) return false;
        const int b = find_sequence(p, cut, unit, count, &before);
        take_sequence(p, b);
        const int32_t local = unit - before.units[SUMS], of_outer = local / inner;
        i = local - of_outer * inner;
        head = of_outer / outer;
        o = of_outer - head * outer;
        find_steps(p);
        return true;
    }
    __device__ __forceinline__ bool next(const PromptParams &p)
    {
        if (++unit >= end) return false;
        if (++i == inner) {
            i = 0;
            if (++o == outer) {
                o = 0;
                if (++head == p.g.heads) {
                    head = 0;
                    do {  // there is one: units are left
                        const Counts c = counts(p, sequence<8>(p, u.seq), cut);
                        before.tiles += c.tiles;
                        before.units[0] += c.units[0];
                        before.units[1] += c.units[1];
                        before.parts += c.parts;
                        take_sequence(p, u.seq + 1);
                    } while (u.seq + 1 < p.batch && (held == 0 || (!SUMS && columns == 0)));
                }
            }
        }
        find_steps(p);
        return true;
    }
    // Whether the second half of what stays exists.
    __device__ __forceinline__ int halves() const { return 256 * o + 128 < (SUMS ? held : columns) ? 2 : 1; }
    __device__ __forceinline__ int64_t image(const PromptParams &p, int32_t tile) const { return (int64_t)(before.tiles + tile) * p.g.heads + head; }
};

// Rows of q as f16 operands and what their scores are multiplied with: a thread to a row, a block to 128 columns.
template <int B>
__global__ void __launch_bounds__(kTokens) kv_weights_rows_kernel(const __grid_constant__ PromptParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int ROWS8 = 512 * B;
    Counts before;
    const Cut cut{1, 1};
    const int seq = find_sequence(p, cut, blockIdx.x, [](const Counts &c) { return c.tiles; }, &before), head = blockIdx.y;
    if (seq < 0) return;
    const Sequence s = sequence<8>(p, seq);
    const int column = (blockIdx.x - before.tiles) * 128 + threadIdx.x, row = column / p.group;
    const int64_t at = (s.row0 + row) * p.q_token + ((int64_t)head * p.group + (column - row * p.group)) * p.q_head, image = (int64_t)blockIdx.x * p.g.heads + head;
    uint8_t *const to = p.images + image * (kTokens * 64 * B) + (threadIdx.x >> 3) * ROWS8 + (threadIdx.x & 7) * 16;
    int k = 0;
    bool finite = true;
    const auto take_row = [&](auto element, auto vectors) {
        using T = decltype(element);
        Eight<T> e[4 * B];  // the whole row at once
#pragma unroll
        for (int c = 0; c < 4 * B; ++c) e[c] = load_eight<T, decltype(vectors)::value>(static_cast<const T *>(p.q) + at + 8 * c, row < s.rows ? p.g.dim - 8 * c : 0);
        uint32_t magnitude = 0;  // magnitudes compare like integers, infinity and NaN above all others
        float v[8];
#pragma unroll
        for (int c = 0; c < 4 * B; ++c) {
            e[c].expand(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) magnitude = max(magnitude, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        finite = magnitude < 0x7f800000u;
        // times 2^k, so that the largest is in [2^14, 2^15); a scale below zero changes q's sign
        k = 14 - (finite && magnitude > 0 ? ilogbf(__uint_as_float(magnitude)) : 0);
        const int k1 = k / 2, k2 = k - k1;
        const float s1 = __uint_as_float((uint32_t)(127 + k1) << 23) * (p.scale < 0.0f ? -1.0f : 1.0f), s2 = __uint_as_float((uint32_t)(127 + k2) << 23);
#pragma unroll
        for (int c = 0; c < 4 * B; ++c) {
            e[c].expand(v);
            // in the order in which a word's codes are decoded; a row that is not finite is one by its factor
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = finite ? v[i] * s1 * s2 : 0.0f;
            *reinterpret_cast<uint4 *>(to + c * 128) = make_uint4(pack_half2(v[0], v[4]), pack_half2(v[1], v[5]), pack_half2(v[2], v[6]), pack_half2(v[3], v[7]));
        }
    };
    if (p.type == LCE_TYPE_FLOAT16) {
        if (p.q_vectors) take_row(__half(), std::true_type());
        else take_row(__half(), std::false_type());
    } else {
        if (p.q_vectors) take_row(__nv_bfloat16(), std::true_type());
        else take_row(__nv_bfloat16(), std::false_type());
    }
    const int kc = -11 - k, c1 = kc / 2, c2 = kc - c1;
    p.factors[image * kTokens + threadIdx.x] =
        (finite ? fabsf(p.scale) : __uint_as_float(0x7fc00000u)) * __uint_as_float((uint32_t)(127 + c1) << 23) * __uint_as_float((uint32_t)(127 + c2) << 23);
}

// What a producer thread has of a tile before it decodes it.
template <int B>
struct Raw {
    uint32_t scales[B];  // of its token
    uint32_t keys[4][B];
    uint32_t valid;
};

template <int B>
__device__ __forceinline__ void load_raw(const PromptParams &p, int32_t page, int head, int held, int tile, int thread, Raw<B> &r)
{
    constexpr int TILE = kv_tile_words(B);
    const int lane = thread & 31, warp = thread >> 5, tiles_per_page = p.g.page_size / kKvTile;
    const int32_t place = page >= 0 && page < p.g.pages ? (page * p.g.heads + head) * tiles_per_page + (tile * 8 + lane) % tiles_per_page : -1;
    r.valid = __ballot_sync(0xffffffffu, place >= 0);
    const auto tile_at = [&](int t) -> const uint32_t * {
        const int32_t at = __shfl_sync(0xffffffffu, place, t);
        return at >= 0 ? p.cache + (int64_t)at * TILE : nullptr;
    };
#pragma unroll
    for (int b = 0; b < B; ++b) r.scales[b] = 0;
    {
        const uint32_t *const at = tile_at(thread >> 4);
        if (at && tile * kTokens + thread < held) load_planes<B, 16>(at + 128 * B, thread & 15, r.scales);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int half = i * 4 + warp;
        const uint32_t *const at = tile_at(half >> 1);
#pragma unroll
        for (int b = 0; b < B; ++b) r.keys[i][b] = 0;
        if (at) load_planes<B, 64>(at, (half & 1) * 32 + (lane & 7) * 4 + (lane >> 3), r.keys[i]);
    }
}

// A wait of a whole warp.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bounded(bar, parity)); }
// Four warps meet; whether all of them are well.
__device__ __forceinline__ bool half_sync_and(uint32_t barrier, bool ok)
{
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
        "bar.red.and.pred p, %2, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)ok), "r"(barrier)
        : "memory");
    return all != 0;
}

// The tiles of keys that a block's units want, one after the other.
template <bool SUMS>
struct Tiles {
    Work<SUMS> w;
    int32_t step;   // of the unit, or the half
    bool there;
    __device__ __forceinline__ void begin(const PromptParams &p, const Work<SUMS> &first)
    {
        w = first;
        there = true;
        settle(p);
    }
    __device__ __forceinline__ void settle(const PromptParams &p)  // at the first tile of a unit that has one
    {
        while (there && w.step0 == w.step1) there = w.next(p);
        step = SUMS ? 0 : w.step0;
    }
    __device__ __forceinline__ int32_t tile() const { return SUMS ? 2 * w.o + step : step; }
    __device__ __forceinline__ void next(const PromptParams &p)
    {
        if (++step < (SUMS ? w.halves() : w.step1)) return;
        there = w.next(p);
        settle(p);
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
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Work<SUMS> work;
    if (!work.begin(p)) return;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.bars[BAR_STAY_FULL + i], SUMS ? 32 * kProducerWarps : 1);
            mbar_init(&sh.bars[BAR_STAY_EMPTY + i], 1);
            mbar_init(&sh.bars[BAR_STREAM_FULL + i], SUMS ? 1 : 32 * kProducerWarps);
            mbar_init(&sh.bars[BAR_STREAM_EMPTY + i], 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&sh.bars[BAR_S_FULL + i], 1);
            mbar_init(&sh.bars[BAR_S_EMPTY + i], 128);
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
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegisters));
        // ---- powers of two: a thread to a column, or to a token ---------------------------------------
        const int half = warp >> 2, in_tile = threadIdx.x & 127;
        const uint32_t s_at = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 256 * half;
        uint32_t steps = 0, units = 0, tiles = 0;  // steps of this half, units that have some, tiles of keys in front of the unit's
        bool more = true;
        while (ok && more) {
            const bool here = half < work.halves();
            const int32_t own = 256 * work.o + 128 * half + in_tile;
            int32_t lo = 0, hi = 0;  // what it sees: of the tokens, or of the columns
            float factor = 0.0f, top = kNothing;
            uint64_t sum[2] = {};  // pairs of fp32 sums
            if (here) {
                if (SUMS) {
                    if (own < work.held) work.columns_of(p, own, own + 1, &lo, &hi);
                } else {
                    column_range(p, work.u, own, &lo, &hi);
                    if (work.step1 > work.step0) factor = p.factors[work.image(p, 2 * work.o + half) * kTokens + in_tile];
                }
            }
            float2 constant = make_float2(0.0f, 0.0f);  // of a column of the next step
            if (SUMS && here && work.step1 > work.step0) constant = p.constants[work.image(p, work.step0) * kTokens + in_tile];
            float unit = 0.0f;
            for (int32_t step = work.step0; ok && here && step < work.step1; ++step, ++steps) {
                const uint32_t buffer = steps & 1;
                ok = warp_wait(&sh.bars[BAR_S_FULL + 2 * half + buffer], steps >> 1 & 1);
                if (!SUMS && !ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const int first = step * 128;  // token, or column
                uint32_t valid = 0xffu;
                if (!SUMS || step == work.step0) {
                    const TileInfo info = sh.info[(SUMS ? 2 * units + half : tiles + (uint32_t)(step - work.step0)) % kInfos];
                    unit = info.unit;
                    if (SUMS) {
                        if (!(info.valid >> (in_tile >> 4) & 1)) hi = lo;  // its page is not in the pool
                    } else {
                        valid = info.valid;
                    }
                }
                if (SUMS) {
                    // every thread brings a column's constants; the buffer before last is read by nobody any more
                    float *const pair = sh.columns[half][buffer][in_tile >> 1] + (in_tile & 1);
                    pair[0] = constant.x * unit;
                    pair[2] = constant.y;
                    if (step + 1 < work.step1) constant = p.constants[work.image(p, step + 1) * kTokens + in_tile];
                    ok = half_sync_and(2 + half, ok);  // all four warps leave together
                    if (!ok) break;
                }
                const bool all = __all_sync(0xffffffffu, valid == 0xffu && first >= lo && first + 128 <= hi);
                const float f = factor * unit;
                // 64 of the 128 at a time
#pragma unroll 1
                for (int c0 = 0; c0 < 128; c0 += 64) {
                    uint32_t r[64];
                    tmem_load64(s_at + 128 * buffer + c0, r);
                    if (c0 == 64) {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        mbar_arrive(&sh.bars[BAR_S_EMPTY + 2 * half + buffer]);
                    }
                    if (!all) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int32_t at = first + c0 + 32 * c, from = min(max(lo - at, 0), 32), to = min(max(hi - at, 0), 32);
                            const uint32_t below = to >= 32 ? 0xffffffffu : (1u << to) - 1, above = from >= 32 ? 0u : 0xffffffffu << from;
                            const uint32_t pages = valid >> ((c0 >> 4) + 2 * c);
                            const uint32_t seen = below & above & ((pages & 1 ? 0xffffu : 0u) | (pages & 2 ? 0xffff0000u : 0u));
#pragma unroll
                            for (int i = 0; i < 32; ++i) r[32 * c + i] = seen >> i & 1 ? r[32 * c + i] : 0xff800000u;
                        }
                    }
                    uint64_t f2 = pair_of(f, f), plus = 0;
                    if (!SUMS) {
                        float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int i = 0; i < 64; ++i) tops[i & 3] = fmaxf(tops[i & 3], __uint_as_float(r[i]));
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
                    for (int i = 0; i < 64; i += 2) {
                        if (SUMS) {
                            const ulonglong2 c = *reinterpret_cast<const ulonglong2 *>(sh.columns[half][buffer][(c0 + i) >> 1]);
                            f2 = c.x;
                            plus = c.y;
                        }
                        float x, y;
                        of_pair(fma_pair(pair_of(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), f2, plus), x, y);
                        if (!all) {  // 0, or what a column that is not finite has, times minus infinity
                            x = r[i] == 0xff800000u ? -INFINITY : x;
                            y = r[i + 1] == 0xff800000u ? -INFINITY : y;
                        }
                        sum[i >> 1 & 1] = add_pair(sum[i >> 1 & 1], pair_of(exp2_fast(x), exp2_fast(y)));
                    }
                }
            }
            if (!ok) break;
            float w0, w1, w2, w3;
            of_pair(sum[0], w0, w1);
            of_pair(sum[1], w2, w3);
            const float total = (w0 + w1) + (w2 + w3);
            if (!SUMS) {
                p.stats_units[(int64_t)work.unit * 256 + 128 * half + in_tile] = make_float2(top, total);
            } else if (own < work.held) {
                if (work.inner > 1) p.parts[(int64_t)(work.before.parts + work.unit - work.before.units[1]) * 256 + 128 * half + in_tile] = total;
                else put_weight(p, work.u, work.head, own, total);
            }
            if (work.step1 > work.step0) {
                ++units;
                tiles += (uint32_t)(work.step1 - work.step0);
            }
            more = work.next(p);
        }
    } else if (warp < kIssuerWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProducerRegisters));
        // ---- keys: from 4 bits to f16 operands ------------------------------------------------------------
        const int thread = threadIdx.x - 32 * kSoftmaxWarps, producer = warp - kSoftmaxWarps;
        Tiles<SUMS> ahead;  // the tile behind the one whose words are on their way
        ahead.begin(p, work);
        struct Tile {
            bool there;
            uint32_t half;  // of a unit; whether it is the last one
            bool last;
        };
        Raw<B> even_raw, odd_raw;
        Tile even{}, odd{};
        int32_t page = -1;
        const auto find = [&]() { page = ahead.there ? find_page(p, p.page_table + (int64_t)ahead.w.u.seq * p.table_pages, ahead.w.held, ahead.tile(), lane) : -1; };
        const auto load = [&](Raw<B> &raw, Tile &tile) {
            tile.there = ahead.there;
            if (!ahead.there) return;
            tile.half = SUMS ? (uint32_t)ahead.step : 0;
            tile.last = SUMS && ahead.step + 1 == ahead.w.halves();
            load_raw<B>(p, page, ahead.w.head, ahead.w.held, ahead.tile(), thread, raw);
            ahead.next(p);
            find();
        };
        find();
        load(even_raw, even);
        uint32_t n = 0, units = 0;
        const auto produce = [&](const Raw<B> &raw, const Tile &tile, Raw<B> &next_raw, Tile &next) -> bool {
            load(next_raw, next);
            // the largest scale of the tile (bits of bf16 numbers compare like integers; a NaN does not count)
            const int turn = n & 1;
            uint32_t top = 0;
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const uint32_t s = key_scale(raw.scales[b]);
                if (s < 0x7f800000u) top = max(top, s);
            }
            top = __reduce_max_sync(0xffffffffu, top);
            if (lane == 0) sh.largest[turn][producer] = top;
            ok = producers_sync_and(ok);
            if (!ok) return false;
#pragma unroll
            for (int i = 0; i < kProducerWarps; ++i) top = max(top, sh.largest[turn][i]);
            const int exponent = max((int)(top >> 23) - 127, -100);
            const float by = __uint_as_float((uint32_t)(127 + 11 - exponent) << 23);  // relative scales, below 2^12: 7 of them fit
#pragma unroll
            for (int b = 0; b < B; ++b) sh.scales[turn][thread][b] = __float2half_rn(__uint_as_float(key_scale(raw.scales[b])) * by);
            // second kernel: a unit's tile i is its half i, whether there is a second one or not
            const uint32_t slot = SUMS ? 2 * (units & 1) + tile.half : n & 1;
            uint8_t *const to_tile = (SUMS ? stay_smem : stream_smem) + slot * TILE_BYTES;
            if (SUMS) {
                if (units >= 2 && tile.half == 0) ok = wait_bounded(&sh.bars[BAR_STAY_EMPTY + (units & 1)], (units >> 1 & 1) ^ 1);
            } else if (n >= 2) {
                ok = wait_bounded(&sh.bars[BAR_STREAM_EMPTY + slot], (n >> 1 & 1) ^ 1);
            }
            if (thread == 0) sh.info[(SUMS ? 2 * units + tile.half : n) % kInfos] = TileInfo{__uint_as_float((uint32_t)(127 + exponent) << 23), raw.valid};
            producers_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int eight = i * 4 + producer, token = eight * 8 + (lane & 7), quarter = lane >> 3;
                uint8_t *const to = to_tile + eight * ROWS8 + quarter * 128 + (lane & 7) * 16;
                const uint2 scales = *reinterpret_cast<const uint2 *>(sh.scales[turn][token]);
#pragma unroll
                for (int b = 0; b < B; ++b)
                    *reinterpret_cast<uint4 *>(to + b * 512) = decode(raw.keys[i][b], as_half2(__byte_perm(b & 2 ? scales.y : scales.x, 0, b & 1 ? 0x3232 : 0x1010)));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (!SUMS) {
                mbar_arrive(&sh.bars[BAR_STREAM_FULL + slot]);
            } else if (tile.last) {
                mbar_arrive(&sh.bars[BAR_STAY_FULL + (units & 1)]);
                ++units;
            }
            ++n;
            return true;
        };
        while (even.there) {
            if (!produce(even_raw, even, odd_raw, odd)) break;
            if (!odd.there || !produce(odd_raw, odd, even_raw, even)) break;
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssuerRegisters));
        if (warp == kIssuerWarp) {
            // ---- the products ---------------------------------------------------------------------------------
            constexpr uint32_t kIdesc = 1u << 4 | (uint32_t)(128 >> 4) << 24 | (uint32_t)(128 >> 3) << 17;  // fp32 sums of f16 products, both operands along k, 128 x 128
            const uint32_t stay_at = smem_u32(stay_smem), stream_at = smem_u32(stream_smem);
            uint32_t units = 0, streamed = 0, steps[2] = {0, 0};
            bool more = true;
            while (ok && more) {
                if (work.step1 > work.step0) {
                    const uint32_t pair = units & 1;
                    const int halves = work.halves();
                    ok = warp_wait(&sh.bars[BAR_STAY_FULL + pair], units >> 1 & 1);
                    for (int32_t step = work.step0; ok && step < work.step1; ++step, ++streamed) {
                        const uint32_t slot = streamed & 1;
                        ok = warp_wait(&sh.bars[BAR_STREAM_FULL + slot], streamed >> 1 & 1);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (!ok || half >= halves) break;
                            const uint32_t buffer = steps[half] & 1;
                            if (steps[half] >= 2) ok = warp_wait(&sh.bars[BAR_S_EMPTY + 2 * half + buffer], (steps[half] >> 1 & 1) ^ 1);
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
                more = work.next(p);
            }
            // whatever happened: nothing is in flight when the tensor memory goes
            if (lane == 0) mma_commit(&sh.bars[BAR_DONE]);
            __syncwarp();
            if (!wait_bounded(&sh.bars[BAR_DONE], 0)) ok = false;
        } else if (warp == kCopyWarp) {
            // ---- rows of q: images to shared memory -------------------------------------------------------------
            uint32_t units = 0, streamed = 0;
            bool more = true;
            const auto copy = [&](uint8_t *to, int32_t tile, uint64_t *bar) { bulk_copy_g2s(to, p.images + work.image(p, tile) * TILE_BYTES, TILE_BYTES, bar); };
            while (ok && more) {
                if (work.step1 > work.step0) {
                    if (!SUMS) {
                        const uint32_t pair = units & 1;
                        if (units >= 2) ok = warp_wait(&sh.bars[BAR_STAY_EMPTY + pair], (units >> 1 & 1) ^ 1);
                        if (!ok) break;
                        if (lane == 0) {
                            const int halves = work.halves();
                            mbar_expect_tx(&sh.bars[BAR_STAY_FULL + pair], halves * TILE_BYTES);
                            for (int half = 0; half < halves; ++half) copy(stay_smem + (2 * pair + half) * TILE_BYTES, 2 * work.o + half, &sh.bars[BAR_STAY_FULL + pair]);
                        }
                        __syncwarp();
                        ++units;
                    } else {
                        for (int32_t step = work.step0; step < work.step1; ++step, ++streamed) {
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
                if (ok) more = work.next(p);
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

// The pieces' sums of a column joined, always in the same order: a thread to a column, a block to 128.
__global__ void __launch_bounds__(kTokens) kv_weights_columns_kernel(const __grid_constant__ PromptParams p)
{
    Counts before;
    const Cut cut = find_cut(p);
    // the lengths are what the kernels in front read: nothing has written them since
    const int seq = find_sequence(p, cut, blockIdx.x, [](const Counts &c) { return c.tiles; }, &before), head = blockIdx.y;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the ones in front, too
    if (seq < 0) return;
    const Sequence s = sequence<8>(p, seq);
    const int tile = blockIdx.x - before.tiles, columns = s.rows * p.group, pieces = up(up(tokens_held(p, s.length), kTokens), cut.first);
    const int64_t at = ((int64_t)blockIdx.x * p.g.heads + head) * kTokens + threadIdx.x;
    float2 constant = make_float2(0.0f, -INFINITY);  // a column that is none, or sees nothing
    if (tile * 128 + (int)threadIdx.x < columns) {
        const float2 *const from = p.stats_units + (before.units[0] + (int64_t)(head * up(columns, 256) + tile / 2) * pieces) * 256 + (tile & 1) * 128 + threadIdx.x;
        float top = kNothing, sum = 0.0f;
#pragma unroll 4
        for (int i = 0; i < pieces; ++i) {
            const float2 part = from[(int64_t)i * 256];
            const float high = fmaxf(top, part.x);
            sum = sum * exp2f(top - high) + part.y * exp2f(part.x - high);
            top = high;
        }
        constant = make_float2(p.factors[at], sum == 0.0f ? -INFINITY : -(top + log2f(sum)));
    }
    p.constants[at] = constant;
}

// The chunks' weights of a token added up, always in the same order.
__global__ void __launch_bounds__(256) kv_weights_chunks_kernel(const __grid_constant__ PromptParams p)
{
    Counts before;
    const Cut cut = find_cut(p);
    const int seq = find_sequence(p, cut, blockIdx.x, [](const Counts &c) { return c.parts; }, &before);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the ones in front, too
    if (seq < 0) return;
    const Sequence s = sequence<8>(p, seq);
    const int held = tokens_held(p, s.length), outer = up(held, 256), chunks = up(up(s.rows * p.group, 128), cut.second);
    const int local = blockIdx.x - before.parts, of_outer = local / chunks, head = of_outer / outer, t = (of_outer - head * outer) * 256 + threadIdx.x;
    if (local != of_outer * chunks || t >= held) return;  // a block to 256 tokens
    const float *const from = p.parts + (int64_t)blockIdx.x * 256 + threadIdx.x;
    float w = 0.0f;
#pragma unroll 4
    for (int i = 0; i < chunks; ++i) w += from[(int64_t)i * 256];
    Unit u{};
    u.seq = seq;
    u.length = s.length;
    u.rows = s.rows;
    put_weight(p, u, head, t, w);
}

// Tiles of columns, units and parts that there can be.
struct Bounds {
    int64_t tiles, units, parts;
};
Bounds bounds(const WeightsParams &p)
{
    // at most kSteps units by the cut, and one more for every 256 columns of a head; parts: the chunks are at most twice the steps by the cut
    const int64_t columns = p.tokens * p.group;
    return {columns / 128 + p.batch, kSteps + p.g.heads * (columns / 256 + p.batch), 2 * kSteps};
}

int64_t rounded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

template <int B>
lce_status launch(PromptParams &p, const TimeoutReport &report, cudaStream_t s)
{
    static SmemOptIn first_opt_in, second_opt_in;
    if (!first_opt_in.ensure(kv_weights_prompt_kernel<B, false>, weights_smem(B)) || !second_opt_in.ensure(kv_weights_prompt_kernel<B, true>, weights_smem(B))) return LCE_ERR_CUDA;
    const Bounds most = bounds(p);
    const dim3 tiles((unsigned)most.tiles, (unsigned)p.g.heads);
    lce_status st = launch_dependent(kv_weights_rows_kernel<B>, tiles, kTokens, 0, s, p);
    if (st == LCE_OK) st = launch_dependent(kv_weights_prompt_kernel<B, false>, dim3(kBlocks), kThreads, weights_smem(B), s, p, report);
    if (st == LCE_OK) st = launch_dependent(kv_weights_columns_kernel, tiles, kTokens, 0, s, p);
    if (st == LCE_OK) st = launch_dependent(kv_weights_prompt_kernel<B, true>, dim3(kBlocks), kThreads, weights_smem(B), s, p, report);
    if (st == LCE_OK) st = launch_dependent(kv_weights_chunks_kernel, dim3((unsigned)most.parts), 256, 0, s, p);
    return st;
}

}  // namespace

size_t kv_weights_prompt_bytes(const WeightsParams &p)
{
    const Bounds most = bounds(p);
    const int64_t columns = most.tiles * p.g.heads * kTokens;
    return (size_t)(rounded(columns * 64 * p.g.blocks) + rounded(columns * 4) + rounded(columns * 8) + rounded(most.units * 256 * 8) + rounded(most.parts * 256 * 4));
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
    char *at = static_cast<char *>(workspace);
    const auto take = [&](int64_t bytes) {
        char *const here = at;
        at += rounded(bytes);
        return here;
    };
    p.images = reinterpret_cast<uint8_t *>(take(columns * 64 * p.g.blocks));
    p.factors = reinterpret_cast<float *>(take(columns * 4));
    p.constants = reinterpret_cast<float2 *>(take(columns * 8));
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
