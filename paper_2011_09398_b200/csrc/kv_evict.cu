// Eviction from the 4-bit cache: which tokens of a head stay, and their rows moved to pages of their own.
//
// Choosing: a cluster of up to eight blocks to a (sequence, head).  Scores become whole numbers that compare alike, and the budget-th largest is
// found from the top in three digits: every block counts its own tokens' digits in shared memory, and all read all blocks' counts where
// they are.  Then each warp counts what it keeps of its own run of tokens, and from the counts in front of it knows where that goes: the
// order of the tokens stays, and ties fall to the earlier ones.
//
// Moving: words go from place to place as they are, in vectors, keys and scales token by token, values by the halves of a pair's word.
// Sixteen kept tokens of a head make a tile, whose words a thread each puts together; where they come from is only known token by token.
#include "kv_common.cuh"

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048, kDigits = 3;
constexpr int kClusterTokens = 2048; // tokens that a block more is worth

struct EvictParams {
    KvGeom g;
    int32_t batch, table_pages, table_tokens, kept_pages;
    int32_t budget, first, recent;
    int32_t cluster;
    int64_t scores_seq, scores_head, kept_seq, kept_head;
    FastDiv by_page;
    uint32_t *cache;
    const int32_t *page_table, *lengths, *kept_table;
    const float *scores;
    int32_t *kept, *kept_lengths;
    float *kept_scores;
};

__device__ __forceinline__ uint4 remote4(const void *p, int rank)
{
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(remote_place(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint2 remote2(const void *p, int rank)
{
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(remote_place(p, rank)) : "memory");
    return v;
}

// Where a token of a sequence lies: its slot, or negative on a page outside the pool.
__device__ __forceinline__ int32_t slot_of(const EvictParams &p, const int32_t *table, int32_t token)
{
    const int32_t in_table = p.by_page(token), page = __ldg(table + in_table);
    return page >= 0 && page < p.g.pages ? page * p.g.page_size + (token - in_table * p.g.page_size) : -1;
}
__device__ __forceinline__ uint32_t *tile_of(const EvictParams &p, int32_t slot, int head)
{
    const int32_t page = p.by_page(slot);
    const int64_t tile = ((int64_t)page * p.g.heads + head) * (p.g.page_size / kKvTile) + (slot - page * p.g.page_size) / kKvTile;
    return p.cache + tile * kv_tile_words(p.g.blocks);
}

// 0 never stays and the highest always does; in between NaN and then numbers in their order, both zeros alike.
__device__ __forceinline__ uint32_t key_of(const EvictParams &p, const int32_t *table, const float *scores, int32_t token, int32_t length)
{
    const int32_t in_table = p.by_page(token), page = __ldg(table + in_table);
    const float score = __ldg(scores + token);
    const uint32_t bits = __float_as_uint(score + 0.0f);
    uint32_t key = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    if (score != score) key = 1;
    if (length > p.budget && (token < p.first || token >= length - p.recent)) key = 0xffffffffu;
    return page >= 0 && page < p.g.pages ? key : 0;
}

struct alignas(16) SelectShared {
    uint32_t bins[kDigits][kBins];
    uint32_t warp_sums[kWarps];
    uint2 warp_counts[kWarps];
    uint2 counts;                 // of the block: tokens above the threshold, on it
    uint32_t digit, left, whole;
};

// KEYS of a thread, the warp's run of tokens 32 at a time, in registers; 0: any number, made again from the scores wherever they are
// looked at.
template <int KEYS>
__global__ void __launch_bounds__(kThreads) kv_evict_select_kernel(const __grid_constant__ EvictParams p)
{
    __shared__ SelectShared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x / p.cluster, rank = blockIdx.x - row * p.cluster, seq = row / p.g.heads, head = row - seq * p.g.heads;
    for (int i = threadIdx.x; i < kDigits * kBins / 4; i += kThreads) reinterpret_cast<uint4 *>(&sh.bins[0][0])[i] = make_uint4(0, 0, 0, 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the moving takes its place; it waits for all of this kernel
    const int32_t length = max(__ldg(p.lengths + seq), 0), held = min(length, p.table_tokens);
    const int32_t *const table = p.page_table + (int64_t)seq * p.table_pages;
    const float *const scores = p.scores + seq * p.scores_seq + head * p.scores_head;
    // the block's tokens, and the warp's run of them: whole steps of 32
    const int32_t share = (held + p.cluster - 1) / p.cluster, begin = min(rank * (int64_t)share, (int64_t)held), end = min(begin + (int64_t)share, (int64_t)held);
    const int32_t run = ((end - begin + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int32_t run_begin = min(begin + (int64_t)warp * run, (int64_t)end), run_end = min(run_begin + (int64_t)run, (int64_t)end);
    uint32_t keys[KEYS > 0 ? KEYS : 1];
    if (KEYS > 0) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int32_t t = run_begin + 32 * i + lane;
            keys[i] = t < run_end ? key_of(p, table, scores, t, length) : 0;
        }
    }
    // body(first of 32 tokens, the lane's key; 0 behind the run), by whole warps
    const auto each_key = [&](auto body) {
        if (KEYS > 0) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i)
                if (run_begin + 32 * i < run_end) body(run_begin + 32 * i, keys[i]);
        } else {
#pragma unroll 4
            for (int32_t t0 = run_begin; t0 < run_end; t0 += 32) body(t0, t0 + lane < run_end ? key_of(p, table, scores, t0 + lane, length) : 0);
        }
    };
    __syncthreads();

    // the threshold's digits so far; how many are still to be taken among the keys that have them
    uint32_t prefix = 0, left = (uint32_t)p.budget, threshold = 0, ties = 0;
#pragma unroll 1
    for (int digit = 0; digit < kDigits; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
        uint32_t *const bins = sh.bins[digit];
        each_key([&](int32_t, uint32_t key) {
            const bool counts = key != 0 && (digit == 0 || key >> (shift + bits) == prefix);
            const uint32_t bin = key >> shift & ((1u << bits) - 1);
            // all alike in one go: they would queue up
            const uint32_t those = __ballot_sync(0xffffffffu, counts);
            if (!those) return;
            const int leader = __ffs(those) - 1;
            const uint32_t common = __shfl_sync(0xffffffffu, bin, leader);
            if (__all_sync(0xffffffffu, !counts || bin == common)) {
                if (lane == leader) atomicAdd(&bins[common], (uint32_t)__popc(those));
            } else if (counts) {
                atomicAdd(&bins[bin], 1u);
            }
        });
        cluster_sync();
        // four bins a thread, the highest first, over all blocks
        const int bin0 = kBins - 4 - 4 * (int)threadIdx.x;
        uint32_t n[4] = {};
#pragma unroll 8
        for (int r = 0; r < p.cluster; ++r) {
            const uint4 v = remote4(&bins[bin0], r);
            n[0] += v.w;
            n[1] += v.z;
            n[2] += v.y;
            n[3] += v.x;
        }
        const uint32_t mine = n[0] + n[1] + n[2] + n[3];
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) sh.warp_sums[warp] = upto;
        __syncthreads();
        uint32_t before = upto - mine, total = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sh.warp_sums[w];
            total += sh.warp_sums[w];
        }
        if (digit == 0 && total <= left) break;  // all that there are stay
        if (before < left && before + mine >= left) {
            int i = 0;
            while (before + n[i] < left) before += n[i++];
            sh.digit = bin0 + 3 - i;
            sh.left = left - before;
            sh.whole = before + n[i] == left;
        }
        __syncthreads();
        prefix = prefix << bits | sh.digit;
        left = sh.left;
        if (sh.whole) {  // all keys that begin like this stay: their other digits do not matter
            threshold = max(prefix << shift, 1u) - 1;
            break;
        }
        threshold = prefix;
        ties = digit == kDigits - 1 ? left : 0;
    }

    uint2 mine = make_uint2(0, 0);
    each_key([&](int32_t, uint32_t key) {
        mine.x += __popc(__ballot_sync(0xffffffffu, key > threshold));
        mine.y += __popc(__ballot_sync(0xffffffffu, key == threshold && key != 0));
    });
    if (lane == 0) sh.warp_counts[warp] = mine;
    __syncthreads();
    uint2 before = make_uint2(0, 0), all = make_uint2(0, 0);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const uint2 c = sh.warp_counts[w];
        if (w < warp) {
            before.x += c.x;
            before.y += c.y;
        }
        all.x += c.x;
        all.y += c.y;
    }
    if (threadIdx.x == 0) sh.counts = all;
    cluster_sync();
    uint32_t above = 0;
    for (int r = 0; r < p.cluster; ++r) {
        const uint2 c = remote2(&sh.counts, r);
        if (r < rank) {
            before.x += c.x;
            before.y += c.y;
        }
        above += c.x;
    }
    const uint32_t count = above + ties;
    int32_t *const kept = p.kept + (int64_t)row * p.budget;
    float *const kept_scores = p.kept_scores ? p.kept_scores + seq * p.kept_seq + head * p.kept_head : nullptr;
    each_key([&](int32_t t0, uint32_t key) {
        const uint32_t below = (1u << lane) - 1;
        const bool is_equal = key == threshold && key != 0;
        const uint32_t higher = __ballot_sync(0xffffffffu, key > threshold), equal = __ballot_sync(0xffffffffu, is_equal);
        const uint32_t ties_before = before.y + __popc(equal & below);
        const uint32_t at = before.x + __popc(higher & below) + min(ties_before, ties);
        if (key > threshold || (is_equal && ties_before < ties)) {
            kept[at] = t0 + lane;
            if (kept_scores) kept_scores[at] = __ldg(scores + t0 + lane);
        }
        before.x += __popc(higher);
        before.y += __popc(equal);
    });
    for (int64_t i = count + (int64_t)rank * kThreads + threadIdx.x; i < p.budget; i += (int64_t)p.cluster * kThreads) {
        kept[i] = -1;
        if (kept_scores) kept_scores[i] = 0.0f;
    }
    if (head == 0 && rank == 0 && threadIdx.x == 0) p.kept_lengths[seq] = (int32_t)count;
    cluster_sync();  // nobody leaves while its counts are read
}

template <int W>
struct Words {
    uint32_t w[W];
};
template <int W>
__device__ __forceinline__ Words<W> load_words(const uint32_t *p)
{
    Words<W> r;
    if constexpr (W == 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    } else if constexpr (W == 2) {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
        r.w[0] = v.x; r.w[1] = v.y;
    } else {
        r.w[0] = __ldg(p);
    }
    return r;
}
template <int W>
__device__ __forceinline__ void store_words(uint32_t *p, const Words<W> &r)
{
    if constexpr (W == 4) *reinterpret_cast<uint4 *>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    else if constexpr (W == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(r.w[0], r.w[1]);
    else *p = r.w[0];
}

// 64 places of keys, 64 of values, 16 of scales for a plane of a tile; two tiles side by side in a block, TILES pairs of them one behind the
// other.  A word is four loads away (where it goes, what is kept there, that token's page, the word), so a thread has its tiles'
// loads of each kind on their way together.
constexpr int kPlaces = 144, kMoveThreads = 2 * kPlaces;

template <int TILES>
__global__ void __launch_bounds__(kMoveThreads) kv_evict_move_kernel(const __grid_constant__ EvictParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int in_block = threadIdx.x / kPlaces, place = threadIdx.x - in_block * kPlaces;
    const int head = blockIdx.y, seq = blockIdx.z, blocks = p.g.blocks;
    const bool values = place >= 64 && place < 128;
    const int in_part = values ? place - 64 : place < 64 ? place : place - 128;
    // the token, or the first of the two, that the place is for
    const int token = values ? 8 * (in_part >> 5) + 2 * (in_part & 3) : place < 64 ? 8 * (in_part >> 5) + ((in_part & 31) >> 2) : in_part;
    const int32_t *const kept = p.kept + ((int64_t)seq * p.g.heads + head) * p.budget, *const table = p.page_table + (int64_t)seq * p.table_pages;
    uint32_t *to[TILES];
    int32_t from0[TILES], from1[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int j0 = (2 * (blockIdx.x * TILES + i) + in_block) * kKvTile, in_table = p.by_page(j0);
        const int32_t page = j0 < p.budget ? __ldg(p.kept_table + (int64_t)seq * p.kept_pages + in_table) : -1;
        to[i] = page >= 0 && page < p.g.pages ? tile_of(p, page * p.g.page_size + (j0 - in_table * p.g.page_size), head) : nullptr;
        from0[i] = j0 + token < p.budget ? kept[j0 + token] : -1;  // where it is none, those behind are none either
        from1[i] = values && j0 + token + 1 < p.budget ? kept[j0 + token + 1] : -1;
    }
    const uint32_t *tile0[TILES], *tile1[TILES];
    int t0[TILES], t1[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        if (from0[i] < 0) to[i] = nullptr;
        const int32_t slot0 = to[i] ? slot_of(p, table, from0[i]) : 0, slot1 = to[i] && from1[i] >= 0 ? slot_of(p, table, from1[i]) : slot0;
        tile0[i] = tile_of(p, slot0, head);
        tile1[i] = tile_of(p, slot1, head);
        t0[i] = slot0 % kKvTile;
        t1[i] = slot1 % kKvTile;
    }
    const auto plane = [&](int first, auto width) {
        constexpr int W = decltype(width)::value;
        Words<W> a[TILES], b[TILES];
        const int base = values ? 64 * blocks + 64 * first : place < 64 ? 64 * first : 128 * blocks + 16 * first;
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            if (!to[i]) continue;
            const auto word = [&](int t) {
                if (values) return (t >> 3) * 32 + (in_part & 28) + (t >> 1 & 3);
                return place < 64 ? (t >> 3) * 32 + (t & 7) * 4 + (in_part & 3) : t;
            };
            a[i] = load_words<W>(tile0[i] + base + word(t0[i]) * W);
            if (values) b[i] = load_words<W>(tile1[i] + base + word(t1[i]) * W);
        }
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            if (!to[i]) continue;
            uint32_t *const at = to[i] + base + in_part * W;
            if (!values) {
                store_words<W>(at, a[i]);
            } else if (from1[i] >= 0) {
                Words<W> r;
#pragma unroll
                for (int w = 0; w < W; ++w) r.w[w] = __byte_perm(a[i].w[w], b[i].w[w], (t0[i] & 1 ? 0x32 : 0x10) | (t1[i] & 1 ? 0x7600 : 0x5400));
                store_words<W>(at, r);
            } else {  // the last token: its half of the words
#pragma unroll
                for (int w = 0; w < W; ++w) *reinterpret_cast<uint16_t *>(at + w) = (uint16_t)(a[i].w[w] >> (t0[i] & 1 ? 16 : 0));
            }
        }
    };
    for (int first = 0; first + 4 <= blocks; first += 4) plane(first, std::integral_constant<int, 4>());
    if (blocks & 2) plane(blocks & ~3, std::integral_constant<int, 2>());
    if (blocks & 1) plane(blocks - 1, std::integral_constant<int, 1>());
}

lce_status launch_move(const EvictParams &p, cudaStream_t s)
{
    constexpr int kTogether = 4;
    const int64_t pairs = ((p.budget + kKvTile - 1) / kKvTile + 1) / 2;
    // several tiles to a thread once every SM has its blocks without
    if (pairs * p.g.heads * p.batch > 148 * 6)
        return launch_dependent(kv_evict_move_kernel<kTogether>, dim3((unsigned)((pairs + kTogether - 1) / kTogether), (unsigned)p.g.heads, (unsigned)p.batch), kMoveThreads, 0, s, p);
    return launch_dependent(kv_evict_move_kernel<1>, dim3((unsigned)pairs, (unsigned)p.g.heads, (unsigned)p.batch), kMoveThreads, 0, s, p);
}

lce_status launch_select(const EvictParams &p, cudaStream_t s)
{
    const int64_t share = ((int64_t)p.table_tokens + p.cluster - 1) / p.cluster;
    const auto kernel = share <= 2 * kThreads ? kv_evict_select_kernel<2> : share <= 8 * kThreads ? kv_evict_select_kernel<8>
                      : share <= 32 * kThreads ? kv_evict_select_kernel<32> : kv_evict_select_kernel<0>;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.batch * p.g.heads * p.cluster), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) {
        cudaGetLastError();
        return LCE_ERR_CUDA;
    }
    return LCE_OK;
}

bool stride_ok(int64_t s) { return s >= 0 && s < (1ll << 40); }

}  // namespace
}  // namespace lce

extern "C" lce_status lce_kv_evict(const lce_kv_evict_desc *desc, void *cache, const int32_t *page_table, const int32_t *lengths, const float *scores,
                                   const int32_t *kept_table, int32_t *kept, int32_t *kept_lengths, float *kept_scores, void *stream)
{
    using namespace lce;
    EvictParams p{};
    if (!desc) return LCE_ERR_INVALID_ARG;
    const lce_kv_evict_desc &d = *desc;
    const lce_status st = make_kv_geom(&d.cache, &p.g);
    if (st != LCE_OK) return st;
    if (d.batch <= 0 || d.table_pages <= 0 || d.kept_pages <= 0 || d.budget <= 0 || d.first < 0 || d.recent < 0) return LCE_ERR_INVALID_ARG;
    if ((int64_t)d.first + d.recent > d.budget || d.budget > (int64_t)d.kept_pages * d.cache.page_size) return LCE_ERR_INVALID_ARG;
    for (const int64_t s : {d.scores_seq_stride, d.scores_head_stride, d.kept_scores_seq_stride, d.kept_scores_head_stride})
        if (!stride_ok(s)) return LCE_ERR_INVALID_ARG;
    if ((int64_t)d.table_pages * d.cache.page_size >= (1ll << 30) || (int64_t)d.kept_pages * d.cache.page_size >= (1ll << 30) || d.batch > 65535 ||
        (int64_t)d.batch * d.cache.kv_heads * 8 >= (1ll << 31))
        return LCE_ERR_UNSUPPORTED;
    if (!cache || !page_table || !lengths || !scores || !kept_table || !kept || !kept_lengths) return LCE_ERR_INVALID_ARG;
    if (!aligned(cache, 16) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(scores, 4) || !aligned(kept_table, 4) || !aligned(kept, 4) ||
        !aligned(kept_lengths, 4) || !aligned(kept_scores, 4))
        return LCE_ERR_ALIGNMENT;
    p.batch = d.batch; p.table_pages = d.table_pages; p.kept_pages = d.kept_pages;
    p.table_tokens = d.table_pages * d.cache.page_size;
    p.budget = d.budget; p.first = d.first; p.recent = d.recent;
    p.scores_seq = d.scores_seq_stride; p.scores_head = d.scores_head_stride;
    p.kept_seq = d.kept_scores_seq_stride; p.kept_head = d.kept_scores_head_stride;
    fast_div_constants((uint32_t)p.g.page_size, &p.by_page.mul, &p.by_page.sh);
    p.cache = static_cast<uint32_t *>(cache);
    p.page_table = page_table; p.lengths = lengths; p.kept_table = kept_table;
    p.scores = scores; p.kept = kept; p.kept_lengths = kept_lengths; p.kept_scores = kept_scores;
    // blocks to a row, as long as the GPU has places for them
    p.cluster = 1;
    while (p.cluster < 8 && p.table_tokens > kClusterTokens * p.cluster && (int64_t)p.batch * p.g.heads * p.cluster * 2 <= 148 * 2) p.cluster *= 2;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const lce_status chosen = launch_select(p, s);
    return chosen != LCE_OK ? chosen : launch_move(p, s);
}
