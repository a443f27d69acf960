// Eviction from the 4-bit cache: which tokens of a head stay, and their rows moved to pages of their own.
//
// Choosing: a cluster of up to eight blocks to a (sequence, head).  Scores become whole numbers that compare alike, and the budget-th largest is
// found from the top in three digits: every block counts its own tokens' digits in shared memory, adds a share of the bins up over all blocks
// where they are, and reads the others' shares.  Then each warp counts what it keeps of its own run of tokens, and from the counts in front of it knows where that goes: the
// order of the tokens stays, and ties fall to the earlier ones.
//
// Moving: words go from place to place as they are, in vectors, keys and scales token by token, values by the halves of a pair's word.
// Where they come from is only known token by token, so that is looked up once, a thread to a token, for up to sixteen tiles.
//
// Measured: 131072 tokens of 8 heads of 128 channels cut to 32768: choosing 25 us (64 blocks, a chain of counts and cluster barriers for each digit), moving 22
// (38 MB of rows read and written, 12 at the copy rate; values lie in pairs of tokens, so that a quarter that stays touches most sectors: 105 MB are
// read); 24 sequences of up to 8192 tokens cut to 2048, 64 channels: 19 and 17 us.
#include "kv_common.cuh"
#include "row_overlap.cuh"

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

constexpr int kMostWarps = 32;
constexpr int kMostCluster = 8;      // blocks to a row (sixteen: 32 us instead of 26 for 131072 tokens of eight heads)
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

__device__ __forceinline__ uint32_t remote1(const void *p, int rank)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote_place(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint2 remote2(const void *p, int rank)
{
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(remote_place(p, rank)) : "memory");
    return v;
}

// 0 never stays and the highest always does; in between NaN and then numbers in their order, both zeros alike.
__device__ __forceinline__ uint32_t key_of(const EvictParams &p, int32_t page, float score, int32_t token, int32_t length)
{
    const uint32_t bits = __float_as_uint(score + 0.0f);
    uint32_t key = bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
    if (score != score) key = 1;
    if (length > p.budget && (token < p.first || token >= length - p.recent)) key = 0xffffffffu;
    return (uint32_t)page < (uint32_t)p.g.pages ? key : 0;
}

struct alignas(16) SelectShared {
    uint32_t bins[kDigits][kBins];
    uint32_t sums[kBins / 2];     // of the block's share of the bins, where there are several blocks
    uint32_t warp_sums[kMostWarps];
    uint2 warp_counts[kMostWarps];
    uint2 counts;                 // of the block: tokens above the threshold, on it
    uint32_t digit, left, whole;
};

// KEYS of a thread, the warp's run of tokens 32 at a time, in registers; 0: any number, made again from the scores wherever they are
// looked at.
template <int KEYS, int THREADS>
__global__ void __launch_bounds__(THREADS) kv_evict_select_kernel(const __grid_constant__ EvictParams p)
{
    constexpr int kThreads = THREADS, kWarps = THREADS / 32, BINS = kBins / THREADS;  // bins of a thread
    __shared__ SelectShared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x / p.cluster, rank = blockIdx.x - row * p.cluster, seq = row / p.g.heads, head = row - seq * p.g.heads;
    for (int i = threadIdx.x; i < kDigits * kBins / 4; i += kThreads) reinterpret_cast<uint4 *>(&sh.bins[0][0])[i] = make_uint4(0, 0, 0, 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    release_join();
    const int32_t length = max(__ldg(p.lengths + seq), 0), held = min(length, p.table_tokens);
    const int32_t *const table = p.page_table + (int64_t)seq * p.table_pages;
    const float *const scores = p.scores + seq * p.scores_seq + head * p.scores_head;
    // the block's tokens, and the warp's run of them: whole steps of 32
    const int32_t share = (held + p.cluster - 1) / p.cluster, begin = min(rank * (int64_t)share, (int64_t)held), end = min(begin + (int64_t)share, (int64_t)held);
    const int32_t run = ((end - begin + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int32_t run_begin = min(begin + (int64_t)warp * run, (int64_t)end), run_end = min(run_begin + (int64_t)run, (int64_t)end);
    uint32_t keys[KEYS > 0 ? KEYS : 1];
#pragma unroll
    for (int i = 0; i < KEYS; ++i) keys[i] = 0;
    if (KEYS > 0 && run_begin < run_end) {
        // all loads at once; behind the run its last token again
        float score[KEYS > 0 ? KEYS : 1];
#pragma unroll
        for (int i = 0; i < KEYS; ++i) score[i] = __ldg(scores + min(run_begin + 32 * i + lane, run_end - 1));
#pragma unroll
        for (int i = 0; i < KEYS; ++i) keys[i] = (uint32_t)__ldg(table + p.by_page(min(run_begin + 32 * i + lane, run_end - 1)));
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int32_t t = run_begin + 32 * i + lane;
            keys[i] = t < run_end ? key_of(p, (int32_t)keys[i], score[i], t, length) : 0;
        }
    }
    // body(first of 32 tokens, the lane's key; 0 behind the run), by whole warps
    const auto each_key = [&](auto body) {
        if (KEYS > 0) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) body(run_begin + 32 * i, keys[i]);
        } else {
#pragma unroll 4
            for (int32_t t0 = run_begin; t0 < run_end; t0 += 32) {
                const int32_t t = min(t0 + lane, run_end - 1);
                const uint32_t key = key_of(p, __ldg(table + p.by_page(t)), __ldg(scores + t), t, length);
                body(t0, t0 + lane < run_end ? key : 0);
            }
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
            const uint32_t common = __shfl_sync(0xffffffffu, bin, 0);
            const bool alike = counts && bin == common;
            if (__all_sync(0xffffffffu, alike)) {
                if (lane == 0) atomicAdd(&bins[bin], 32u);
            } else if (counts) {
                atomicAdd(&bins[bin], 1u);
            }
        });
        cluster_sync();
        // a thread's bins, the highest first, over all blocks: each block adds its share of them up for the others, which read the sums (all blocks'
        // counts read by all of them: 30 us instead of 26 for 131072 tokens of eight heads)
        const int bin0 = kBins - BINS - BINS * (int)threadIdx.x;
        uint32_t n[BINS], mine = 0;
        if (p.cluster > 1) {
            const int each = kBins / p.cluster;
            for (int i = threadIdx.x; i < each; i += kThreads) {
                uint32_t sum = 0;
#pragma unroll 8
                for (int r = 0; r < p.cluster; ++r) sum += remote1(&bins[rank * each + i], r);
                sh.sums[i] = sum;
            }
            cluster_sync();
#pragma unroll
            for (int i = 0; i < BINS; ++i) {
                const int bin = bin0 + BINS - 1 - i;
                n[i] = remote1(&sh.sums[bin % each], bin / each);
            }
        } else {
#pragma unroll
            for (int i = 0; i < BINS; ++i) n[i] = bins[bin0 + BINS - 1 - i];
        }
#pragma unroll
        for (int i = 0; i < BINS; ++i) mine += n[i];
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) sh.warp_sums[warp] = upto;
        __syncthreads();
        const uint32_t of_lane = lane < kWarps ? sh.warp_sums[lane] : 0, total = __reduce_add_sync(0xffffffffu, of_lane);
        uint32_t before = upto - mine + __reduce_add_sync(0xffffffffu, lane < warp ? of_lane : 0);
        if (digit == 0 && total <= left) break;  // all that there are stay
        if (before < left && before + mine >= left) {
            int i = 0;
#pragma unroll
            for (int k = 1; k < BINS; ++k)
                if (i == k - 1 && before + n[k - 1] < left) {
                    before += n[k - 1];
                    i = k;
                }
            uint32_t there = n[0];
#pragma unroll
            for (int k = 1; k < BINS; ++k) there = i == k ? n[k] : there;
            sh.digit = bin0 + BINS - 1 - i;
            sh.left = left - before;
            sh.whole = before + there == left;
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
        mine.x += key > threshold;
        mine.y += key == threshold && ties > 0;  // ties: of a threshold above 0
    });
    mine.x = __reduce_add_sync(0xffffffffu, mine.x);
    mine.y = __reduce_add_sync(0xffffffffu, mine.y);
    if (lane == 0) sh.warp_counts[warp] = mine;
    __syncthreads();
    const uint2 of_lane = lane < kWarps ? sh.warp_counts[lane] : make_uint2(0, 0);
    uint2 before = make_uint2(__reduce_add_sync(0xffffffffu, lane < warp ? of_lane.x : 0), __reduce_add_sync(0xffffffffu, lane < warp ? of_lane.y : 0));
    const uint2 all = make_uint2(__reduce_add_sync(0xffffffffu, of_lane.x), __reduce_add_sync(0xffffffffu, of_lane.y));
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
        const uint32_t below = (1u << lane) - 1, higher = __ballot_sync(0xffffffffu, key > threshold);
        uint32_t at = before.x + __popc(higher & below);
        bool stays = key > threshold;
        if (ties > 0) {
            const uint32_t equal = __ballot_sync(0xffffffffu, key == threshold), ties_before = before.y + __popc(equal & below);
            at += min(ties_before, ties);
            stays = stays || (key == threshold && ties_before < ties);
            before.y += __popc(equal);
        }
        if (stays) {
            kept[at] = t0 + lane;
            if (kept_scores) kept_scores[at] = __ldg(scores + t0 + lane);
        }
        before.x += __popc(higher);
    });
    for (int64_t i = count + (int64_t)rank * kThreads + threadIdx.x; i < p.budget; i += (int64_t)p.cluster * kThreads) {
        kept[i] = -1;
        if (kept_scores) kept_scores[i] = 0.0f;
    }
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

// TILES tiles to a block: where their tokens are (what is kept there, its page) is found out once, a thread to a token.  Then every thread
// has one of the 64 places of keys, 64 of values and 16 of scales that a plane of a tile has, of several tiles whose loads are on
// their way together.
constexpr int kMoveThreads = 256;

// The token's tile of the cache and its place there; negative: there is none.
struct Source {
    int32_t tile, token;
};

template <int TILES>
__global__ void __launch_bounds__(kMoveThreads, 4) kv_evict_move_kernel(const __grid_constant__ EvictParams p)
{
    static_assert(TILES * kKvTile <= kMoveThreads && TILES % 4 == 0, "");
    __shared__ alignas(16) Source sources[TILES * kKvTile];
    __shared__ int32_t targets[TILES];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int head = blockIdx.y, seq = blockIdx.z, blocks = p.g.blocks, tiles_per_page = p.g.page_size / kKvTile;
    const int32_t first = blockIdx.x * TILES * kKvTile;
    const auto tile_on = [&](int32_t page, int32_t in_page) { return (page * p.g.heads + head) * tiles_per_page + in_page / kKvTile; };
    if (threadIdx.x < TILES * kKvTile) {
        const int32_t j = first + threadIdx.x;
        const int32_t *const kept = p.kept + ((int64_t)seq * p.g.heads + head) * p.budget;
        const int32_t from = j < p.budget ? kept[j] : -1;
        // Every head has as many.  Here and not in the kernel in front, which reads the lengths: they may be the same memory.
        if (head == 0 && j < p.budget && from >= 0 && (j + 1 == p.budget || kept[j + 1] < 0)) p.kept_lengths[seq] = j + 1;
        if (head == 0 && j == 0 && from < 0) p.kept_lengths[seq] = 0;
        const int32_t in_kept = p.by_page(j), target = j < p.budget ? __ldg(p.kept_table + (int64_t)seq * p.kept_pages + in_kept) : -1;
        Source s{-1, 0};
        if (from >= 0 && from < p.table_tokens) {
            const int32_t in_table = p.by_page(from), page = __ldg(p.page_table + (int64_t)seq * p.table_pages + in_table), in_page = from - in_table * p.g.page_size;
            if ((uint32_t)page < (uint32_t)p.g.pages) s = Source{tile_on(page, in_page), in_page % kKvTile};
        }
        sources[threadIdx.x] = s;
        if (threadIdx.x % kKvTile == 0) targets[threadIdx.x / kKvTile] = (uint32_t)target < (uint32_t)p.g.pages ? tile_on(target, j - in_kept * p.g.page_size) : -1;
    }
    __syncthreads();
    const int words = kv_tile_words(blocks);
    const auto plane = [&](int plane0, auto width) {
        constexpr int W = decltype(width)::value, EACH = TILES / 4;
        // keys: thread's place of every fourth tile
        {
            const int place = threadIdx.x & 63, token = 8 * (place >> 5) + ((place & 31) >> 2), at = 64 * plane0;
            Words<W> w[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const Source s = sources[(4 * i + (threadIdx.x >> 6)) * kKvTile + token];
                if (s.tile >= 0) w[i] = load_words<W>(p.cache + (int64_t)s.tile * words + at + ((s.token >> 3) * 32 + (s.token & 7) * 4 + (place & 3)) * W);
            }
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int tile = 4 * i + (threadIdx.x >> 6);
                if (sources[tile * kKvTile + token].tile >= 0 && targets[tile] >= 0) store_words<W>(p.cache + (int64_t)targets[tile] * words + at + place * W, w[i]);
            }
        }
        // values: a word is of two tokens
        {
            const int place = threadIdx.x & 63, token = 8 * (place >> 5) + 2 * (place & 3), at = 64 * blocks + 64 * plane0;
            constexpr int SOME = EACH > 2 ? 2 : EACH;
#pragma unroll
            for (int i0 = 0; i0 < EACH; i0 += SOME) {
                Words<W> w[SOME][2];
                int4 both[SOME];
#pragma unroll
                for (int i = 0; i < SOME; ++i) {
                    both[i] = *reinterpret_cast<const int4 *>(&sources[(4 * (i0 + i) + (threadIdx.x >> 6)) * kKvTile + token]);
                    const auto load = [&](int32_t tile, int32_t t) { return load_words<W>(p.cache + (int64_t)tile * words + at + ((t >> 3) * 32 + (place & 28) + (t >> 1 & 3)) * W); };
                    if (both[i].x >= 0) w[i][0] = load(both[i].x, both[i].y);
                    if (both[i].z >= 0) w[i][1] = load(both[i].z, both[i].w);
                }
#pragma unroll
                for (int i = 0; i < SOME; ++i) {
                    const int32_t target = targets[4 * (i0 + i) + (threadIdx.x >> 6)];
                    if (target < 0 || both[i].x < 0) continue;
                    uint32_t *const to = p.cache + (int64_t)target * words + at + place * W;
                    if (both[i].z >= 0) {
                        Words<W> r;
                        const uint32_t select = (both[i].y & 1 ? 0x32 : 0x10) | (both[i].w & 1 ? 0x7600 : 0x5400);
#pragma unroll
                        for (int x = 0; x < W; ++x) r.w[x] = __byte_perm(w[i][0].w[x], w[i][1].w[x], select);
                        store_words<W>(to, r);
                    } else {  // the last token: its half of the words
#pragma unroll
                        for (int x = 0; x < W; ++x) *reinterpret_cast<uint16_t *>(to + x) = (uint16_t)(w[i][0].w[x] >> (both[i].y & 1 ? 16 : 0));
                    }
                }
            }
        }
        // scales: a thread to a token
        if (threadIdx.x < TILES * kKvTile) {
            const Source s = sources[threadIdx.x];
            const int32_t target = targets[threadIdx.x / kKvTile];
            const int at = 128 * blocks + 16 * plane0;
            if (s.tile >= 0 && target >= 0)
                store_words<W>(p.cache + (int64_t)target * words + at + (threadIdx.x % kKvTile) * W, load_words<W>(p.cache + (int64_t)s.tile * words + at + s.token * W));
        }
    };
    for (int plane0 = 0; plane0 + 4 <= blocks; plane0 += 4) plane(plane0, std::integral_constant<int, 4>());
    if (blocks & 2) plane(blocks & ~3, std::integral_constant<int, 2>());
    if (blocks & 1) plane(blocks - 1, std::integral_constant<int, 1>());
}

lce_status launch_move(const EvictParams &p, cudaStream_t s)
{
    const int64_t tiles = (p.budget + kKvTile - 1) / kKvTile;
    const auto go = [&](auto kernel, int each) {
        return launch_dependent(kernel, dim3((unsigned)((tiles + each - 1) / each), (unsigned)p.g.heads, (unsigned)p.batch), kMoveThreads, 0, s, p);
    };
    // as many tiles to a block as leave every SM its blocks
    return tiles * p.g.heads * p.batch > 148 * 16 ? go(kv_evict_move_kernel<16>, 16) : go(kv_evict_move_kernel<4>, 4);
}

template <int KEYS, int THREADS>
lce_status launch_select(const EvictParams &p, cudaStream_t s)
{
    const auto kernel = kv_evict_select_kernel<KEYS, THREADS>;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.batch * p.g.heads * p.cluster), 1, 1);
    cfg.blockDim = dim3(THREADS, 1, 1);
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

lce_status launch_select(const EvictParams &p, cudaStream_t s)
{
    const int64_t share = ((int64_t)p.table_tokens + p.cluster - 1) / p.cluster;
    if (share <= 1024) return launch_select<1, 1024>(p, s);
    if (share <= 4 * 1024) return launch_select<4, 1024>(p, s);
    // half the threads where there are rows for two blocks to an SM
    if (share <= 16 * 512 && (int64_t)p.batch * p.g.heads * p.cluster > 148) return launch_select<16, 512>(p, s);
    if (share <= 8 * 1024) return launch_select<8, 1024>(p, s);
    if (share <= 16 * 1024) return launch_select<16, 1024>(p, s);
    return launch_select<0, 1024>(p, s);
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
        (int64_t)d.batch * d.cache.kv_heads * kMostCluster >= (1ll << 31) || (int64_t)p.g.slots / kKvTile * p.g.heads >= (1ll << 31))
        return LCE_ERR_UNSUPPORTED;
    if (!cache || !page_table || !lengths || !scores || !kept_table || !kept || !kept_lengths) return LCE_ERR_INVALID_ARG;
    if (!aligned(cache, 16) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(scores, 4) || !aligned(kept_table, 4) || !aligned(kept, 4) ||
        !aligned(kept_lengths, 4) || !aligned(kept_scores, 4))
        return LCE_ERR_ALIGNMENT;
    // Scores are read again where they are written to their new places, by other warps and blocks, too.  How long rows of scores are follows from the
    // lengths, on the device: here every row is looked at by its first element.
    const RowSet new_scores{kept_scores, d.batch, p.g.heads, d.kept_scores_seq_stride, d.kept_scores_head_stride, d.budget, 4};
    if (kept_scores && (!rows_apart(new_scores) || rows_meet({scores, d.batch, p.g.heads, d.scores_seq_stride, d.scores_head_stride, 1, 4}, new_scores))) return LCE_ERR_INVALID_ARG;
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
    while (p.cluster < kMostCluster && p.table_tokens > kClusterTokens * p.cluster && (int64_t)p.batch * p.g.heads * p.cluster * 2 <= 148 * 2) p.cluster *= 2;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const lce_status chosen = launch_select(p, s);
    return chosen != LCE_OK ? chosen : launch_move(p, s);
}
