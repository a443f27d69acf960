// Attention of many rows of a sequence (a prompt, a chunk of one) over the 4-bit cache, on the 5th-generation tensor cores.
//
// A block works on 256 columns (rows of q that share a key/value head), two tiles of 128 that take turns, over tiles of 128 tokens:
//   warps 0 - 3, 4 - 7  a tile of columns each, a thread to a column: scores from TMEM, running softmax, weights back to TMEM as f16
//   warps 8 - 11        4-bit words from the cache to f16 keys and values in shared memory, two stages
//   warp 12             one thread issues the products: S = Q K^T (128 x 128 x channels, both operands in shared memory) and
//                       O += P V (P from TMEM), S of one tile of columns while the other one's weights are made
// TMEM: S of both tiles (columns 0 - 255; the weights P take the place of the scores they come from), O of both (256 - 511).
//
// f16 holds a code times its scale exactly, 3 and 8 bits, so keys and values lose nothing as long as they fit its exponents.  They are
// taken relative to a power of two: for the keys above the tile's largest scale, which goes back into the scores; for the values
// above the largest so far, and when that grows O is scaled down, as it is when a row's running maximum grows by more than 2^8 (rare).
// Exact are then all whose scale is not below 2^-28 of that, whether a row sees the largest one or not.  Two codes take an AND-OR
// (1024 + n), a packed multiply-add (n - 8) and a packed product with the scale.  (One multiply-add from the subnormal numbers that
// their bits are would do, but its results reach down to 2^-10 of the largest only.)
//
// Per 128 tokens and 256 columns of 128 channels: four products of 512 clocks at the tensor cores' rate (those for the scores take longer:
// both operands come from shared memory), 32768 exponentials at 16 a clock, 2048 clocks, and 8000 instructions, 2000 clocks.  Measured
// 2.5 us, 1.84 with the products alone, and 13 us to begin and end a block: 16384 tokens and 4096 columns of 8 heads 394 us (697
// TFLOP/s), two sequences of 1024 rows of 4 columns on 5120 tokens 262 us (1140 on the kernel for few rows).
//
// Scores, softmax and sums are fp32.  Weights are rounded to f16 (2^-11 of each, as in the kernel for few rows): what the products take.
#include "kv_attention.cuh"
#include "mx_common.cuh"

#include <algorithm>
#include <type_traits>

namespace lce {
namespace {

constexpr int kTokens = 128;                    // of a tile here: eight tiles of the cache
constexpr int kSoftmaxWarps = 8, kProducerWarps = 4, kIssuerWarp = kSoftmaxWarps + kProducerWarps;
constexpr int kThreads = 32 * (kIssuerWarp + 4);  // whole warpgroups: registers are shared out between them
// Registers a thread: 128 at the launch, 512 * 128 in all = 256 * 176 + 128 * 104 + 128 * 56.
constexpr int kSoftmaxRegisters = 176, kProducerRegisters = 104, kIssuerRegisters = 56;
static_assert(256 * kSoftmaxRegisters + 128 * kProducerRegisters + 128 * kIssuerRegisters <= kThreads * 128, "more registers than the block has");
constexpr float kRise = 8.0f;                   // a running maximum is raised when a score passes it by 2^8
constexpr float kHeadroom = 7.0f;               // weights are held times 2^7: 2^(7 + 8) is the most that meets f16
constexpr int kInfos = 4;                       // the producers are less than three tiles ahead of the softmax

enum { BAR_Q = 0, BAR_K_FULL, BAR_V_FULL = BAR_K_FULL + 2, BAR_K_EMPTY = BAR_V_FULL + 2, BAR_V_EMPTY = BAR_K_EMPTY + 2, BAR_S_FULL = BAR_V_EMPTY + 2,
       BAR_P_FULL = BAR_S_FULL + 2,
       BAR_P_REST = BAR_P_FULL + 2, BAR_DONE = BAR_P_REST + 2, BAR_COUNT };

// What the softmax has to know of a tile.
struct TileInfo {
    float key_unit;      // 2^e: scores count in it
    int32_t value_exponent;
    uint32_t valid;      // bit per 16 tokens: their page is in the pool
    uint32_t nan;        // some value's scale is NaN: see nans
};

struct Shared {
    uint64_t bars[BAR_COUNT];
    uint32_t tmem, largest[2][2][kProducerWarps];     // [turn][keys, values]
    TileInfo info[kInfos];
    alignas(16) __half key_scales[2][kTokens][4];     // relative to the tile's largest; [turn]
    alignas(16) __half value_scales[2][kTokens / 2][4][2];
    uint8_t nans[kInfos][kTokens];                    // blocks of a token's value that are NaN
};

constexpr int kMiscBytes = 8192;
static_assert(sizeof(Shared) <= kMiscBytes, "");
constexpr size_t prompt_smem(int blocks) { return kMiscBytes + 6 * (size_t)(kTokens * 64 * blocks); }

__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// Operand in shared memory without swizzle: 8 rows x 16 bytes are 128 bytes in a row, those of the next eight k behind them, those of the next
// eight rows `rows8` bytes on.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t rows8)
{
    return (uint64_t)(at >> 4) | (uint64_t)(128 >> 4) << 16 | (uint64_t)(rows8 >> 4) << 32 | 1ull << 46;
}

// 32 columns of this warp's 32 lanes of TMEM
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at)
        : "memory");
}
// 128 columns
__device__ __forceinline__ void tmem_load128(uint32_t at, uint32_t (&r)[128])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31"
        "}, [%128];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63"
        "}, [%129];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%64,%65,%66,%67,%68,%69,%70,%71,%72,%73,%74,%75,%76,%77,%78,%79,%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95"
        "}, [%130];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%96,%97,%98,%99,%100,%101,%102,%103,%104,%105,%106,%107,%108,%109,%110,%111,%112,%113,%114,%115,%116,%117,%118,%119,%120,%121,%122,%123,%124,%125,"
        "%126,%127"
        "}, [%131];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), 
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), 
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), 
          "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), 
          "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), 
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]), "=r"(r[64]), "=r"(r[65]), "=r"(r[66]), 
          "=r"(r[67]), "=r"(r[68]), "=r"(r[69]), "=r"(r[70]), "=r"(r[71]), "=r"(r[72]), "=r"(r[73]), "=r"(r[74]), "=r"(r[75]), "=r"(r[76]), "=r"(r[77]), 
          "=r"(r[78]), "=r"(r[79]), "=r"(r[80]), "=r"(r[81]), "=r"(r[82]), "=r"(r[83]), "=r"(r[84]), "=r"(r[85]), "=r"(r[86]), "=r"(r[87]), "=r"(r[88]), 
          "=r"(r[89]), "=r"(r[90]), "=r"(r[91]), "=r"(r[92]), "=r"(r[93]), "=r"(r[94]), "=r"(r[95]), "=r"(r[96]), "=r"(r[97]), "=r"(r[98]), "=r"(r[99]), 
          "=r"(r[100]), "=r"(r[101]), "=r"(r[102]), "=r"(r[103]), "=r"(r[104]), "=r"(r[105]), "=r"(r[106]), "=r"(r[107]), "=r"(r[108]), "=r"(r[109]), 
          "=r"(r[110]), "=r"(r[111]), "=r"(r[112]), "=r"(r[113]), "=r"(r[114]), "=r"(r[115]), "=r"(r[116]), "=r"(r[117]), "=r"(r[118]), "=r"(r[119]), 
          "=r"(r[120]), "=r"(r[121]), "=r"(r[122]), "=r"(r[123]), "=r"(r[124]), "=r"(r[125]), "=r"(r[126]), "=r"(r[127])
        : "r"(at), "r"(at + 32), "r"(at + 64), "r"(at + 96)
        : "memory");
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
                 "r"(r[6]), "r"(r[7]), "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]),
        "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at)
        : "memory");
}

// The B words of a place (a lane's of ROWS = 64 places, a token's of 16), plane by plane.
template <int B, int ROWS>
__device__ __forceinline__ void load_planes(const uint32_t *base, int place, uint32_t (&w)[B])
{
    if (B == 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(base) + place);
        w[0] = v.x; w[B > 1 ? 1 : 0] = v.y; w[B > 2 ? 2 : 0] = v.z; w[B > 3 ? 3 : 0] = v.w;
    } else {
        if (B & 2) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(base) + place);
            w[0] = v.x; w[B > 1 ? 1 : 0] = v.y;
        }
        if (B & 1) w[B - 1] = __ldg(base + ROWS * (B - 1) + place);
    }
}

__device__ __forceinline__ uint32_t half2_bits(__half2 v) { return *reinterpret_cast<const uint32_t *>(&v); }
__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<const __half2 *>(&v); }
// c s of the eight codes of a word, pair by pair: codes 0 and 4 (of the low and the high half), 1 and 5, 2 and 6, 3 and 7.
__device__ __forceinline__ uint4 decode(uint32_t word, __half2 scale)
{
    constexpr uint32_t kEven = 0x003c003cu, kOdd = 0x03c003c0u, kBase = 0x64006400u;
    const __half2 quarter = as_half2(0x34003400u), less264 = as_half2(0xdc20dc20u), part64 = as_half2(0x24002400u), less24 = as_half2(0xce00ce00u);
    const uint32_t other = swap_bytes(word);
    return make_uint4(half2_bits(__hmul2(__hfma2(as_half2(and_or(word, kEven, kBase)), quarter, less264), scale)),
                      half2_bits(__hmul2(__hfma2(as_half2(and_or(word, kOdd, kBase)), part64, less24), scale)),
                      half2_bits(__hmul2(__hfma2(as_half2(and_or(other, kEven, kBase)), quarter, less264), scale)),
                      half2_bits(__hmul2(__hfma2(as_half2(and_or(other, kOdd, kBase)), part64, less24), scale)));
}

__device__ __forceinline__ uint32_t key_scale(uint32_t word) { return word << 16; }  // as fp32 bits
__device__ __forceinline__ void producers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// The same, and whether all of them are well: where one's wait gave up, all leave together.
__device__ __forceinline__ bool producers_sync_and(bool ok)
{
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
        "bar.red.and.pred p, 1, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)ok)
        : "memory");
    return all != 0;
}

// mbar_wait_bounded in place: a kernel that calls a function cannot share its registers out.
__device__ __forceinline__ bool wait_bounded(uint64_t *bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    do {
#pragma unroll 1
        for (int i = 0; i < 32; ++i)
            if (mbar_try_wait(bar, parity)) return true;
    } while (globaltimer_ns() - t0 < kWaitLimitNs);
    return false;
}

// What a producer thread has of a tile before it decodes it.
template <int B>
struct Raw {
    uint32_t scales[B];          // of its token
    uint32_t keys[4][B], values[4][B];
    uint32_t valid;
};

// The page that lane l's tile of the cache, the l-th of eight, lies on; negative behind the sequence.  Only loaded here: what is done with
// it comes a tile later.
__device__ __forceinline__ int32_t find_page(const AttnParams &p, const int32_t *table, int length, int tile, int lane)
{
    const int32_t t = tile * 8 + lane;
    if (lane >= 8 || t >= (length + kKvTile - 1) / kKvTile) return -1;
    return __ldg(table + t / (p.g.page_size / kKvTile));
}

template <int B>
__device__ __forceinline__ void load_raw(const AttnParams &p, int32_t page, int head, int length, int tile, int thread, Raw<B> &r)
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
        if (at && tile * kTokens + thread < length) load_planes<B, 16>(at + 128 * B, thread & 15, r.scales);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int half = i * 4 + warp;
        const uint32_t *const at = tile_at(half >> 1);
#pragma unroll
        for (int b = 0; b < B; ++b) r.keys[i][b] = 0;
        if (at) load_planes<B, 64>(at, (half & 1) * 32 + (lane & 7) * 4 + (lane >> 3), r.keys[i]);
    }
    const uint32_t *const at = tile_at(thread >> 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int b = 0; b < B; ++b) r.values[i][b] = 0;
        if (at) load_planes<B, 64>(at + 64 * B, (thread >> 3 & 1) * 32 + (thread & 7) * 4 + i, r.values[i]);
    }
}

template <int B>
__global__ void __launch_bounds__(kThreads, 1) kv_prompt_kernel(const __grid_constant__ AttnParams p, const TimeoutReport report)
{
    constexpr uint32_t ROWS8_QK = 512 * B, ROWS8_V = 2048;   // bytes from eight rows to the next
    constexpr uint32_t TILE_BYTES = kTokens * 64 * B;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem);
    uint8_t *const q_smem = smem + kMiscBytes, *const k_smem = q_smem + 2 * TILE_BYTES, *const v_smem = k_smem + 2 * TILE_BYTES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    Unit u;
    int first_unit;
    if (p.join) release_join();
    // the last column tiles see most tokens and come first
    const int unit = p.units - 1 - (int)blockIdx.x;
    if (!find_unit<kPromptColumns, false>(p, unit, &u, &first_unit)) return;
    const int head = blockIdx.y;
    int32_t any_lo, any_hi, unused;
    const int columns = u.rows * p.group;
    column_range(p, u, u.column0, &any_lo, &unused);
    column_range(p, u, min(u.column0 + kPromptColumns, columns) - 1, &unused, &any_hi);
    // pieces are cut in tiles of the cache: at whole tiles of this kernel, each piece's end where the next one begins
    const int32_t tile0 = max(any_lo / kTokens, u.first ? 0 : u.tile0 * kKvTile / kTokens);
    const int32_t tiles = any_hi > any_lo ? max(min((any_hi + kTokens - 1) / kTokens, u.last ? 0x7fffffff : u.tile1 * kKvTile / kTokens) - tile0, 0) : 0;
    const int tiles_of_columns = u.column0 + 128 < columns ? 2 : 1;

    if (threadIdx.x == 0) {
        mbar_init(&sh.bars[BAR_Q], 32 * kSoftmaxWarps);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.bars[BAR_K_FULL + i], 32 * kProducerWarps);
            mbar_init(&sh.bars[BAR_V_FULL + i], 32 * kProducerWarps);
            mbar_init(&sh.bars[BAR_K_EMPTY + i], 1);
            mbar_init(&sh.bars[BAR_V_EMPTY + i], 1);
            mbar_init(&sh.bars[BAR_S_FULL + i], 1);
            mbar_init(&sh.bars[BAR_P_FULL + i], 128);
            mbar_init(&sh.bars[BAR_P_REST + i], 128);
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
        // ---- softmax: a thread to a column ------------------------------------------------------------
        const int half = warp >> 2, in_tile = threadIdx.x & 127, column = u.column0 + 128 * half + in_tile, row = column / p.group;
        int32_t lo, hi;
        column_range(p, u, column, &lo, &hi);
        float factor;
        {
            const int64_t at = (u.row0 + row) * p.q_token + ((int64_t)head * p.group + (column - row * p.group)) * p.q_head;
            int k = 0;
            bool finite = true;
            uint8_t *const to = q_smem + half * TILE_BYTES + (in_tile >> 3) * ROWS8_QK + (in_tile & 7) * 16;
            const auto take_row = [&](auto element, auto vectors) {
                using T = decltype(element);
                Eight<T> e[4 * B];  // the whole row at once
#pragma unroll
                for (int c = 0; c < 4 * B; ++c) e[c] = load_eight<T, decltype(vectors)::value>(static_cast<const T *>(p.q) + at + 8 * c, row < u.rows ? p.g.dim - 8 * c : 0);
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
                    // in the order in which a word's codes are decoded
                    *reinterpret_cast<uint4 *>(to + c * 128) = make_uint4(pack_half2(v[0] * s1 * s2, v[4] * s1 * s2), pack_half2(v[1] * s1 * s2, v[5] * s1 * s2),
                                                                          pack_half2(v[2] * s1 * s2, v[6] * s1 * s2), pack_half2(v[3] * s1 * s2, v[7] * s1 * s2));
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
            factor = (finite ? fabsf(p.scale) : __uint_as_float(0x7fc00000u)) * __uint_as_float((uint32_t)(127 + c1) << 23) * __uint_as_float((uint32_t)(127 + c2) << 23);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(&sh.bars[BAR_Q]);
        }
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16, s_at = tmem + lanes + 128 * half, o_at = tmem + lanes + 256 + 128 * half;
        float top = kLowest;
        uint64_t weight[2] = {};  // pairs of fp32 sums
        int32_t exponent = 0;
        uint32_t nan_blocks = 0;
        if (half < tiles_of_columns) {
            for (int j = 0; ok && j < tiles; ++j) {
                ok = __all_sync(0xffffffffu, wait_bounded(&sh.bars[BAR_S_FULL + half], j & 1));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const TileInfo info = sh.info[j % kInfos];
                const int32_t token0 = (tile0 + j) * kTokens;
                const float f = factor * info.key_unit;
                // bits of tokens that count, where not all do
                const bool all = __all_sync(0xffffffffu, info.valid == 0xffu && token0 >= lo && token0 + kTokens <= hi);
                uint32_t seen[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
                if (!all) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int32_t from = min(max(lo - (token0 + 32 * c), 0), 32), to = min(max(hi - (token0 + 32 * c), 0), 32);
                        const uint32_t below = to >= 32 ? 0xffffffffu : (1u << to) - 1, above = from >= 32 ? 0u : 0xffffffffu << from;
                        const uint32_t pages = (info.valid >> (2 * c) & 1 ? 0xffffu : 0u) | (info.valid >> (2 * c + 1) & 1 ? 0xffff0000u : 0u);
                        seen[c] = below & above & pages;
                    }
                }
                if (info.nan) {
                    for (int t = 0; t < kTokens; ++t)
                        if (seen[t >> 5] >> (t & 31) & 1) nan_blocks |= sh.nans[j % kInfos][t];
                }
                uint32_t r[kTokens];
                tmem_load128(s_at, r);
                if (!all) {
#pragma unroll
                    for (int i = 0; i < kTokens; ++i) r[i] = seen[i >> 5] >> (i & 31) & 1 ? r[i] : 0xff800000u;
                }
                float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < kTokens; ++i) tops[i & 3] = fmaxf(tops[i & 3], __uint_as_float(r[i]));
                float m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                m = m == -INFINITY ? m : m * f;
                // whole warps: the accumulators are read and written by warps
                if (__any_sync(0xffffffffu, m > top + kRise || exponent != info.value_exponent)) {
                    const float new_top = fmaxf(m, top), by = exp2f(top - new_top), by_o = by * exp2f((float)(exponent - info.value_exponent));
                    if (j > 0) {
#pragma unroll
                        for (int c = 0; c < 2 * B; ++c) {
                            float o[16];
                            tmem_ld16(o_at + 16 * c, o);
                            uint32_t x[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(o[i] * by_o);
                            tmem_store16(o_at + 16 * c, x);
                        }
                    }
                    weight[0] = mul_pair(weight[0], pair_of(by, by));
                    weight[1] = mul_pair(weight[1], pair_of(by, by));
                    top = new_top;
                    exponent = info.value_exponent;
                }
                const uint64_t f2 = pair_of(f, f), plus = pair_of(kHeadroom - top, kHeadroom - top);
                const bool masked = !all && !(f > 0.0f);  // 0, or what a row that is not finite has, times minus infinity
                // the first half of the weights is worked on while the second is made
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int t = 16 * c + 2 * i;
                        float x, y;
                        of_pair(fma_pair(pair_of(__uint_as_float(r[t]), __uint_as_float(r[t + 1])), f2, plus), x, y);
                        if (masked) {
                            x = r[t] == 0xff800000u ? -INFINITY : x;
                            y = r[t + 1] == 0xff800000u ? -INFINITY : y;
                        }
                        x = exp2_fast(x);
                        y = exp2_fast(y);
                        weight[i & 1] = add_pair(weight[i & 1], pair_of(x, y));
                        w[i] = pack_half2(x, y);
                    }
                    tmem_store8(s_at + 8 * c, w);
                    if (c == 3 || c == 7) {
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        mbar_arrive(&sh.bars[(c == 3 ? BAR_P_FULL : BAR_P_REST) + half]);
                    }
                }
            }
            if (ok && tiles > 0) ok = __all_sync(0xffffffffu, wait_bounded(&sh.bars[BAR_DONE], 0));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (ok) {
                float w0, w1, w2, w3;
                of_pair(weight[0], w0, w1);
                of_pair(weight[1], w2, w3);
                const float total = (w0 + w1) + (w2 + w3);
                const float by = (total == 0.0f ? 0.0f : 1.0f / total), scale_up = exp2f((float)(exponent - 11));
                constexpr int D = 32 * B;
                float *const part = p.parts + (((int64_t)unit * p.g.heads + head) * kPromptColumns + 128 * half + in_tile) * (D + 4);
                if (u.chunks > 1) *reinterpret_cast<float2 *>(part + D) = make_float2(top, total);
                const int64_t at = (u.row0 + row) * p.out_token + ((int64_t)head * p.group + (column - row * p.group)) * p.out_head;
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    uint32_t r[32];
                    if (tiles > 0) {
                        tmem_load32(o_at + 32 * b, r);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = 0;
                    }
                    // channel 4 g + i of the block is row 8 i + g of the product
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float x = total == 0.0f ? 0.0f : __uint_as_float(r[(i & 3) * 8 + 2 * c + (i >> 2)]) * scale_up * (u.chunks > 1 ? 1.0f : by);
                            v[i] = nan_blocks >> b & 1 ? __uint_as_float(0x7fc00000u) : x;
                        }
                        const int channel = 32 * b + 8 * c, count = row < u.rows ? p.g.dim - channel : 0;
                        if (u.chunks > 1) {
                            *reinterpret_cast<float4 *>(part + channel) = make_float4(v[0], v[1], v[2], v[3]);
                            *reinterpret_cast<float4 *>(part + channel + 4) = make_float4(v[4], v[5], v[6], v[7]);
                            continue;
                        }
                        if (p.type == LCE_TYPE_FLOAT16) {
                            __half *const out = static_cast<__half *>(p.out) + at + channel;
                            if (p.out_vectors) store8<__half, true>(out, count, v);
                            else store8<__half, false>(out, count, v);
                        } else {
                            __nv_bfloat16 *const out = static_cast<__nv_bfloat16 *>(p.out) + at + channel;
                            if (p.out_vectors) store8<__nv_bfloat16, true>(out, count, v);
                            else store8<__nv_bfloat16, false>(out, count, v);
                        }
                    }
                }
            }
        }
    } else if (warp < kIssuerWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProducerRegisters));
        // ---- keys and values: from 4 bits to f16 operands ------------------------------------------------
        const int thread = threadIdx.x - 32 * kSoftmaxWarps, producer = warp - kSoftmaxWarps;
        const int32_t *const table = p.page_table + (int64_t)u.seq * p.table_pages;
        const int32_t held = tokens_held(p, u.length);
        Raw<B> even_raw, odd_raw;
        int32_t page = -1;  // two tiles ahead; words one
        if (tiles > 0) {
            load_raw<B>(p, find_page(p, table, held, tile0, lane), head, held, tile0, thread, even_raw);
            page = find_page(p, table, held, tile0 + 1, lane);
        }
        int32_t value_exponent = -1000;
        // One tile; false where a wait gave up.
        const auto produce = [&](int j, const Raw<B> &raw, Raw<B> &next) -> bool {
            if (j + 1 < tiles) load_raw<B>(p, page, head, held, tile0 + j + 1, thread, next);
            page = find_page(p, table, held, tile0 + j + 2, lane);
            const int stage = j & 1, turn = j & 1;
            // the largest scales of the tile (bits of bf16 numbers compare like integers; a NaN does not count)
            uint32_t nan = 0, top_k = 0, top_v = 0;
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const uint32_t ks = key_scale(raw.scales[b]), vs = raw.scales[b] & 0xffff0000u;
                if (ks < 0x7f800000u) top_k = max(top_k, ks);
                if (vs < 0x7f800000u) top_v = max(top_v, vs);
                else nan |= 1u << b;
            }
            top_k = __reduce_max_sync(0xffffffffu, top_k);
            top_v = __reduce_max_sync(0xffffffffu, top_v);
            const uint32_t some_nan = __ballot_sync(0xffffffffu, nan != 0);
            if (lane == 0) {
                sh.largest[turn][0][producer] = top_k;
                sh.largest[turn][1][producer] = top_v | (some_nan ? 1u : 0u);
            }
            ok = producers_sync_and(ok);
            if (!ok) return false;
            top_k = top_v = 0;
            uint32_t any_nan = 0;
#pragma unroll
            for (int i = 0; i < kProducerWarps; ++i) {
                top_k = max(top_k, sh.largest[turn][0][i]);
                any_nan |= sh.largest[turn][1][i] & 1u;
                top_v = max(top_v, sh.largest[turn][1][i] & 0xffff0000u);
            }
            const int key_exponent = max((int)(top_k >> 23) - 127, -100);
            const int here = max((int)(top_v >> 23) - 127, -100);
            if (top_v > 0 && here > value_exponent) value_exponent = here + 1;  // one more, so that it does not move often
            const int ve = max(value_exponent, -100);
            // relative scales, below 2^12: 7 of them fit
            const float k_by = __uint_as_float((uint32_t)(127 + 11 - key_exponent) << 23), v_by = __uint_as_float((uint32_t)(127 + 11 - ve) << 23);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const float vs = __uint_as_float(raw.scales[b] & 0xffff0000u);
                sh.key_scales[turn][thread][b] = __float2half_rn(__uint_as_float(key_scale(raw.scales[b])) * k_by);
                sh.value_scales[turn][thread >> 1][b][thread & 1] = __float2half_rn(nan >> b & 1 ? 0.0f : vs * v_by);
            }
            if (any_nan) sh.nans[j % kInfos][thread] = (uint8_t)nan;
            if (thread == 0) sh.info[j % kInfos] = TileInfo{__uint_as_float((uint32_t)(127 + key_exponent) << 23), ve, raw.valid, any_nan};
            producers_sync();
            if (j >= 2) ok = wait_bounded(&sh.bars[BAR_K_EMPTY + stage], (j >> 1 & 1) ^ 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int unit = i * 4 + producer, token = unit * 8 + (lane & 7), quarter = lane >> 3;
                uint8_t *const to = k_smem + stage * TILE_BYTES + unit * ROWS8_QK + quarter * 128 + (lane & 7) * 16;
                const uint2 scales = *reinterpret_cast<const uint2 *>(sh.key_scales[turn][token]);
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const __half2 scale = as_half2(__byte_perm(b & 2 ? scales.y : scales.x, 0, b & 1 ? 0x3232 : 0x1010));
                    *reinterpret_cast<uint4 *>(to + b * 512) = decode(raw.keys[i][b], scale);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(&sh.bars[BAR_K_FULL + stage]);
            if (j >= 2) ok = wait_bounded(&sh.bars[BAR_V_EMPTY + stage], (j >> 1 & 1) ^ 1) && ok;
            {
                const int eighth = thread & 7, group = thread >> 3;  // eight tokens
                uint8_t *const to = v_smem + stage * TILE_BYTES + group * 128 + eighth * 16;
                uint4 scales[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) scales[t] = *reinterpret_cast<const uint4 *>(sh.value_scales[turn][group * 4 + t]);
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    uint4 w[4];  // [pair of tokens]: its four channels
#pragma unroll
                    for (int t = 0; t < 4; ++t) w[t] = decode(raw.values[t][b], as_half2(b == 0 ? scales[t].x : b == 1 ? scales[t].y : b == 2 ? scales[t].z : scales[t].w));
                    // channel 4 eighth + i of the block is row 8 i + eighth of the operand
                    *reinterpret_cast<uint4 *>(to + (4 * b + 0) * ROWS8_V) = make_uint4(w[0].x, w[1].x, w[2].x, w[3].x);
                    *reinterpret_cast<uint4 *>(to + (4 * b + 1) * ROWS8_V) = make_uint4(w[0].y, w[1].y, w[2].y, w[3].y);
                    *reinterpret_cast<uint4 *>(to + (4 * b + 2) * ROWS8_V) = make_uint4(w[0].z, w[1].z, w[2].z, w[3].z);
                    *reinterpret_cast<uint4 *>(to + (4 * b + 3) * ROWS8_V) = make_uint4(w[0].w, w[1].w, w[2].w, w[3].w);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(&sh.bars[BAR_V_FULL + stage]);
            return true;
        };
        for (int j = 0; j < tiles; j += 2) {
            if (!produce(j, even_raw, odd_raw)) break;
            if (j + 1 < tiles && !produce(j + 1, odd_raw, even_raw)) break;
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssuerRegisters));
    }
    if (warp == kIssuerWarp && lane == 0 && tiles > 0) {
        // ---- the products ---------------------------------------------------------------------------------
        constexpr uint32_t kCommon = 1u << 4 | (uint32_t)(128 >> 4) << 24;  // fp32 sums of f16 products, both operands along k, 128 rows
        const uint32_t idesc_s = kCommon | (uint32_t)(kTokens >> 3) << 17, idesc_o = kCommon | (uint32_t)(32 * B >> 3) << 17;
        const uint32_t q_at = smem_u32(q_smem), k_at = smem_u32(k_smem), v_at = smem_u32(v_smem);
        const auto scores = [&](int half, int stage) {
#pragma unroll
            for (int k = 0; k < 2 * B; ++k)
                mma_shared(tmem + 128 * half, operand(q_at + half * TILE_BYTES + k * 256, ROWS8_QK), operand(k_at + stage * TILE_BYTES + k * 256, ROWS8_QK), idesc_s, k > 0);
        };
        const auto sums = [&](int half, int stage, int part, bool add) {
#pragma unroll
            for (int k = 4 * part; k < 4 * part + 4; ++k)
                mma_tmem(tmem + 256 + 128 * half, tmem + 128 * half + 8 * k, operand(v_at + stage * TILE_BYTES + k * 256, ROWS8_V), idesc_o, add || k > 0);
        };
        ok = wait_bounded(&sh.bars[BAR_Q], 0) && wait_bounded(&sh.bars[BAR_K_FULL], 0);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (ok) {
            for (int half = 0; half < tiles_of_columns; ++half) {
                scores(half, 0);
                mma_commit(&sh.bars[BAR_S_FULL + half]);
            }
            mma_commit(&sh.bars[BAR_K_EMPTY]);
        }
        for (int j = 0; ok && j < tiles; ++j) {
            const int stage = j & 1, next = stage ^ 1;
            ok = wait_bounded(&sh.bars[BAR_V_FULL + stage], j >> 1 & 1);
            if (ok && j + 1 < tiles) ok = wait_bounded(&sh.bars[BAR_K_FULL + next], (j + 1) >> 1 & 1);
            for (int half = 0; ok && half < tiles_of_columns; ++half) {
                ok = wait_bounded(&sh.bars[BAR_P_FULL + half], j & 1);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                sums(half, stage, 0, j > 0);
                ok = wait_bounded(&sh.bars[BAR_P_REST + half], j & 1);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                sums(half, stage, 1, true);
                if (j + 1 < tiles) {  // in order behind the sums, which read the weights in its place
                    scores(half, next);
                    mma_commit(&sh.bars[BAR_S_FULL + half]);
                }
            }
            if (!ok) break;
            mma_commit(&sh.bars[BAR_V_EMPTY + stage]);
            if (j + 1 < tiles) mma_commit(&sh.bars[BAR_K_EMPTY + next]);
        }
        // whatever happened: nothing is in flight when the tensor memory goes
        mma_commit(&sh.bars[BAR_DONE]);
        if (!wait_bounded(&sh.bars[BAR_DONE], 0)) ok = false;
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

// Joins the pieces of the columns, always in the same order: a warp to a column, eight columns to a block.
template <int B>
__global__ void __launch_bounds__(256) kv_prompt_join_kernel(const __grid_constant__ AttnParams p)
{
    constexpr int D = 32 * B;
    Unit u;
    int first_unit;
    const bool found = find_unit<kPromptColumns, true>(p, blockIdx.x, &u, &first_unit);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // every block: what comes behind this kernel relies on the one in front, too
    const int head = blockIdx.y, in_tile = blockIdx.z * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (!found) return;
    const int column = u.column0 + in_tile, row = column / p.group;
    if (row >= u.rows) return;
    const int64_t step = (int64_t)p.g.heads * kPromptColumns * (D + 4);
    const float *const from = p.parts + (((int64_t)first_unit * p.g.heads + head) * kPromptColumns + in_tile) * (D + 4);
    const int chunks = min(u.chunks, p.units - first_unit);
    float top = -INFINITY;
    for (int i = lane; i < chunks; i += 32) top = fmaxf(top, from[i * step + D]);
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    float sum[B] = {}, weight = 0.0f;
#pragma unroll 4
    for (int i = 0; i < chunks; ++i) {
        const float f = exp2f(from[i * step + D] - top);
        weight = fmaf(f, from[i * step + D + 1], weight);
#pragma unroll
        for (int b = 0; b < B; ++b) sum[b] = fmaf(f, from[i * step + 32 * b + lane], sum[b]);
    }
    const int64_t at = (u.row0 + row) * p.out_token + ((int64_t)head * p.group + (column - row * p.group)) * p.out_head;
#pragma unroll
    for (int b = 0; b < B; ++b)
        if (32 * b + lane < p.g.dim) store_element(p.out, p.type, at + 32 * b + lane, weight == 0.0f ? 0.0f : sum[b] / weight);
}

template <int B>
lce_status launch(const AttnParams &p, const TimeoutReport &report, cudaStream_t s)
{
    static SmemOptIn opt_in;
    if (!opt_in.ensure(kv_prompt_kernel<B>, prompt_smem(B))) return LCE_ERR_CUDA;
    const lce_status st = launch_dependent(kv_prompt_kernel<B>, dim3((unsigned)p.units, (unsigned)p.g.heads), kThreads, prompt_smem(B), s, p, report);
    if (st != LCE_OK || !p.join) return st;
    return launch_dependent(kv_prompt_join_kernel<B>, dim3((unsigned)std::min(p.column_tiles, p.target), (unsigned)p.g.heads, kPromptColumns / 8), 256, 0, s, p);
}

}  // namespace

lce_status launch_kv_prompt(const AttnParams &p, cudaStream_t s)
{
    if (tensor_timeout_flagged()) return LCE_ERR_DEVICE_TIMEOUT;
    const TimeoutReport report = tensor_timeout_report(s);
    if (!report.device_word) return LCE_ERR_CUDA;
    switch (p.g.blocks) {
        case 1: return launch<1>(p, report, s);
        case 2: return launch<2>(p, report, s);
        case 3: return launch<3>(p, report, s);
        default: return launch<4>(p, report, s);
    }
}

}  // namespace lce
