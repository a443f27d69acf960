// What the kernels of attention over the 4-bit cache share: the call's parameters, which piece of it a block works on, small helpers.
#pragma once
#include "kv_common.cuh"

namespace lce {

constexpr float kLowest = -1e30f;

struct AttnParams {
    KvGeom g;
    int32_t batch, group, table_pages, table_tokens;
    int32_t causal, window, type;
    int32_t q_vectors, out_vectors;    // eight channels of q, of out are one access
    int64_t tokens;
    int64_t q_token, q_head, out_token, out_head;
    float scale;                       // times log2(e)
    int32_t least_exponent;            // of the scales' reference, in the kernel for few rows
    const void *q;
    const uint32_t *cache;
    const int32_t *page_table, *lengths, *q_starts;
    void *out;
    float *parts;                      // [unit][kv head][column][32 blocks + 4]: sums, largest, weight
    int32_t units, column_tiles, target, least_tiles;
    int32_t cluster;                   // blocks that share a unit
    int32_t solo;                      // a warp to a unit and head: many short sequences
    int32_t join;                      // there may be units that are not a whole column tile
    int32_t prompt;                    // the kernel for prompts
    int32_t one_row;                   // each sequence has one row of q
};

// What a unit (a range of tiles for one tile of columns of a sequence) works on.
struct Unit {
    int32_t seq, column0, chunks;
    int32_t length, rows;                             // tokens of the sequence, which its rows' positions follow from; its rows of q
    int64_t row0;                                     // its first row of q
    int32_t tile0, tile1;                             // the unit's tiles
    bool first, last;                                 // piece of its column tile
};

struct Sequence {
    int32_t length, rows, column_tiles, first_tile, tiles;
    int64_t row0;
};

// Tokens of a sequence that its row of the page table can hold; those behind are masked.
__device__ __forceinline__ int32_t tokens_held(const AttnParams &p, int32_t length) { return min(length, p.table_tokens); }

template <int COLUMNS>
__device__ __forceinline__ Sequence sequence(const AttnParams &p, int b)
{
    Sequence s{};
    if (b >= p.batch) return s;
    s.length = max(__ldg(p.lengths + b), 0);
    s.row0 = b;
    s.rows = 1;
    if (p.q_starts) {
        const int64_t from = min(max((int64_t)__ldg(p.q_starts + b), (int64_t)0), p.tokens), to = min(max((int64_t)__ldg(p.q_starts + b + 1), from), p.tokens);
        s.row0 = from;
        s.rows = (int32_t)(to - from);
    }
    s.column_tiles = (int32_t)(((int64_t)s.rows * p.group + COLUMNS - 1) / COLUMNS);
    // tiles that some row sees
    const int32_t held = tokens_held(p, s.length);
    int32_t low = 0;
    if (p.window > 0) low = (int32_t)min(max((int64_t)s.length - s.rows + 1 - p.window, (int64_t)0), (int64_t)held);
    s.first_tile = low / kKvTile;
    s.tiles = (held + kKvTile - 1) / kKvTile - s.first_tile;
    return s;
}

// The work is cut evenly whatever the sequences' lengths: every column tile of a sequence into pieces of at most `most` tiles, where
// `most` follows from the whole batch's tiles.  Every warp works this out for itself from the lengths (no launch in front, no host
// copy of them).  Finds the `at`-th unit, or the first unit of the `at`-th column tile that is in pieces; false: there is no such one.
template <int COLUMNS, bool IN_PIECES>
__device__ __forceinline__ bool find_unit(const AttnParams &p, int at, Unit *u, int *first_unit)
{
    const int lane = threadIdx.x & 31;
    if (!p.join && !p.q_starts) {
        // a row for each sequence, and whole column tiles: no search
        const int32_t column_tiles = (p.group + COLUMNS - 1) / COLUMNS, seq = at / column_tiles;
        if (seq >= p.batch) return false;
        const Sequence s = sequence<COLUMNS>(p, seq);
        u->seq = seq;
        u->chunks = 1;
        u->length = s.length;
        u->rows = 1;
        u->row0 = seq;
        u->column0 = (at - seq * column_tiles) * COLUMNS;
        u->tile0 = s.first_tile;
        u->tile1 = s.first_tile + s.tiles;
        u->first = u->last = true;
        *first_unit = at;
        return true;
    }
    const Sequence first = sequence<COLUMNS>(p, lane);
    int64_t total = 0;
    if (p.join) {
        total = (int64_t)first.column_tiles * first.tiles;
#pragma unroll 4
        for (int b0 = 32; b0 < p.batch; b0 += 32) {
            const Sequence s = sequence<COLUMNS>(p, b0 + lane);
            total += (int64_t)s.column_tiles * s.tiles;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    }
    int32_t most = 1 << 30;
    if (p.join) {
        most = total < (1ll << 31) ? (int32_t)(((uint32_t)total + p.target - 1) / p.target) : (int32_t)min((total + p.target - 1) / p.target, (int64_t)most);
        most = max(most, p.least_tiles);
    }
    int before = 0, units_before = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const Sequence s = b0 ? sequence<COLUMNS>(p, b0 + lane) : first;
        const int32_t chunks = max((s.tiles + most - 1) / most, 1), units = s.column_tiles * chunks, mine = !IN_PIECES ? units : chunks > 1 ? s.column_tiles : 0;
        int32_t upto = mine, units_upto = units;  // of this and the lanes below
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t o = __shfl_up_sync(0xffffffffu, upto, d), n = __shfl_up_sync(0xffffffffu, units_upto, d);
            if (lane >= d) {
                upto += o;
                units_upto += n;
            }
        }
        const uint32_t has = __ballot_sync(0xffffffffu, before + upto > at);
        if (has) {
            const int from = __ffs(has) - 1;
            const int32_t local = at - (before + __shfl_sync(0xffffffffu, upto - mine, from));
            u->seq = b0 + from;
            u->chunks = __shfl_sync(0xffffffffu, chunks, from);
            u->length = __shfl_sync(0xffffffffu, s.length, from);
            u->rows = __shfl_sync(0xffffffffu, s.rows, from);
            u->row0 = __shfl_sync(0xffffffffu, s.row0, from);
            const int32_t tiles = __shfl_sync(0xffffffffu, s.tiles, from), first_tile = __shfl_sync(0xffffffffu, s.first_tile, from);
            const int32_t column_tile = IN_PIECES ? local : local / u->chunks, chunk = IN_PIECES ? 0 : local - column_tile * u->chunks;
            u->column0 = column_tile * COLUMNS;
            *first_unit = units_before + __shfl_sync(0xffffffffu, units_upto - units, from) + column_tile * u->chunks;
            // equal pieces
            const int32_t each = tiles / u->chunks, more = tiles - each * u->chunks;
            u->tile0 = first_tile + chunk * each + min(chunk, more);
            u->tile1 = u->tile0 + each + (chunk < more ? 1 : 0);
            u->first = chunk == 0;
            u->last = chunk == u->chunks - 1;
            return true;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
        units_before += __shfl_sync(0xffffffffu, units_upto, 31);
    }
    return false;
}

// Tokens [lo, hi) that the row of a column sees; none for a column that does not exist.
__device__ __forceinline__ void column_range(const AttnParams &p, const Unit &u, int column, int32_t *lo, int32_t *hi)
{
    const int32_t row = column / p.group;
    *lo = *hi = 0;
    if (row >= u.rows) return;
    const int64_t position = (int64_t)u.length - u.rows + row;
    const int32_t held = tokens_held(p, u.length);
    *hi = p.causal ? (int32_t)min(max(position + 1, (int64_t)0), (int64_t)held) : held;
    *lo = p.window > 0 ? (int32_t)min(max(position + 1 - p.window, (int64_t)0), (int64_t)held) : 0;
}

__device__ __forceinline__ void store_element(void *p, int32_t type, int64_t i, float v)
{
    switch (type) {
        case LCE_TYPE_FLOAT32: static_cast<float *>(p)[i] = v; return;
        case LCE_TYPE_FLOAT16: static_cast<__half *>(p)[i] = __float2half_rn(v); return;
        default: static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v); return;
    }
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float half_low(uint32_t v) { return __half2float(__ushort_as_half((unsigned short)(v & 0xffffu))); }
__device__ __forceinline__ float half_high(uint32_t v) { return __half2float(__ushort_as_half((unsigned short)(v >> 16))); }
__device__ __forceinline__ float exp2_fast(float x)
{
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
    return d;
}

// a & mask | with
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t with)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "r"(mask), "r"(with));
    return d;
}
// Bytes exchanged in either half.
__device__ __forceinline__ uint32_t swap_bytes(uint32_t w) { return __byte_perm(w, 0, 0x2301); }
// Lets the join, which this call launches behind, take its place while this kernel runs.  It waits for all of it, and nothing
// that a caller launches can start before the join is done.
__device__ __forceinline__ void release_join() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Prompts: kv_prompt.cu.  16-bit rows of up to 128 channels; `units` column tiles of kPromptColumns.
constexpr int kPromptColumns = 256;
lce_status launch_kv_prompt(const AttnParams &p, cudaStream_t s);

}  // namespace lce
