// What the kernels of the attention weights by token share: the call's parameters and which piece of a sequence a block works on.
#pragma once
#include "kv_attention.cuh"

namespace lce {

constexpr int kMostTiles = 256;   // of a piece: its tokens' sums are in shared memory
constexpr int kLeastTiles = 4;    // that a piece is worth

struct WeightsParams : AttnParams {
    float decay;
    int64_t previous_seq, previous_head, out_seq, out_head;
    const float *previous;
    float *sums;                            // where the weights go
    float2 *stats;                          // [kv head][row * group + query head][piece]: largest, sum
    float *scores;                          // [kv head], then each sequence's [token][columns, rounded up to an even number]; or null
    int64_t scores_head;
    int32_t pieces;                         // that a sequence can have
};

// A range of tiles of a sequence.
struct Piece {
    Unit u;                // columns [column0, ..): set by the loops over them
    int32_t index, pieces; // which one of the sequence's
    int32_t columns;
    int64_t scores_before; // scores of the sequences in front
};

// Between a token's scores and the next one's: pairs of them are one access.
__host__ __device__ __forceinline__ constexpr int scores_stride(int columns) { return (columns + 1) & ~1; }

// Finds the `at`-th piece; false: there is no such one.  Every warp works this out from the lengths: pieces of at most `most` tiles, where
// `most` follows from the whole batch's.
__device__ __forceinline__ bool find_piece(const WeightsParams &p, int at, Piece *piece)
{
    const int lane = threadIdx.x & 31;
    const auto tiles_of = [&](const Sequence &s) { return (tokens_held(p, s.length) + kKvTile - 1) / kKvTile; };
    const Sequence first = sequence<8>(p, lane);
    int64_t total = tiles_of(first);
    for (int b0 = 32; b0 < p.batch; b0 += 32) total += tiles_of(sequence<8>(p, b0 + lane));
#pragma unroll
    for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    const int32_t most = (int32_t)min(max((total + p.target - 1) / p.target, (int64_t)kLeastTiles), (int64_t)kMostTiles);
    int32_t before = 0;
    int64_t scores_before = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const Sequence s = b0 ? sequence<8>(p, b0 + lane) : first;
        const int32_t tiles = tiles_of(s), pieces = (tiles + most - 1) / most;
        const int64_t scores = (int64_t)tiles * kKvTile * scores_stride(s.rows * p.group);
        int32_t upto = pieces;
        int64_t scores_upto = scores;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            const int64_t n = __shfl_up_sync(0xffffffffu, scores_upto, d);
            if (lane >= d) {
                upto += o;
                scores_upto += n;
            }
        }
        const uint32_t has = __ballot_sync(0xffffffffu, before + upto > at);
        if (has) {
            const int from = __ffs(has) - 1;
            const int32_t n = __shfl_sync(0xffffffffu, tiles, from);
            piece->pieces = __shfl_sync(0xffffffffu, pieces, from);
            piece->index = at - (before + __shfl_sync(0xffffffffu, upto - pieces, from));
            piece->scores_before = scores_before + __shfl_sync(0xffffffffu, scores_upto - scores, from);
            piece->u.seq = b0 + from;
            piece->u.length = __shfl_sync(0xffffffffu, s.length, from);
            piece->u.rows = __shfl_sync(0xffffffffu, s.rows, from);
            piece->u.row0 = __shfl_sync(0xffffffffu, s.row0, from);
            piece->u.column0 = 0;
            piece->columns = piece->u.rows * p.group;
            // more scores than there is room for: rows of q that are several sequences' (q_starts that decrease); none are taken then
            if (p.scores && piece->scores_before + __shfl_sync(0xffffffffu, scores, from) > p.scores_head) piece->columns = 0;
            const int32_t each = n / piece->pieces, more = n - each * piece->pieces;  // equal pieces
            piece->u.tile0 = piece->index * each + min(piece->index, more);
            piece->u.tile1 = piece->u.tile0 + each + (piece->index < more ? 1 : 0);
            return true;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
        scores_before += __shfl_sync(0xffffffffu, scores_upto, 31);
    }
    return false;
}

// Tiles of the piece that some column of [column0, column0 + count) sees: columns' ranges move up with the rows.  all_lo, all_hi: tokens that
// each of them sees.
struct View {
    int32_t tile0, tile1, all_lo, all_hi;
};
__device__ __forceinline__ View view(const WeightsParams &p, const Piece &piece, int count)
{
    View v;
    int32_t any_lo, any_hi;
    column_range(p, piece.u, piece.u.column0, &any_lo, &v.all_hi);
    column_range(p, piece.u, min(piece.u.column0 + count, piece.columns) - 1, &v.all_lo, &any_hi);
    v.tile0 = max(piece.u.tile0, any_lo / kKvTile);
    v.tile1 = min(piece.u.tile1, (any_hi + kKvTile - 1) / kKvTile);
    if (any_hi <= any_lo) v.tile1 = v.tile0;
    return v;
}

// What stood there before, as far as it counts, and the weight w of token t.
__device__ __forceinline__ void put_weight(const WeightsParams &p, const Unit &u, int head, int32_t t, float w)
{
    if (p.previous && t < u.length - u.rows) w = fmaf(p.decay, p.previous[u.seq * p.previous_seq + head * p.previous_head + t], w);
    p.sums[u.seq * p.out_seq + head * p.out_head + t] = w;
}

// Many rows: kv_weights_prompt.cu.  16-bit rows of up to 128 channels; a workspace of so many bytes, 16-byte aligned.
size_t kv_weights_prompt_bytes(const WeightsParams &p);
lce_status launch_kv_weights_prompt(const WeightsParams &p, void *workspace, cudaStream_t s);

}  // namespace lce
