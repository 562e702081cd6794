// Causal attention of packed prompt chunks over the paged cache.
//
// The g = q_heads / kv_heads query heads of a kv head are stacked on the tokens: row r of a sequence's
// m g rows is token r / g, head r % g. A tile is tile_rows() of these rows; a wave holds 32 of them as the
// columns of its products, in registers from first to last:
//   S^T = K Q^T    on 32x32 tiles; a lane holds 16 scores of one query per 32 tokens
//   O^T = V^T P^T  the lane's scores are this product's operand as they stand: entries 8 s .. 8 s + 7 are
//                  tokens 16 s + 4 half + {0 .. 3} and 16 s + 8 + 4 half + {0 .. 3}, which over both lane
//                  halves are the 16 tokens of one K-step once; v comes from LDS in that order, by the
//                  transposing 64-bit LDS reads (one value per lane in float32 above 128 values a head).
// So the softmax needs one exchange between lanes per step (the maximum of the two halves), and the
// rescale of O is one factor per lane. K and V steps of TOK tokens go through LDS, shared by the
// waves, in two buffers: the next step's loads are in flight while the present one is computed.
//
// Work: the plan kernel lists (tile, range of tokens) items so that no item is longer than a share of
// the whole work (that of one place, tile_places(), or half of it); tiles behind a long cache are cut into several items
// whose partial results (m, l and the unnormalised o, float32) a third kernel joins in order. Items are
// listed longest first, and the workgroups of one item's kv heads are neighbours.
//
// Bound by instructions beside the MFMAs: 8192 tokens, 32 heads of 128 in bf16, 524 us a call of many in a row, 1.05
// PFLOP/s (535 to 641 for the kernel in a trace of ten), with the matrix cores' pipe 56% busy (a large library
// product reaches 1.65); three prompts of 2048 tokens in all, one behind 4096, 16 heads of 112: 36 us, the plan and
// the join 7 and 8; 33 tokens behind 40000 in fp8, 32 heads of 128: 52 us, and 16 for those two.
#pragma once
#include "kv.h"

namespace ssm {

// Rows of a tile: 32 for each of 4 waves, or of 8 for heads of 97 to 128 values where the tiles of 256 rows are
// one for every compute unit and more. Kernel and join, 8 and 4 waves: 32 heads of 128, 8192 tokens 526 and 568
// us, 4096 tokens 152 and 171; 16 heads of 112, 4096 tokens 104 and 107, three prompts of 2048 tokens in all, one
// behind 4096, 57 and 43. Heads of 64 values, 16 of them, 6000 tokens: 114 and 108.
inline int tile_rows(bool bf16_act, int DP, int64_t rows_heads) { return bf16_act && DP == 128 && rows_heads >= 65536 ? 256 : 128; }
constexpr int kStep = 64;          // the plan counts tokens in steps of this many
// Workgroups that run at once: two on a compute unit where their registers and LDS allow it (PrefillShape)
inline int tile_places(bool bf16_act, int rows, int DP) { return rows == 128 && DP <= (bf16_act ? 128 : 96) ? 512 : 256; }
// The least that the longest item's steps are limited to: what steps take (1 to 2 us one of bf16, twice that above 128
// values a head, 4 to 5 of float32) against the join. A tile above it is cut evenly (9 steps at 8: 5 and 4). Ten sequences of 1 to 7 rows, the longest behind 3059 tokens, 16 heads
// of 256: 8 steps 37 us, 4 30, 2 29; 8 of 64 fp8, 2745 tokens: 26, 23, 22; eight prompts of 28 to 441 rows, 20 of
// 80 fp8: 23, 31, 34. Float32, nine calls of up to 2500 rows, mean: 4 steps 26.6 us, 2 25.6, 1 25.9.
constexpr int tile_min_steps(bool bf16_act, int DP) { return !bf16_act ? 2 : DP <= 128 ? 8 : 4; }

// Tokens [k0, k1) for the tile at row0 of a sequence whose rows begin at lo (m tokens, n cached).
// part: its partial result; -1: the item is the whole tile; -2: no item
struct AttnItem { int32_t seq, row0, k0, k1, part, lo, m, n; };
struct AttnJoin { int32_t row0, part, pieces, lo, m, pad[3]; };
struct AttnPlan {
    int32_t* count;      // joins
    int32_t* prefix;     // [nseq + 1] tiles before each sequence
    AttnItem* items;
    AttnJoin* joins;
    float* parts;        // [Hkv][max_parts][rows (DP + 2)]
    int rows, places, min_steps, max_tiles, max_items, max_joins, max_parts;
    size_t total;
};
// sizes for up to T rows of nseq sequences
inline AttnPlan attn_plan(bool bf16_act, int Hq, int Hkv, int DP, int64_t T, int nseq, char* base) {
    AttnPlan p{};
    p.rows = tile_rows(bf16_act, DP, T * Hq);
    const int64_t tiles = (T * (Hq / Hkv) + p.rows - 1) / p.rows + nseq;
    // cut tiles have more steps than a share of the work: their number and their items' are bounded by it
    p.places = tile_places(bf16_act, p.rows, DP);
    p.min_steps = tile_min_steps(bf16_act, DP);
    const int64_t share = (p.places * (bf16_act ? 1 : 2) + Hkv - 1) / Hkv + 1;
    p.max_tiles = (int)tiles;
    p.max_items = (int)(tiles + share);
    p.max_joins = (int)(tiles < share ? tiles : share);
    p.max_parts = (int)(2 * share);
    size_t off = 0;
    auto take = [&](size_t bytes) { char* q = base ? base + off : nullptr; off += align256(bytes); return q; };
    p.count = (int32_t*)take(16);
    p.prefix = (int32_t*)take((size_t)(nseq + 1) * 4);
    p.items = (AttnItem*)take((size_t)p.max_items * sizeof(AttnItem));
    p.joins = (AttnJoin*)take((size_t)p.max_joins * sizeof(AttnJoin));
    p.parts = (float*)take((size_t)Hkv * p.max_parts * p.rows * (DP + 2) * 4);
    p.total = off;
    return p;
}

template <typename T, int FMT, int DP>
hipError_t launch_attn_prefill_tile(const AttnArgs& p, const AttnPlan& pl, hipStream_t s);

}  // namespace ssm
