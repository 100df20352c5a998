// Matmuls in 8-bit integers: which kernel a launch takes, and its grid.
#pragma once
#include "i8_ops.h"

namespace ftk {

// I8_STREAM: tiles of 16 x 16 (16 x 32 with gates) straight from memory into the matrix cores (i8_gemm.hip); the others pass through LDS
// (i8_blocks.hip), I8_64x64 with two groups of waves along the reduce axis.
enum I8Kind { I8_STREAM, I8_64x64, I8_64x128, I8_128x128, I8_128x256, I8_256x256, I8_KINDS };

struct I8KindInfo {
    uint32_t tm, tn, per_cu;             // tile, workgroups that a CU holds
    // microseconds of a launch: once, for each round of tiles, for each k-tile of 128 of a round; for all tiles that there are over
    // those of a round, and for each k-tile of theirs.  The first kind of a round's cost is latency, which is there however
    // few its tiles are; the second is what they share: the caches' bandwidth and the power.
    float once, round, round_k, tile, tile_k;
};
// Least squares over 348 shapes, m 8 .. 32768, n 768 .. 11008, k 64 .. 4096, all kinds measured at each (bf16 results, rows on whole blocks, an idle device): the times
// are met to 5 .. 13 % (root of the mean square), and at those shapes the kind with the least is within 0.3 % of the fastest on average, 10 % at most.  Gates, a bias, fp32
// results and longer reduce axes go by the same numbers, and results whose rows begin anywhere too, which cost a third more (403 x 1003 x 1001: 7.4 us for 5.7).
constexpr I8KindInfo kI8Kinds[I8_KINDS] = {
    {16, 16, 1, 2.60f, 0.11f, 0.101f, 0.13f, 0.000f},
    {64, 64, 1, 2.92f, 1.22f, 0.141f, 0.57f, 0.053f},
    {64, 128, 2, 2.63f, 1.49f, 0.233f, 0.85f, 0.306f},
    {128, 128, 2, 3.30f, 0.60f, 0.426f, 2.93f, 0.422f},
    {128, 256, 1, 2.93f, 2.37f, 0.458f, 1.87f, 0.349f},
    {256, 256, 1, 2.15f, 5.08f, 0.710f, 2.90f, 0.707f},
};
inline I8KindInfo i8_kind_info(I8Kind kind, bool gated) {
    I8KindInfo i = kI8Kinds[kind];
    if (kind == I8_STREAM && gated) i.tn = 32, i.tile *= 2.f, i.tile_k *= 2.f;      // twice the columns
    return i;
}

// Rows of tiles, about, where experts have different numbers of rows: each that has any ends in a tile that is half full on average.
inline float i8_row_tiles(const I8Args &a, uint32_t tm, bool grouped) {
    if (!grouped) return (float)((a.m + tm - 1u) / tm);
    const float used = (float)(a.experts < a.m ? a.experts : a.m), full = (float)a.m / (float)tm + 0.5f * used;
    return full > used ? full : used;
}
inline float i8_time(const I8Args &a, I8Kind kind, bool grouped) {
    const I8KindInfo i = i8_kind_info(kind, a.gated != 0);
    const float row_tiles = i8_row_tiles(a, i.tm, grouped), tiles = row_tiles * (float)((a.n + i.tn - 1u) / i.tn), share = tiles / (float)(a.cus * i.per_cu);
    const float k = (float)((a.k + 127u) / 128u);
    float rounds = (float)(uint64_t)share;
    if (rounds < share) rounds += 1.f;
    // By expert a tile first reads where its rows lie, then their numbers: a microsecond more.  Blocks ask for the next tile's ahead; the first kind
    // waits anew once for what a CU holds, four workgroups, two with gates (4 tokens, 2 of 16 experts, 2816 x 2048 gated: 11.0 us in three
    // rounds of the first kind, 10.5 in one of the third, which are expected at 8.5 and 9.8 without this).
    const float held = kind == I8_STREAM ? (a.gated ? 2.f : 4.f) : rounds, waits = grouped ? (float)(uint64_t)((rounds + held - 1.f) / held) : 0.f;
    // ... and each row of tiles reads its expert's weights, which other rows of tiles seldom find in the caches: 10 us a GB (32 products of 256 .. 65536
    // entries and 8 .. 64 experts, all kinds measured: the chosen one is 1.3 % slower than the fastest on average, without this term 3.1 %).
    const float weights = grouped ? 1e-8f * row_tiles * (float)a.n * (float)a.k : 0.f;
    return i.once + waits + weights + rounds * (i.round + i.round_k * k) + share * (i.tile + i.tile_k * k);
}
inline I8Kind i8_choose(const I8Args &a, bool grouped) {
    I8Kind best = I8_STREAM;
    float least = i8_time(a, best, grouped);
    for (int k = 1; k < I8_KINDS; ++k) {
        const float t = i8_time(a, (I8Kind)k, grouped);
        if (t < least) { least = t; best = (I8Kind)k; }
    }
    return best;
}

// The grid of a launch in tiles of tm x tn; false: more workgroups than a launch has.  By expert the rows of tiles are the most there can
// be: all tiles full but the last of each expert.
inline bool i8_grid(I8Args &a, uint32_t tm, uint32_t tn, bool grouped) {
    const uint64_t rows = grouped ? (uint64_t)a.m / tm + (a.experts < a.m ? a.experts : a.m) : ((uint64_t)a.m + tm - 1) / tm;
    a.col_tiles = (a.n + tn - 1) / tn;
    if (rows * a.col_tiles > 0x7fffffffull) return false;
    a.row_tiles = (uint32_t)rows;
    const uint32_t band = tm >= 256 ? 4u : tm >= 128 ? 8u : 16u;       // rows of tiles that are walked together
    a.group = a.row_tiles < band ? a.row_tiles : band;
    return true;
}

// Where the t-th turn of `groups` k-tiles, one for each group of waves, begins.  `first`: through a long reduce axis every XCD goes from another of its `whole`
// whole turns on, and round to there (a last turn that the axis ends inside stays the last one).  This is the copies' scalar offset, always inside the axis; the
// groups' tiles of a turn are 128 bytes apart in the lanes' offsets, so that one beyond the axis is held to the buffer's bound: that is compared with the
// lanes' offsets, less the scalar one, which must not pass it (a tile of one row can end before the second group's last tile begins).
constexpr uint32_t i8_turn_begin(uint32_t t, uint32_t groups, uint32_t first, uint32_t whole) {
    const uint32_t x = t + first;
    return (t >= whole ? t : x >= whole ? x - whole : x) * groups * 128u;
}

ft_status i8_launch_blocks(I8Kind kind, bool grouped, I8Args &a, void *stream);

}  // namespace ftk
