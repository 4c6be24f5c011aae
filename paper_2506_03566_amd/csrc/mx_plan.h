// How the products with microscaled weights run: which kernel, with which tiles, in how many K splits.  Host code only.
#pragma once
#include <math.h>

namespace poss {

// How a product runs: a kernel with its tile shape, and K splits.  Chosen by an estimate of the time in us: for each shape the sum of eight
// terms whose weights were fitted (none negative) to times measured in graphs, 19 row counts (1 to 4096) x 10 matrices (512 x 512 to
// 28672 x 4096 and 5120 x 13824) x up to ten splits.  What the estimate picks is 0.9 % slower on average than the fastest of all that was
// measured; of 190 sizes 7 (microscaled X: 6) are more than a tenth slower, a fifth at most.  Where the shapes cross (4096 x 4096, us): 16
// rows stream 6.2, 16 x 64 7.0; 128 rows 16 x 64 10.3, 32 x 128 11.1; 244 rows 32 x 128 13.7, 64 x 128 15.1; 512 rows 64 x 128 20.0, 64 x 256
// 24.8; 1024 rows 43.0 and 31.5; 4096 rows 64 x 256 121, 256 x 256 108.
constexpr int MX_GROUP = 512;      // columns of a group of k-steps: what K is split in
struct MxPlan { int shape, splits; };
struct MxTile { int tm, tn; float us[8]; };
enum { MX_STREAM = 0 };
constexpr int CHIP_CUS = 256;
// us: a launch; k-groups of a tile; the same times rounds of the chip (256 tiles); ... times tiles / 256; rounds; planes: their launch, a million
// of their values; a million results.  The first row (no tiles): a launch; sixteen k-groups; 10^4 column x k-groups; the same times a hundred rows.
constexpr MxTile MX_TILES[] = {
    {16, 16, {2.407f, 0.851f, 0.417f, 6.06f}},                                       // mx_stream_kernel
    {16, 64, {1.920f, 0.493f, 0.021f, 0.218f, 0.879f, 2.158f, 0.769f, 0.686f}},      // mx_fed_kernel
    {32, 128, {2.557f, 0.434f, 0.179f, 0.604f, 1.368f, 1.809f, 1.034f, 1.411f}},
    {32, 256, {3.053f, 0.778f, 0.285f, 0.959f, 2.049f, 1.233f, 1.156f, 1.376f}},
    {64, 128, {2.855f, 0.000f, 1.160f, 0.657f, 1.158f, 2.713f, 1.373f, 0.771f}},
    {64, 256, {4.774f, 0.000f, 1.850f, 1.065f, 0.000f, 2.511f, 1.524f, 0.827f}},
    {256, 256, {7.758f, 0.096f, 8.969f, 1.422f, 0.107f, 1.133f, 0.896f, 0.854f}}};   // mx_tile_kernel
constexpr MxTile MX_BOTH_TILES[] = {
    {16, 16, {2.334f, 0.381f, 0.347f, 2.44f}},                                       // mx_stream_both_kernel
    {16, 64, {1.337f, 0.748f, 0.000f, 0.193f, 0.782f, 2.452f, 0.836f, 0.462f}},      // mx_fed_both_kernel
    {32, 128, {1.353f, 0.881f, 0.000f, 0.331f, 1.418f, 2.265f, 1.356f, 1.889f}},
    {64, 128, {2.659f, 0.354f, 0.539f, 0.262f, 1.552f, 2.436f, 1.456f, 0.903f}},
    {64, 256, {4.124f, 0.105f, 1.079f, 0.327f, 0.000f, 2.889f, 1.496f, 0.698f}},
    {256, 256, {6.552f, 0.000f, 2.005f, 1.094f, 4.886f, 4.424f, 1.030f, 0.407f}}};   // mx_block_both_kernel

static inline int mx_groups(int K) { return (K - 1) / MX_GROUP + 1; }      // K > 0
// Waves of a column tile: four, sixteen where the tiles leave CUs with one each and K is long (one row, us, 4 / 8 / 16 waves: 4096 x 14336 9.0 / 8.5 / 8.0,
// 5120 x 13824 10.8 / 12.0 / 12.2, 6144 x 4096 5.4 / 5.7, 4096 x 4096 3.4 / 3.6).
static inline int stream_waves(int tiles, int kgroups) { return tiles <= 256 && kgroups >= 16 ? 16 : kgroups < 4 ? kgroups : 4; }

// fixed > 0: the number of splits, for a context's layers.  Those are not streamed: there mx_stream_kernel would have a wave per split, not the four or sixteen
// that its weights were fitted with, and weights come from HBM, not the last cache (one row, us, streamed / 16 x 64 tiles: 6144 x 2048 2 splits 5.0 / 5.3,
// 4096 x 4096 4 splits 5.3 / 5.4, 6144 x 4096 2 splits 7.6 / 7.2, 15360 x 5120 unsplit 15.7 / 13.3, 4096 x 14336 4 splits 11.7 / 10.1, 5120 x 13824 3 splits
// 15.8 / 12.3; ten rows 6.2 / 5.4 to 23.6 / 12.4).  Plain decoding in the 8B and 13B shapes, ms, with streaming where the estimate had it / without: 2.24 / 2.17,
// 3.15 / 3.01.
template <int SHAPES> static inline MxPlan best_plan(const MxTile (&tiles)[SHAPES], int M, int N, int groups, int fixed = 0) {
    MxPlan best{MX_STREAM, 1};
    float least = 1e30f;
    if (M <= 16 && fixed == 0) {
        const float *u = tiles[MX_STREAM].us, ng = (float)N * groups * 1e-4f;
        least = u[0] + u[1] * groups / 16 + u[2] * ng + u[3] * ng * M * 1e-2f;
    }
    const float mn = (float)M * N * 1e-6f;
    for (int i = 1; i < SHAPES; ++i) {
        const MxTile &t = tiles[i];
        const float n = (float)((M + t.tm - 1) / t.tm) * (float)((N + t.tn - 1) / t.tn);
        if (n > 4e6f && i + 1 < SHAPES) continue;         // (a launch has fewer than 2^32 threads)
        for (int s = fixed > 0 ? fixed : 1; s <= (fixed > 0 ? fixed : 16) && s <= groups && (fixed > 0 || s == 1 || n * s <= 1024); ++s) {
            const float g = (float)((groups + s - 1) / s), chips = n * s / 256, rounds = ceilf(chips);
            float us = t.us[0] + t.us[1] * g + t.us[2] * g * rounds + t.us[3] * g * chips + t.us[4] * rounds + t.us[7] * mn;
            if (s > 1) us += t.us[5] + t.us[6] * s * mn;
            if (us < least) { least = us; best = MxPlan{i, s}; }
        }
    }
    return best;
}
// both: microscaled X; parts: 3 of float32 X, otherwise 1.
static inline MxPlan mx_plan_of(bool both, int parts, int M, int N, int K) {
    return both ? best_plan(MX_BOTH_TILES, M, N, mx_groups(K)) : best_plan(MX_TILES, M, N, mx_groups(K) * parts);
}

// For a context's layers.
// Splits of a matrix whose planes the layer's own epilogues add up: as many as give half the CUs a 128-column tile (a tree's rows are two
// tiles of 32), two where the columns alone give a quarter of them one, none where they give more than three quarters of them one; the groups dealt
// out evenly.  They follow the matrix alone, and every kernel adds a split's products in the same order: a row's sums do not depend on the rows beside
// it, and a tree's rows get what plain decoding gives them.  Rounds of 61 rows and plain decoding, ms: 8B shape 4.39 and 2.16, 13B shape 5.28 and 2.91;
// twice as many of the splits below the last line 4.58 and 2.16, 5.40 and 2.88, half as many 4.61 and 2.32, 5.48 and 3.04.  That line, rounds, two
// splits / none: 16 layers whose QKV, gate and up have 160 to 180 column tiles 2.56 / 2.58, 192 tiles 2.62 / 2.64; gate and up of 224 (8B) 4.46 / 4.39, of
// 216 (13B) 5.32 / 5.28.
static inline int mx_plane_splits(int N, int K) {
    const int groups = mx_groups(K), cols = (N + 127) / 128;
    int s = cols > CHIP_CUS * 3 / 4 ? 1 : cols > CHIP_CUS / 4 ? 2 : CHIP_CUS / 2 / cols;
    if (s > groups) s = groups;
    if (s > 16) s = 16;
    if (s < 1) s = 1;
    const int longest = (groups + s - 1) / s;
    return (groups + longest - 1) / longest;
}

}  // namespace poss
