// Which kernel the grouped product with experts in 4 bits takes.  Plain code: the rule is checked without a GPU.  The tiles of all sizes
// add in the same order; the split sum has another.
#pragma once

#include <cstdint>

namespace sida {

// The sum over K split over a workgroup's wavefronts, or tiles of 32 x 128, 64 x 256 or (tokens in 4 bits) 128 x 256 tokens and columns.
enum class MxTiles { split, rows32, rows64, rows128 };

inline MxTiles mx_tiles(bool x4, int64_t M, int64_t groups, int64_t N, int64_t K)
{
    // The sum over K split over a workgroup, or 128 columns to a workgroup and K in one go.  The first takes 3.3 us for each round of 256
    // stripes (1 token, 4096 x 1024: 6.2 us against 17.5; 16 tokens of 64 experts, 4096 x 1024, 512 stripes: 11.9 against 19.9), the second 4.5 us and
    // 0.2 for each 64 of K in up to a thousand stripes (8 tokens of 8 experts, 768 x 3072, 768 stripes: 6.7 us against 10.4;
    // 64 of 64, 3072 x 768, 1536 stripes: 20.6 against 27.0).
    if ((M / 32 + (groups < M ? groups : M)) * ((N + 31) / 32) <= K / 4) return MxTiles::split;
    // Tile height and width, by how many rows a group has on average and how many tiles of 64 x 256 there would be (1024 of them, four to a
    // compute unit, are a round).  us, 32 x 128 against 64 x 256, 64 groups, K x N: tokens in bf16, 48 a group, 768 x 3072 27.3 / 22.6, 64 a group,
    // 1024 x 1024 16.6 / 18.0, 3072 x 768 29.8 / 41.6, 128 a group 48.9 / 44.8; in 4 bits, 24 a group, 768 x 3072 16.2 / 15.7, 32 a
    // group, 4096 x 1024, Zipf sizes, 28.3 / 29.7, 64 a group 34.2 / 30.8.
    const int64_t mean = M / groups, wide = (M / 64 + groups / 2) * ((N + 255) / 256);
    if (x4 ? mean <= 16 || wide < 320 : mean <= 32 || wide < 480) return MxTiles::rows32;
    // 128 x 256 for long rows in 4 bits: 256 tokens for each of 128 groups, 4096 x 1024, 109 us against 122; with rows of 768 three stages
    // are a tile's whole sum, and two workgroups to a compute unit too few (256 a group, 64 groups, 43.0 against 38.1).
    return x4 && K >= 2048 && mean >= 192 ? MxTiles::rows128 : MxTiles::rows64;
}

}  // namespace sida
