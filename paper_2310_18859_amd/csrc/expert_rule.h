// How the operators of plain bf16 experts cut up their work.  Plain code for host and device: the rules are checked without a GPU.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define SIDA_HD __host__ __device__ __forceinline__
#else
#define SIDA_HD inline
#endif

namespace sida {

// ---- sort: pairs of a workgroup (a multiple of 1024), and workgroups; at most 256 of them up to 2^31 pairs.  Up to 4096 pairs are one workgroup and one launch.
constexpr int kExpertSortChunks = 256;
inline int expert_sort_chunk(int64_t pairs)
{
    if (pairs <= 4096) return 4096;
    const int64_t c = (pairs + kExpertSortChunks - 1) / kExpertSortChunks;
    return (int)(c <= 2048 ? 2048 : (c + 1023) / 1024 * 1024);
}
inline int64_t expert_sort_most(int64_t pairs)                // workgroups that this many pairs or fewer need
{
    const int64_t c = (pairs + 2047) / 2048;
    return pairs <= 4096 ? 1 : c < kExpertSortChunks ? c : kExpertSortChunks;
}
inline int expert_sort_chunks(int64_t pairs)
{
    const int64_t c = expert_sort_chunk(pairs);
    return pairs <= c ? 1 : (int)((pairs + c - 1) / c);
}

// ---- rows: a token's lanes, 8 to 64
inline int rows_lanes_log2(int pieces)
{
    int l = 3;
    while (l < 6 && 1 << l < pieces) ++l;
    return l;
}

// ---- products: bytes between two rows at most, so that 256 rows span less than 2^31
constexpr int64_t kMostExpertPitch = 1 << 23;

// Which tiles the products of rows take, rows x columns: 32 x 32 with the sum shared by a workgroup's wavefronts, 32 x 128, 64 x 256, 128 x 128 (two
// workgroups to a compute unit), 256 x 256 (one).  us for each, sizes as groups, mean rows of a group, length of the sum, columns:
//     groups  rows  length  columns     few   32x128  64x256  128x128  256x256
//          8   1/8    1024     4096     6.2     11.5    14.8     12.7     16.2
//         64    17    1024     2048   137       61      64       60       83
//         64    32    1024     4096   318      132     120      125      142
//         64    64    4096     1024   254      155     137      159      222
//         64   128    1024     4096   795      339     191      173      186
//         64   256    1024     4096  1450      643     307      266      249
//         64   512    4096     1024  2773     1249     598      503      405
//          1  4096    1024     1024    79       27.5    22       21       37.5
//          1  4096    1024     4096   329      130      54       54       45
// `few`: as long as its tiles are one round of workgroups, more of them the longer the sum that is shared.  256 x 256 wants its tiles to fill the compute
// units once at least, and four times where groups of fewer than 400 rows leave their last tile half empty.
enum class ExpertTiles { few, rows32, rows64, square128, rows256 };
inline ExpertTiles expert_tiles(int64_t M, int64_t groups, int64_t cols, int64_t length)
{
    const int64_t active = groups < M ? groups : M, mean = M / groups;
    auto tiles = [&](int64_t rows, int64_t width) { return (M / rows + active) * ((cols + width - 1) / width); };
    if (tiles(32, 32) <= 256 + length / 8) return ExpertTiles::few;
    if (mean <= 24 || tiles(128, 128) <= 200) return ExpertTiles::rows32;
    if (mean <= 96) return ExpertTiles::rows64;
    return mean >= 256 && tiles(256, 256) >= (mean >= 400 ? 256 : 1024) ? ExpertTiles::rows256 : ExpertTiles::square128;
}

// Workgroups of `few`, one for each of the tiles that M rows in `groups` groups have at most, in eights.
inline int64_t expert_few_grid(int64_t M, int64_t groups, int64_t cols)
{
    return ((M / 32 + (groups < M ? groups : M)) * ((cols + 31) / 32) + 7) / 8 * 8;
}

// The items that workgroup b of `workgroups` (a multiple of 8) takes one after the other, of n: b runs on XCD b % 8, and an XCD takes `block` items in a row of
// every eight times as many, so that a row tile's rows and a group's matrix are fetched into few L2s while all XCDs get their share of large and small tiles.
// kItemsInARow at most, fewer where there are few items: from 8 to 4096 made no difference beyond that of two runs, nor did staggered starts.
// Workgroups that take one item only need an eighth of all items to an XCD: with shorter runs the last, incomplete eight of them are partly second items.
constexpr int kItemsInARow = 64, kFewInARow = INT32_MAX;
struct Items {
    int total, block, xcd, at, step;
    SIDA_HD Items(int64_t n, int workgroups, int most, int b) : total((int)n), xcd(b & 7), at(b >> 3), step(workgroups >> 3)
    {
        const int rounds = (int)((n + workgroups - 1) / workgroups);
        const int64_t even = rounds ? (n + 8 * rounds - 1) / (8 * rounds) : 1;
        block = (int)(most < even ? most : even);
    }
    SIDA_HD int next()                                        // -1: none
    {
        const int id = at / block * 8 * block + xcd * block + at % block;
        at += step;
        return id < total ? id : -1;
    }
};

// ---- the weights' gradient: rows of a part (0: a group's rows are summed in one go).  Parts of 128 x 128 tiles where tiles of whole groups would leave
// compute units idle, of as many rows as give each of the 512 workgroup slots one: with 384, 512, 768 and 1024 slots counted 4 experts of 520 x 264 and 16385
// rows take 27.4, 28.5, 30.2 and 34.0 us (133 without parts), one of 1024 x 1024 and 4096 rows 32.5, 31.7, 35.7 and 43.8.
inline int64_t expert_tiles_of(int64_t N, int64_t K, int64_t side) { return ((N + side - 1) / side) * ((K + side - 1) / side); }
inline bool expert_weights_small(int64_t groups, int64_t N, int64_t K) { return groups * expert_tiles_of(N, K, 256) < 256; }
inline int64_t expert_weights_most(int64_t groups, int64_t N, int64_t K) { return 512 / expert_tiles_of(N, K, 128) - groups / 2; }
inline int expert_weights_chunk(int64_t M, int64_t groups, int64_t N, int64_t K)
{
    // Twice as many parts as groups at least: they are written and read again (8 groups of 1024 rows, 1024 x 512: 24.1 us whole, 36.9 in 12 parts).
    if (!expert_weights_small(groups, N, K) || expert_weights_most(groups, N, K) < 2 * groups) return 0;
    const int64_t most = expert_weights_most(groups, N, K), rows = ((M + most - 1) / most + 63) / 64 * 64;
    if (rows >= 256) return (int)rows;
    return M > 512 * groups ? 256 : 0;
}
inline int64_t expert_weights_parts(int64_t M, int64_t groups, int64_t chunk) { return M / chunk + (groups < M ? groups : M); }

}  // namespace sida
