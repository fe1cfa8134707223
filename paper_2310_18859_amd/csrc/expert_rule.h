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

// ---- rows: lanes of a token (or pair), 8 to 64; of more than 2^26 - 4 of them at most 32, as a launch has fewer than 2^32 threads in whole workgroups of 256
inline int rows_lanes_log2(int pieces, int64_t tokens = 0)
{
    int l = 3;
    while (l < 6 && 1 << l < pieces) ++l;
    return l == 6 && tokens > (1 << 26) - 4 ? 5 : l;
}

// ---- products: bytes between two rows at most, so that 256 rows span less than 2^31
constexpr int64_t kMostExpertPitch = 1 << 23;

// Which tiles the products of rows take, rows x columns: 32 x 32 with the sum shared by a workgroup's wavefronts, 32 x 128, 64 x 256, 128 x 128 (two
// workgroups to a compute unit), 256 x 256 (one).  us for each as product and as input's gradient, sizes as groups, rows of each (17: Zipf 1.2), length of
// the sum, columns; one run on one card:
//     groups  rows  length  columns       few        32x128      64x256     128x128     256x256
//          8   1/8    1024     4096     8.5    7.5   12    11    15    15    13    12    16    15
//         64    17    1024     2048   114    125     58    62    61    64    52    56    58    58
//         64    32    1024     4096   222    259    102   115   104    97   106   111   107    98
//         64    64    4096     1024   219    248    124   133   136   112   130   112   134    98
//         64   128    1024     4096   665    729    289   323   144   138   129   135   134   121
//         64   256    1024     4096  1269   1362    582   645   217   221   203   209   167   162
//         64   512    4096     1024  1465   1626    672   788   384   382   311   315   260   258
//          1  4096    1024     1024    74     80     27    25    20    20    18    18    31    30
//          1  4096    1024     4096   289    318     87    83    47    48    44    43    39    39
// `few`, a workgroup to a compute unit, against 32 x 128, by the number of its tiles that M and the groups allow.  Groups of one row each, weights out of memory:
//     columns  length     256          384          512          640          768         1024         1280
//        4096    1024    8.4  12.6   13.0  12.9   14.1  13.2   19.0  13.5   19.9  14.8   27.3  17.0   31.5  22.1      product
//        4096    4096     16    31     27    33     36    37     40    42     43    49     64    63     68    77
//        4096    8192     23    54     44    58     51    64     67    77     74    91     96   117    117   150
//        4096    1024    9.0  12.0   14.6  12.8   16.1  13.4   20.4  14.4   21.8  15.7   28.8  18.9   33.3  23.5      input's gradient
//        4096    4096     21    30     33    32     40    33     45    35     52    40     78    51     81    75
//        4096    8192     28    50     57    57     76    60     80    64     94    75    141    96    145   145
// Rows that fill half of their tiles or more make fewer of them than M and the groups allow (groups x rows, few and 32 x 128; length 4096, columns 1024 to 4096):
//     product   8 x 16, 384 tiles: 17 and 31; 8 x 16, 768: 37 and 38; 1 x 128, 640: 28 and 31; 1 x 192, 896: 38 and 31
//     input     8 x 16, 384 tiles: 24 and 34; 4 x 32, 512: 25 and 35; 1 x 128, 640: 36 and 31; 8 x 16, 768: 48 and 36
// So the product takes `few` for more tiles the longer the sum, and the input's gradient, whose transposing reads take longer, for two rounds of workgroups at most.
// 256 x 256 wants its tiles to fill the compute units once at least, and four times where groups of fewer than 400 rows leave
// their last tile half empty.
enum class ExpertTiles { few, rows32, rows64, square128, rows256 };
inline ExpertTiles expert_tiles(int64_t M, int64_t groups, int64_t cols, int64_t length, bool input = false)
{
    const int64_t active = groups < M ? groups : M, mean = M / groups;
    auto tiles = [&](int64_t rows, int64_t width) { return (M / rows + active) * ((cols + width - 1) / width); };
    const int64_t most = 256 + length / 8;
    if (tiles(32, 32) <= (input && most > 512 ? 512 : most)) return ExpertTiles::few;
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
// kItemsInARow at most, fewer where there are few items: from 8 to 4096 made no difference beyond that of two runs, nor did staggered starts.  Nobody's turn depends on
// what the items cost: where they are uneven, so are the workgroups' shares.
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
