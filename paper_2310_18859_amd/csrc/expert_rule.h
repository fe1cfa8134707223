// How the operators of plain bf16 experts cut up their work.  Plain code: the rules are checked without a GPU.
#pragma once

#include <cstdint>

namespace sida {

// ---- sort: pairs of a workgroup (a multiple of 1024), and workgroups; at most 256 of them up to 2^31 pairs
constexpr int kExpertSortChunks = 256;
inline int expert_sort_chunk(int64_t pairs)
{
    if (pairs <= 4096) return 4096;
    const int64_t c = (pairs + kExpertSortChunks - 1) / kExpertSortChunks;
    return (int)(c <= 2048 ? 2048 : (c + 1023) / 1024 * 1024);
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

// ---- products: values between two rows at most, so that 256 rows span less than 2^31 bytes
constexpr int64_t kMostExpertPitch = 1 << 22;

// Which tiles the products of rows take, rows x columns: 32 x 32 with the sum shared by a workgroup's wavefronts, 32 x 128, 64 x 256, 128 x 128 (two
// workgroups to a compute unit), 256 x 256 (one).
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

// ---- the weights' gradient: rows of a part (0: a group's rows are summed in one go).  Parts of 128 x 128 tiles where tiles of whole groups would leave
// compute units idle, of as many rows as give each of the 512 workgroup slots one.
inline int64_t expert_tiles_of(int64_t N, int64_t K, int64_t side) { return ((N + side - 1) / side) * ((K + side - 1) / side); }
inline bool expert_weights_small(int64_t groups, int64_t N, int64_t K) { return groups * expert_tiles_of(N, K, 256) < 256; }
inline int expert_weights_chunk(int64_t M, int64_t groups, int64_t N, int64_t K)
{
    if (!expert_weights_small(groups, N, K)) return 0;
    const int64_t parts = 512 / expert_tiles_of(N, K, 128) - groups / 2;
    if (parts <= groups) return 0;
    const int64_t rows = (M / parts + 63) / 64 * 64;
    return rows < 256 ? (M > 512 * groups ? 256 : 0) : rows >= M / groups ? 0 : (int)rows;
}
inline int64_t expert_weights_parts(int64_t M, int64_t groups, int64_t chunk) { return M / chunk + (groups < M ? groups : M); }

}  // namespace sida
