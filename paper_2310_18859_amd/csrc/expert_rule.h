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

}  // namespace sida
