// Grouped product of token rows with experts in MXFP4:  y[r,:] = W_g x[r,:] for the rows r of group g.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "kernels.h"

namespace sida {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

struct MxArgs {
    const char *x;               // token rows
    const uint8_t *x_scales;
    const char *codes;           // experts, fragment order
    const char *scales;
    const int32_t *offsets;      // NULL: one group of M rows
    void *y;
    int64_t ldx, ldy;            // values between rows
    int64_t code_bytes, scale_bytes;   // between experts
    int M, N, K, groups;
};

// Which rows tile `mt` of BM rows is: tiles are counted group by group.  Every wavefront finds it for itself, four groups to
// a lane; rows = 0 where there are fewer tiles.
struct TokenTile {
    int group, row0, rows;
};
template <int BM>
__device__ __forceinline__ TokenTile find_tile(const MxArgs &a, int mt)
{
    if (!a.offsets) return TokenTile{0, mt * BM, max(0, min(BM, a.M - mt * BM))};
    const int lane = threadIdx.x & 63;
    int at[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) at[i] = max(0, min(a.M, a.offsets[min(lane * 4 + i, a.groups)]));
    int tiles = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) tiles += (max(0, at[i + 1] - at[i]) + BM - 1) / BM;
    int before = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(before, d);
        if (lane >= d) before += v;
    }
    const uint64_t later = __ballot(before > mt);
    if (later == 0) return TokenTile{0, 0, 0};
    const int owner = __builtin_ctzll(later);
    int left = mt - (before - tiles), group = 0, row0 = 0, rows = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = (max(0, at[i + 1] - at[i]) + BM - 1) / BM;
        if (left >= 0 && left < n) {
            group = lane * 4 + i;
            row0 = at[i] + left * BM;
            rows = min(BM, at[i + 1] - row0);
        }
        left -= n;
    }
    return TokenTile{__builtin_amdgcn_readfirstlane(__shfl(group, owner)), __builtin_amdgcn_readfirstlane(__shfl(row0, owner)),
                     __builtin_amdgcn_readfirstlane(__shfl(rows, owner))};
}

// Eight codes times their power of two, exact in bf16.
__device__ __forceinline__ bf16x8 decode(uint32_t c, float s)
{
    bf16x8 o;
    *(reinterpret_cast<bf16x2 *>(&o) + 0) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
    *(reinterpret_cast<bf16x2 *>(&o) + 1) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
    *(reinterpret_cast<bf16x2 *>(&o) + 2) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
    *(reinterpret_cast<bf16x2 *>(&o) + 3) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
    return o;
}

__device__ __forceinline__ float relu_of(float v) { return v <= 0.f ? 0.f : v; }   // NaN stays

// One wavefront: 32 tokens x 32 columns, operands straight from memory.
template <bool X4, class Y, bool RELU>
__global__ __launch_bounds__(256) void mx_gemm_simple(const MxArgs a)
{
    const int lane = threadIdx.x & 63, half = lane >> 5, stripe = blockIdx.y * 4 + (threadIdx.x >> 6);
    const TokenTile t = find_tile<32>(a, blockIdx.x);
    if (t.rows == 0 || stripe * 32 >= a.N) return;
    const int steps = (a.K + 63) / 64;
    const char *w = a.codes + t.group * a.code_bytes + (size_t)stripe * steps * 1024 + lane * 16;
    const char *ws = a.scales + t.group * a.scale_bytes + (size_t)stripe * ((a.K + 255) / 256) * 256 + lane * 4;
    const int row = t.row0 + min(lane & 31, t.rows - 1);
    const int pitch = (a.K + 255) / 256 * 8;
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0;
    for (int s = 0; s < steps; ++s) {
        const i32x4 c = *reinterpret_cast<const i32x4 *>(w + (size_t)s * 1024);
        const uint32_t scale = (uint8_t)ws[(s / 4) * 256 + s % 4];
        const int k = s * 64 + half * 32;
        const bool in = k < a.K;
        if constexpr (X4) {
            i32x4 x = {0, 0, 0, 0};
            uint32_t xs = 127;
            if (in) {
                x = *reinterpret_cast<const i32x4 *>(a.x + (size_t)row * (a.K / 2) + k / 2);
                xs = a.x_scales[(size_t)row * pitch + k / 32];
            }
            const i32x8 c8 = {c[0], c[1], c[2], c[3], 0, 0, 0, 0}, x8 = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(c8, x8, acc, 4, 4, 0, scale, 0, xs);
        } else {
            const float f = __builtin_bit_cast(float, scale << 23);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x8 x;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = (__bf16)0.f;
                if (in) x = *reinterpret_cast<const bf16x8 *>(a.x + ((size_t)row * a.ldx + k + q * 8) * 2);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode(c[q], f), x, acc, 0, 0, 0);
            }
        }
    }
    if ((lane & 31) >= t.rows) return;
    Y *y = (Y *)a.y + (size_t)row * a.ldy;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int col = stripe * 32 + 8 * (r / 4) + 4 * half + r % 4;
        if (col < a.N) y[col] = (Y)(RELU ? relu_of(acc[r]) : acc[r]);
    }
}

template <bool X4, class Y>
int launch_typed(const MxArgs &a, bool relu, hipStream_t st)
{
    const dim3 grid(a.M / 32 + (a.groups < a.M ? a.groups : a.M), (a.N + 127) / 128);
    if (relu) mx_gemm_simple<X4, Y, true><<<grid, 256, 0, st>>>(a);
    else mx_gemm_simple<X4, Y, false><<<grid, 256, 0, st>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_mx_gemm(const MxShape &sh, const void *x, const void *x_scales, int64_t ldx, int32_t M, const void *codes, const void *scales,
                   const int32_t *offsets, void *y, int64_t ldy, hipStream_t st)
{
    MxArgs a{};
    a.x = (const char *)x, a.x_scales = (const uint8_t *)x_scales, a.codes = (const char *)codes, a.scales = (const char *)scales;
    a.offsets = offsets, a.y = y, a.ldx = ldx, a.ldy = ldy, a.M = M, a.N = sh.N, a.K = sh.K, a.groups = sh.groups;
    const int64_t n = (sh.N + 31) / 32 * 32;
    a.code_bytes = n * ((sh.K + 63) / 64 * 32);
    a.scale_bytes = n * ((sh.K + 255) / 256 * 8);
    if (sh.x4) return sh.y32 ? launch_typed<true, float>(a, sh.relu, st) : launch_typed<true, __bf16>(a, sh.relu, st);
    return sh.y32 ? launch_typed<false, float>(a, sh.relu, st) : launch_typed<false, __bf16>(a, sh.relu, st);
}

}  // namespace sida
