// Rounding to MXFP4 (32 values of a row share a power of two, each of them 4 bits).
//
//     m = max |x| of a block,  s = 2^(floor(log2 m) - 2) >= 2^-127,  code = x / s rounded to {0, 1/2, 1, 3/2, 2, 3, 4, 6}
//
// The power of two is read off the exponent field of m, so no logarithm is taken and nothing is rounded but the codes, which
// the conversion instructions round to the nearest, ties to the even code, and bound by 6 (checked against the definition
// for every finite bf16 value and for fp32 values around the midpoints).
//
// Bound by bytes: 2 or 4 in, 17/32 (and 2 where the rounded values are asked for) out, a few operations each.  Four lanes
// share a block, 8 values each: 16-byte loads and stores, two lane exchanges for the maximum.  What is not read again soon is stored
// past L2's replacement.  262144 x 1024 from fp32 with the rounded values, 1.75 GB: 297 us, 5.9 TB/s (341 with ordinary stores); 32768
// x 4096 from bf16, 340 MB, 58 us, 5.9 TB/s; one row 1.5 us, all launch.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "kernels.h"

namespace sida {

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// Eight consecutive values as they lie in memory.
template <class T>
struct Piece;
template <>
struct Piece<__bf16> {
    uint32_t w[4];
    // Exponent field of the largest magnitude; infinities and NaN have 255.
    __device__ uint32_t top() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
        return m >> 7;
    }
    __device__ uint32_t codes(float s) const
    {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), s, 3);
        return c;
    }
    template <bool WIDE>
    __device__ void load(const __bf16 *p)
    {
        if (WIDE) {
            *reinterpret_cast<u32x4 *>(w) = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
        } else {
            const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = q[2 * i] | (uint32_t)q[2 * i + 1] << 16;
        }
    }
};
template <>
struct Piece<float> {
    uint32_t w[8];
    __device__ uint32_t top() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
        return m >> 23;
    }
    __device__ float at(int i) const { return __builtin_bit_cast(float, w[i]); }
    __device__ uint32_t codes(float s) const
    {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, at(0), at(1), s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, at(2), at(3), s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, at(4), at(5), s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, at(6), at(7), s, 3);
        return c;
    }
    template <bool WIDE>
    __device__ void load(const float *p)
    {
        if (WIDE) {
            *reinterpret_cast<u32x4 *>(w) = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
            *reinterpret_cast<u32x4 *>(w + 4) = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p) + 1);
        } else {
            const uint32_t *q = reinterpret_cast<const uint32_t *>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = q[i];
        }
    }
};

struct Rounded {
    uint32_t codes;              // of this lane's eight values
    uint32_t scale;              // of the block
};

// The block's four lanes are lanes 4i .. 4i+3 of a wavefront.
template <class T>
__device__ __forceinline__ Rounded round_piece(const Piece<T> &v)
{
    uint32_t top = v.top();
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xf, 0xf, true));      // quad_perm 1,0,3,2
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xf, 0xf, true));      // quad_perm 2,3,0,1
    Rounded r;
    r.scale = top == 255 ? 255 : (top > 2 ? top - 2 : 0);
    // field 0 stands for 2^-127: the float of that value is 0x00400000
    const float s = __builtin_bit_cast(float, max(r.scale << 23, 0x00400000u));
    r.codes = top == 255 ? 0 : v.codes(s);
    return r;
}

// What eight codes stand for, as bf16 (exact; NaN where the scale is).
__device__ __forceinline__ u32x4 values_of(const Rounded &r)
{
    const float s = __builtin_bit_cast(float, r.scale << 23);
    u32x4 o;
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, s, 0));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, s, 1));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, s, 2));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, s, 3));
    return o;
}

// Token rows.  The rows' pieces are dealt to the threads as one flat range, kDeal to a thread, all loaded before the first
// is rounded.  A row's last block writes the filling of the row's scales too.
constexpr int kDeal = 4;
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void mx_round_rows(const T *__restrict__ x, int64_t rows, int cols, int64_t ld,
                                                     uint32_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                     u32x4 *__restrict__ values)
{
    const uint32_t per_row = (uint32_t)cols / 8, blocks = (uint32_t)cols / 32, pitch = (uint32_t)((cols + 255) / 256) * 8;
    const int64_t total = rows * per_row, first = (int64_t)blockIdx.x * (256 * kDeal);
    const int64_t row0 = first / per_row;                     // uniform: once per workgroup
    const uint32_t rest = (uint32_t)(first - row0 * per_row);
    Piece<T> v[kDeal];
    int64_t row[kDeal];
    uint32_t at[kDeal];
#pragma unroll
    for (int i = 0; i < kDeal; ++i) {
        const uint32_t local = rest + i * 256 + threadIdx.x;  // < per_row + 1024
        const uint32_t r = local / per_row;
        row[i] = row0 + r;
        at[i] = local - r * per_row;
        if (first + i * 256 + threadIdx.x < total) v[i].template load<WIDE>(x + row[i] * ld + at[i] * 8);
    }
#pragma unroll
    for (int i = 0; i < kDeal; ++i) {
        if (first + i * 256 + threadIdx.x >= total) continue;   // blocks are whole: their four lanes go together
        const Rounded q = round_piece(v[i]);
        codes[row[i] * per_row + at[i]] = q.codes;
        if (values) values[row[i] * per_row + at[i]] = values_of(q);
        if (at[i] % 4 == 0) {
            uint8_t *s = scales + row[i] * pitch;
            const uint32_t b = at[i] / 4;
            s[b] = (uint8_t)q.scale;
            if (b + 1 == blocks)
                for (uint32_t f = blocks; f < pitch; ++f) s[f] = 127;
        }
    }
}

// Expert matrices.  A workgroup takes 32 rows x 256 columns: 8 whole row pieces of 256 columns per load, the codes and scales
// turned around in LDS, so that they leave as the 4 KiB and 256 bytes of consecutive memory that they are in the layout.
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void mx_round_tiles(const T *__restrict__ x, int64_t rows, int cols, int64_t ld,
                                                      u32x4 *__restrict__ codes, u32x4 *__restrict__ scales,
                                                      u32x4 *__restrict__ values)
{
    __shared__ __attribute__((aligned(16))) uint32_t code_tile[1024];
    __shared__ __attribute__((aligned(16))) uint8_t scale_tile[256];
    const int tid = threadIdx.x, groups = (cols + 255) / 256, chunks = (cols + 63) / 64;
    const int64_t stripe = blockIdx.x / groups;
    const int group = blockIdx.x % groups;
    const int piece = tid & 31, col = group * 256 + piece * 8;
    Piece<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = stripe * 32 + i * 8 + (tid >> 5);
#pragma unroll
        for (uint32_t &w : v[i].w) w = 0;
        if (row < rows && col < cols) v[i].template load<WIDE>(x + row * ld + col);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (tid >> 5);
        const int64_t row = stripe * 32 + r;
        Rounded q = round_piece(v[i]);
        const bool live = row < rows && col < cols;           // the same for a block's four lanes
        if (!live) q.scale = 127;
        // block j = piece / 4 of this group: 512 bytes of codes per j, 16 per row
        code_tile[(piece / 4) * 128 + r * 4 + piece % 4] = q.codes;
        if (piece % 4 == 0) scale_tile[(piece / 4 % 2) * 128 + r * 4 + piece / 8] = (uint8_t)q.scale;
        if (live && values) __builtin_nontemporal_store(values_of(q), &values[row * (cols / 8) + col / 8]);
    }
    __syncthreads();
    if (group * 4 + (tid >> 6) < chunks)                      // a chunk of 64 columns is 64 pieces of 16 bytes
        __builtin_nontemporal_store(reinterpret_cast<const u32x4 *>(code_tile)[tid], &codes[(stripe * chunks + group * 4) * 64 + tid]);
    if (tid < 16) scales[(stripe * groups + group) * 16 + tid] = reinterpret_cast<const u32x4 *>(scale_tile)[tid];
}

template <class T, bool WIDE>
int launch_typed(const void *x, int64_t rows, int32_t cols, int64_t ld, bool tiles, void *codes, void *scales, void *values,
                 hipStream_t st)
{
    if (tiles) {
        const int64_t grid = (rows + 31) / 32 * ((cols + 255) / 256);
        mx_round_tiles<T, WIDE><<<(uint32_t)grid, 256, 0, st>>>((const T *)x, rows, cols, ld, (u32x4 *)codes, (u32x4 *)scales, (u32x4 *)values);
    } else {
        const int64_t grid = (rows * (cols / 8) + 256 * kDeal - 1) / (256 * kDeal);
        mx_round_rows<T, WIDE><<<(uint32_t)grid, 256, 0, st>>>((const T *)x, rows, cols, ld, (uint32_t *)codes, (uint8_t *)scales, (u32x4 *)values);
    }
    return (int)hipGetLastError();
}

}  // namespace

int launch_mx_quantize(const void *x, bool fp32, int64_t rows, int32_t cols, int64_t ld, bool tiles, void *codes, void *scales,
                       void *values, hipStream_t st)
{
    const size_t size = fp32 ? 4 : 2;
    const bool wide = ((uintptr_t)x | (size_t)ld * size) % 16 == 0;
    if (fp32)
        return wide ? launch_typed<float, true>(x, rows, cols, ld, tiles, codes, scales, values, st)
                    : launch_typed<float, false>(x, rows, cols, ld, tiles, codes, scales, values, st);
    return wide ? launch_typed<__bf16, true>(x, rows, cols, ld, tiles, codes, scales, values, st)
                : launch_typed<__bf16, false>(x, rows, cols, ld, tiles, codes, scales, values, st);
}

}  // namespace sida
