// Grouped product of token rows with experts in MXFP4:  y[r,:] = W_g x[r,:] for the rows r of group g.
//
//     y[r,n] = sum_b  2^(e_w[n,b] - 127) 2^(e_x[r,b] - 127)  sum_{k in block b}  w[n,k] x[r,k]        (sums in fp32; e_x and its factor
//                                                                                                      only where the tokens are codes too)
// Tokens in bf16: a fragment's eight codes become eight bf16 values in registers, times their power of two (exact), one conversion
// for each two, which the matrix cores' time hides; products by the 32x32x16 bf16 instruction.  Tokens in 4 bits: codes and
// scales go into the 32x32x64 instruction as they are, four times as many operations in the same time.
//
// Experts are in the order in which a wavefront's fragments lie, so they go from memory into registers, 1 KiB to an instruction,
// and are read by one wavefront only; the token rows, which all four wavefronts of a workgroup need, go through LDS.
//
// What bounds it.  Few tokens for each expert: the experts' bytes (128 tokens in bf16, 50 experts of 768 x 3072 in use, 12.3 us for 66 MB,
// 5.3 TB/s; 1111 of 64 experts, 3072 x 768, 17.2 us for 87 MB).  Many: neither matrix cores nor loads, but that they overlap only in part.  16384
// tokens, 128 experts of 768 x 3072, bf16: 86 to 94 us, 77 GFLOP, 0.85 PFLOP/s, 48% of the matrix cores' cycles (an earlier build took 70 us
// for the products and 69 for the data).  32768 in 4 bits, 4096 x 1024: 107 to 112 us, 2.5 PFLOP/s for 406 MB, 27% (loads alone 68 us in an earlier
// build: weights are one stage ahead and there are two wavefronts to a SIMD).  One matrix, 16384 x 4096 x 4096, 1.36 PFLOP/s in bf16, 2.95 in 4 bits.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>
#include <utility>

#include "kernels.h"
#include "mx_rule.h"

namespace sida {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

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
    int relu, unit;              // unit: 16, 4 or 2 bytes that every row of y starts and ends on a multiple of
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void *base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}

// Which tile a workgroup takes.  Token tiles are counted group by group (BM rows each, a group's last one less), and each has
// n_tiles column tiles.  Workgroup b runs on XCD b % 8; an XCD takes an eighth of the tiles there are, one after the other, so
// that a token tile's rows and a group's matrix are fetched into one L2.  Every wavefront finds its tile by itself, four groups to
// a lane; rows = 0 where there are fewer tiles than workgroups.
struct Placed {
    int group, row0, rows, nt;
};
template <int BM>
__device__ __forceinline__ Placed place(const MxArgs &a, int n_tiles)
{
    const int lane = threadIdx.x & 63;
    const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
    auto tile_of = [&](int tiles) {                          // (token tile, column tile), or -1
        const int total = tiles * n_tiles, share = (total + 7) / 8, id = xcd * share + local;
        return local < share && id < total ? id : -1;
    };
    if (!a.offsets) {
        const int id = tile_of((a.M + BM - 1) / BM);
        if (id < 0) return Placed{0, 0, 0, 0};
        const int row0 = id / n_tiles * BM;
        return Placed{0, row0, min(BM, a.M - row0), id % n_tiles};
    }
    // Entries past the last one come as zeros: groups without rows.
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.offsets, (uint32_t)(a.groups + 1) * 4);
    const i32x4 mine = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, 0, 0));
    const int next = __builtin_amdgcn_raw_buffer_load_b32(r, lane * 16 + 16, 0, 0);
    int at[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) at[i] = max(0, min(a.M, i < 4 ? mine[i] : next));
    int tiles = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) tiles += (max(0, at[i + 1] - at[i]) + BM - 1) / BM;
    // Sum over this and all lower lanes: in rows of 16 lanes, then row 0's and 2's last lane into rows 1 and 3, lane 31's into the upper half.
    int before = tiles;
    before += __builtin_amdgcn_update_dpp(0, before, 0x111, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x112, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x114, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x118, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x142, 0xa, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x143, 0xc, 0xf, false);
    const int id = tile_of(__builtin_amdgcn_readlane(before, 63));
    if (id < 0) return Placed{0, 0, 0, 0};
    const int mt = id / n_tiles;
    const int owner = __builtin_ctzll(__ballot(before > mt));
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
    return Placed{__builtin_amdgcn_readlane(group, owner), __builtin_amdgcn_readlane(row0, owner), __builtin_amdgcn_readlane(rows, owner), id % n_tiles};
}

// Eight codes times their power of two, exact in bf16, which has room for 1/2 * 2^-127 as well; infinite from 2^128 on (powers of two above
// 2^125, which rounding to MXFP4 does not give).
__device__ __forceinline__ bf16x8 decode(uint32_t c, float s)
{
    bf16x8 o;
    *(reinterpret_cast<bf16x2 *>(&o) + 0) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
    *(reinterpret_cast<bf16x2 *>(&o) + 1) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
    *(reinterpret_cast<bf16x2 *>(&o) + 2) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
    *(reinterpret_cast<bf16x2 *>(&o) + 3) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
    return o;
}

__device__ __forceinline__ i32x8 wide(i32x4 v) { return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }   // 4-bit operands fill half of the registers
__device__ __forceinline__ float relu_of(float v) { return v <= 0.f ? 0.f : v; }   // NaN stays

template <class T>
struct Of {
    typedef T type;
};

template <class F, int... I>
__device__ __forceinline__ void each(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>()), ...);
}

template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// 16 or 4 bytes per lane straight into LDS: lane i's land at dst + 16 * i or 4 * i.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t offset, void *dst)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)dst, 16, (int)offset, 0, 0, 0);
}
__device__ __forceinline__ void load_word_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t offset, void *dst)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)dst, 4, (int)offset, 0, 0, 0);
}
// Lane offset of a load that asks for nothing: past every descriptor here (128 rows less than 2^25 bytes apart).
constexpr uint32_t kNowhere = 0xffffff00u;

constexpr int kWaves = 4;
constexpr int kStageRow = 128;                 // bytes of a token row per stage: 64 values in bf16, 256 in 4 bits

// A tile of up to 32 MI tokens x 128 NS columns by a workgroup of four wavefronts; wavefront w owns NS stripes of 32 columns and all
// tokens.  Token rows are loaded NB stages ahead of their use and weights WB.
template <bool X4, int MI, int NS, int NB, int WB, class Y>
struct TileShape {
    static constexpr int kStage = MI * 32 * kStageRow + (X4 ? 1024 : 0);   // token rows, and their scales
    static constexpr int kRing = (NB + 1) * kStage;
    static constexpr int kTurnCols = sizeof(Y) == 2 ? NS * 32 : 32;        // columns that go through LDS together
    static constexpr int kTurnPitch = kTurnCols * (int)sizeof(Y) + 16;
    static constexpr int kTurn = kWaves * 32 * kTurnPitch;
    static constexpr int kLds = kRing > kTurn ? kRing : kTurn;
};
template <bool X4, int MI, int NS, int NB, int WB, class Y>
__device__ __forceinline__ void take_tile(const MxArgs &a, const Placed &at, char *lds)
{
    typedef TileShape<X4, MI, NS, NB, WB, Y> Shape;
    constexpr int BM = 32 * MI, kStage = Shape::kStage, kTurnCols = Shape::kTurnCols, kTurnPitch = Shape::kTurnPitch;
    constexpr int WQ = X4 ? 4 : 1;                             // weight fragments per stripe and stage
    // After a stage's token loads at least the token loads of NB - 1 later stages and WB stages of weights are asked for
    // before it is used; the waits for the weights themselves are the compiler's.
    constexpr int kLater = (NB - 1) * (MI + (X4 ? 1 : 0)) + WB * NS * (WQ + (X4 ? 1 : 0));
    static_assert(kLater <= 63 && NB % WB == 0, "vmcnt range");

    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int stripe0 = at.nt * (NS * kWaves) + wv * NS, stripes = (a.N + 31) / 32;
    const int chunks = (a.K + 63) / 64, groups = (a.K + 255) / 256;
    const int row_bytes = X4 ? a.K / 2 : a.K * 2;
    const int stages = (row_bytes + kStageRow - 1) / kStageRow;

    // token loads: a wavefront's load j brings rows 8 (wv MI + j) .. + 7; row r's piece c goes to place c ^ (r / 2 & 7)
    const uint32_t pitch = X4 ? (uint32_t)row_bytes : (uint32_t)a.ldx * 2;
    const char *x = a.x + (int64_t)at.row0 * pitch;
    const int full = row_bytes / kStageRow;                    // stages that are whole; there may be one more, partly filled
    uint32_t tok_off[MI], tok_last[MI];
#pragma unroll
    for (int j = 0; j < MI; ++j) {
        const int r = (wv * MI + j) * 8 + (lane >> 3), piece = ((lane & 7) ^ (r >> 1 & 7)) * 16;
        tok_off[j] = r < at.rows ? (uint32_t)r * pitch + piece : kNowhere;
        tok_last[j] = full * kStageRow + piece < row_bytes ? tok_off[j] : kNowhere;
    }
    const uint32_t span = (uint32_t)(at.rows - 1) * pitch + row_bytes;
    const int scale_pitch = groups * 8;
    const char *xs = (const char *)a.x_scales + (X4 ? (int64_t)at.row0 * scale_pitch : 0);
    const uint32_t xs_off = wv * 32 + (lane >> 1) < BM ? (uint32_t)(wv * 32 + (lane >> 1)) * scale_pitch + (lane & 1) * 4 : kNowhere;
    // Stages past the last one ask for nothing (no records), so that every turn of the loop has the same operations.
    auto load_tokens = [&](int stage, int slot) {
        char *dst = lds + slot * kStage;
        const __amdgpu_buffer_rsrc_t r = make_rsrc(x + (int64_t)min(stage, stages) * kStageRow, stage < stages ? span : 0);
#pragma unroll
        for (int j = 0; j < MI; ++j) load_to_lds(r, stage < full ? tok_off[j] : tok_last[j], dst + (wv * MI + j) * 1024);
        if (X4)
            load_word_to_lds(make_rsrc(xs + min(stage, stages) * 8, stage < stages ? at.rows * scale_pitch - stage * 8 : 0), xs_off,
                             dst + BM * kStageRow + wv * 256);
    };

    const char *w_at[NS], *s_at[NS];
    uint32_t w_bytes[NS], s_bytes[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const bool in = stripe0 + s < stripes;
        const int64_t st = in ? stripe0 + s : 0;
        w_at[s] = a.codes + at.group * a.code_bytes + st * chunks * 1024;
        s_at[s] = a.scales + at.group * a.scale_bytes + st * groups * 256;
        w_bytes[s] = in ? chunks * 1024 : 0;
        s_bytes[s] = in ? groups * 256 : 0;
    }
    i32x4 w[WB][NS][WQ];
    // Powers of two: a lane's four bytes are those of 256 columns, in 4 bits a stage, in bf16 four stages (asked for that far ahead).
    uint32_t ws[X4 ? WB : 1][NS], ws_next[NS];
    auto load_scales = [&](uint32_t (&to)[NS], int from256) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const bool in = from256 < groups && s_bytes[s];
            to[s] = __builtin_amdgcn_raw_buffer_load_b32(make_rsrc(s_at[s] + (in ? from256 * 256 : 0), in ? s_bytes[s] - from256 * 256 : 0), lane * 4, 0, 0);
        }
    };
    auto load_weights = [&](int b, int stage) {
        const bool in = stage < stages;
        const int from = in ? stage * (WQ * 1024) : 0;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const __amdgpu_buffer_rsrc_t r = make_rsrc(w_at[s] + from, in && w_bytes[s] ? w_bytes[s] - from : 0);
#pragma unroll
            for (int q = 0; q < WQ; ++q) w[b][s][q] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16 + q * 1024, 0, 0));
        }
        if constexpr (X4) load_scales(ws[b], stage);
    };

    f32x16 acc[NS][MI];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[s][m][r] = 0;
    int frag_off[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) frag_off[q] = (lane & 31) * kStageRow + (((X4 ? 2 * q + half : half * 4 + q) ^ ((lane & 31) >> 1 & 7)) * 16);
    auto multiply = [&](int b, int slot, int turn) {           // turn: which of a loop turn's stages
        const char *src = lds + slot * kStage;
        uint32_t xs[MI];
        if constexpr (X4)
#pragma unroll
            for (int m = 0; m < MI; ++m) {
                const u32x2 both = *reinterpret_cast<const u32x2 *>(src + BM * kStageRow + (m * 32 + (lane & 31)) * 8);
                xs[m] = __builtin_amdgcn_perm(both[1], both[0], half ? 0x07050301u : 0x06040200u);
            }
        // Token fragments are read one step ahead of their products (the compiler would read them where they are used), where the registers
        // allow it; further ahead gains nothing (16384 x 4096 x 4096: 415, 404, 403, 405 us for 0 to 3 steps).
        constexpr int kSteps = 4 * MI, kAhead = X4 && MI == 2 ? 0 : 1, kHeld = kAhead + 1;
        i32x4 held[kHeld];
        auto read = [&](int k) { held[k % kHeld] = *reinterpret_cast<const i32x4 *>(src + (k % MI) * 32 * kStageRow + frag_off[k / MI]); };
#pragma unroll
        for (int k = 0; k < kAhead && k < kSteps; ++k) read(k);
        bf16x8 v[NS];
        auto step = [&](auto place) {
            constexpr int k = decltype(place)::value, q = k / MI, m = k % MI;
            if constexpr (k + kAhead < kSteps) read(k + kAhead);
            if constexpr (!X4 && m == 0)
#pragma unroll
                for (int s = 0; s < NS; ++s) v[s] = decode(w[b][s][0][q], __builtin_bit_cast(float, (ws[0][s] >> (turn * 8) & 255u) << 23));
            const i32x4 x = held[k % kHeld];
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                if constexpr (X4)
                    acc[s][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w[b][s][q]), wide(x), acc[s][m], 4, 4, q, ws[b][s], q, xs[m]);
                else
                    acc[s][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[s], __builtin_bit_cast(bf16x8, x), acc[s][m], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        each(step, std::make_integer_sequence<int, kSteps>());
    };

    // In front of the loop in the loop's order, so that the compiler's waits for the weights are as loose there.  A stage's tokens have to
    // be asked for in front of its weights: kLater counts on it.
    if constexpr (!X4) load_scales(ws[0], 0);
#pragma unroll
    for (int i = -NB; i < 0; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        load_tokens(i + NB, i + NB);
        __builtin_amdgcn_sched_barrier(0);
        if (i + WB >= 0) load_weights((i + NB) % WB, i + WB);
    }
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kTurn = X4 ? WB : 4;                          // stages a turn of the loop
    static_assert(kTurn % WB == 0, "weight registers");
    int t = 0, slot = 0;
    auto stage = [&](int i, auto left) {                        // the turn's stage i
        wait_loads<decltype(left)::value ? 0 : kLater>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        load_tokens(t + i + NB, slot ? slot - 1 : NB);
        multiply(i % WB, slot, i);
        __builtin_amdgcn_sched_barrier(0);                     // loads any earlier would need registers of their own
        load_weights(i % WB, t + i + WB);
        if (!X4 && i == 0) load_scales(ws_next, t / 4 + 1);
        slot = slot == NB ? 0 : slot + 1;
    };
    for (; t + kTurn <= stages; t += kTurn) {
#pragma unroll
        for (int i = 0; i < kTurn; ++i) stage(i, std::false_type());
        if constexpr (!X4)
#pragma unroll
            for (int s = 0; s < NS; ++s) ws[0][s] = ws_next[s];
    }
    if constexpr (kTurn > 1)
#pragma unroll
        for (int i = 0; i < kTurn - 1; ++i) {                  // What is left of the stages, less than a turn.  Loads whose results nobody
            if (t + i >= stages) break;                        // takes are not in the program here: nothing is counted on.
            stage(i, std::true_type());
        }
    wait_loads<0>();                                            // the last loads still write LDS
    __builtin_amdgcn_s_barrier();

    // Results.  A lane holds four times four consecutive columns of one token; turned around in LDS, consecutive lanes store consecutive
    // pieces of a row, 16 bytes each, or as much as the rows' alignment allows (20926 tokens, 320 x 601: 50 us where lanes stored their own
    // columns one by one, 25 so).
    Y *y = (Y *)a.y + (int64_t)at.row0 * a.ldy;
    char *turn = lds + wv * 32 * kTurnPitch;
    constexpr int kPer = kTurnCols / 32;                        // stripes per turn
    auto put = [&](auto unit, int m, int s0) {
        typedef typename decltype(unit)::type Unit;
        constexpr int kOf = (int)(sizeof(Unit) / sizeof(Y)), kLanes = kTurnCols / kOf;   // columns of a piece, pieces of a row
#pragma unroll
        for (int i = 0; i < 32 * kLanes / 64; ++i) {
            const int at_piece = i * 64 + lane, r = at_piece / kLanes, c = at_piece % kLanes * kOf;
            const Unit v = *reinterpret_cast<const Unit *>(turn + r * kTurnPitch + c * (int)sizeof(Y));
            const int row = m * 32 + r, col = (stripe0 + s0) * 32 + c;
            if (row >= at.rows || col >= a.N) continue;
            Unit *to = reinterpret_cast<Unit *>(y + (int64_t)row * a.ldy + col);
            if constexpr (sizeof(Unit) == 16) __builtin_nontemporal_store(v, to);        // whole lines, past L2's replacement
            else *to = v;
        }
    };
#pragma unroll
    for (int m = 0; m < MI; ++m) {
#pragma unroll
        for (int s0 = 0; s0 < NS; s0 += kPer) {
#pragma unroll
            for (int s = 0; s < kPer; ++s)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    typedef __attribute__((ext_vector_type(4))) Y Y4;
                    Y4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e = acc[s0 + s][m][4 * q + j];
                        v[j] = (Y)(a.relu ? relu_of(e) : e);
                    }
                    *reinterpret_cast<Y4 *>(turn + (lane & 31) * kTurnPitch + (s * 32 + q * 8 + half * 4) * (int)sizeof(Y)) = v;
                }
            __builtin_amdgcn_wave_barrier();
            if (a.unit == 16) {
                put(Of<i32x4>(), m, s0);
            } else if (sizeof(Y) == 4 || a.unit == 4) {
                put(Of<uint32_t>(), m, s0);
            } else {
                put(Of<Y>(), m, s0);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// A kernel for tiles of up to 32 MI tokens; each number of 32-token blocks has a way of its own through it, with registers and loads
// for that many blocks and no more.
template <bool X4, int MI, int NS, int NB, int WB, int OCC, class Y>
__global__ __launch_bounds__(kWaves * 64, OCC) void mx_gemm_tiles(const MxArgs a)
{
    __shared__ __attribute__((aligned(1024))) char lds[TileShape<X4, MI, NS, NB, WB, Y>::kLds];
    const Placed at = place<32 * MI>(a, (a.N + 128 * NS - 1) / (128 * NS));
    if (at.rows == 0) return;
    if (MI > 1 && at.rows <= 32) return take_tile<X4, 1, NS, NB, WB, Y>(a, at, lds);
    if (MI > 2 && at.rows <= 64) return take_tile<X4, 2, NS, NB, WB, Y>(a, at, lds);
    if (MI > 3 && at.rows <= 96) return take_tile<X4, 3, NS, NB, WB, Y>(a, at, lds);
    take_tile<X4, MI, NS, NB, WB, Y>(a, at, lds);
}

// Few rows, few tiles: a single token's product is a few hundred kilobytes for the whole chip, and what counts is how long the
// way through K is.  A workgroup takes 32 tokens and one stripe of 32 columns, and its sixteen wavefronts split the sum over K, 64
// values at a time in turn; the parts meet in LDS and are added in a fixed order.  Up to K = 4096 a wavefront has all its
// loads under way at once.  One token, 4096 x 1024: 6.2 us, of which 2 MB of weights at the rate of a large copy would be 0.4; the rest is
// the launch, one way to memory and back, and the sum.
constexpr int kSplit = 16, kSplitAhead = 4;
template <bool X4, class Y>
__global__ __launch_bounds__(kSplit * 64, 4) void mx_gemm_split(const MxArgs a)
{
    __shared__ __attribute__((aligned(16))) float parts[kSplit][1024];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int stripes = (a.N + 31) / 32, chunks = (a.K + 63) / 64, groups = (a.K + 255) / 256;
    const Placed at = place<32>(a, stripes);
    if (at.rows == 0) return;
    const __amdgpu_buffer_rsrc_t w_rsrc = make_rsrc(a.codes + at.group * a.code_bytes + (int64_t)at.nt * chunks * 1024, chunks * 1024);
    const __amdgpu_buffer_rsrc_t s_rsrc = make_rsrc(a.scales + at.group * a.scale_bytes + (int64_t)at.nt * groups * 256, groups * 256);
    const int row_bytes = X4 ? a.K / 2 : a.K * 2, scale_pitch = groups * 8;
    const uint32_t pitch = X4 ? (uint32_t)row_bytes : (uint32_t)a.ldx * 2;
    const int row = lane & 31;
    const __amdgpu_buffer_rsrc_t x_rsrc = make_rsrc(a.x + (int64_t)at.row0 * pitch, (uint32_t)(at.rows - 1) * pitch + row_bytes);
    const __amdgpu_buffer_rsrc_t xs_rsrc = make_rsrc(a.x_scales + (X4 ? (int64_t)at.row0 * scale_pitch : 0), X4 ? at.rows * scale_pitch : 0);
    constexpr int XQ = X4 ? 1 : 4;
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0;
    for (int c0 = wv; c0 < chunks; c0 += kSplit * kSplitAhead) {
        i32x4 w[kSplitAhead], x[kSplitAhead][XQ];
        uint32_t ws[kSplitAhead], xs[kSplitAhead];
#pragma unroll
        for (int i = 0; i < kSplitAhead; ++i) {              // chunks past the last one lie outside of the descriptors: zeros
            const int c = c0 + i * kSplit, k = c * 64 + half * 32;
            w[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, c * 1024 + lane * 16, 0, 0));
            ws[i] = __builtin_amdgcn_raw_buffer_load_b8(s_rsrc, (c >> 2) * 256 + lane * 4 + (c & 3), 0, 0);
            const bool in = row < at.rows && k < a.K;
            const uint32_t from = in ? (uint32_t)row * pitch + (uint32_t)k * 2 / (X4 ? 4 : 1) : kNowhere;
#pragma unroll
            for (int q = 0; q < XQ; ++q) x[i][q] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, (int)(in ? from + q * 16 : kNowhere), 0, 0));
            if (X4) xs[i] = __builtin_amdgcn_raw_buffer_load_b8(xs_rsrc, (int)(in ? (uint32_t)(row * scale_pitch + k / 32) : kNowhere), 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);                     // all of them before the first product
#pragma unroll
        for (int i = 0; i < kSplitAhead; ++i) {
            if constexpr (X4) {
                acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w[i]), wide(x[i][0]), acc, 4, 4, 0, ws[i], 0, xs[i]);
            } else {
                const float f = __builtin_bit_cast(float, ws[i] << 23);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode(w[i][q], f), __builtin_bit_cast(bf16x8, x[i][q]), acc, 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4 *>(&parts[wv][q * 256 + lane * 4]) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    float sum = parts[0][tid];
#pragma unroll
    for (int p = 1; p < kSplit; ++p) sum += parts[p][tid];
    const int from = tid % 256 / 4, token = from & 31, col = at.nt * 32 + tid / 256 * 8 + from / 32 * 4 + tid % 4;
    if (token < at.rows && col < a.N) ((Y *)a.y)[(int64_t)(at.row0 + token) * a.ldy + col] = (Y)(a.relu ? relu_of(sum) : sum);
}

template <bool X4, int MI, int NS, int NB, int WB, int OCC, class Y>
int launch_shape(const MxArgs &a, hipStream_t st)
{
    constexpr int BM = 32 * MI, BN = 32 * NS * kWaves;
    const int64_t tiles = a.M / BM + (a.groups < a.M ? a.groups : a.M), grid = tiles * ((a.N + BN - 1) / BN);
    mx_gemm_tiles<X4, MI, NS, NB, WB, OCC, Y><<<(uint32_t)((grid + 7) / 8 * 8), kWaves * 64, 0, st>>>(a);
    return (int)hipGetLastError();
}

template <bool X4, class Y>
int launch_typed(const MxArgs &a, hipStream_t st)
{
    switch (mx_tiles(X4, a.M, a.groups, a.N, a.K)) {
    case MxTiles::split: {
        const int64_t tiles = (a.M / 32 + (a.groups < a.M ? a.groups : a.M)) * (int64_t)((a.N + 31) / 32);
        mx_gemm_split<X4, Y><<<(uint32_t)((tiles + 7) / 8 * 8), kSplit * 64, 0, st>>>(a);
        return (int)hipGetLastError();
    }
    case MxTiles::rows32: return launch_shape<X4, 1, 1, X4 ? 2 : 4, X4 ? 2 : 4, X4 ? 5 : 6, Y>(a, st);
    case MxTiles::rows128:
        if constexpr (X4) return launch_shape<X4, 4, 2, 2, 1, 2, Y>(a, st);
        break;                                                 // 4 bits alone have it
    case MxTiles::rows64: break;
    }
    return launch_shape<X4, 2, 2, 2, X4 ? 1 : 2, 4, Y>(a, st);
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
    a.relu = sh.relu;
    const size_t size = sh.y32 ? 4 : 2;
    const size_t ends = (uintptr_t)y | (size_t)ldy * size | (size_t)sh.N * size;
    a.unit = ends % 16 == 0 ? 16 : ends % 4 == 0 ? 4 : 2;
    if (sh.x4) return sh.y32 ? launch_typed<true, float>(a, st) : launch_typed<true, __bf16>(a, st);
    return sh.y32 ? launch_typed<false, float>(a, st) : launch_typed<false, __bf16>(a, st);
}

}  // namespace sida
