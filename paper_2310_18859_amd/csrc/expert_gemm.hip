// Grouped products of plain bf16 experts, forward and backward, for the rows r of group g (sums in fp32, one rounding at the end):
//     product   v = W_g x[r] + b_g,  y[r] = act(v) + residual[r]             sum over K
//     input     dx[r] = (W_g^T dy[r]) act'(pre[r])                           sum over N
//     weights   dW_g = sum_r dy[r] x[r]^T,  db_g = sum_r dy[r]               sum over the group's rows
// One tile routine serves the three: C[i,j] = sum_c A[i,c] B[j,c], where an operand lies with c along its rows in memory (x, dy, and W in
// the product) or with c across them (W in `input`, both operands in `weights`).
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>
#include <utility>

#include "expert_rule.h"
#include "kernels.h"

namespace sida {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

enum class Job { product, input, weights };

struct GemmArgs {
    const char *a, *b;           // rows (product: x, input: dy, weights: dy) and the other operand (W, W, x)
    const int32_t *offsets;      // NULL: one group of M rows
    int64_t lda, ldb;            // values between rows
    int64_t b_group;             // values between groups' matrices (product, input)
    int M, groups, N, K;
    char *out;
    int64_t ldo, out_group;      // values between rows, and (weights) between groups' matrices
    int out32, activation;
    const float *bias;           // product
    char *pre;                   // product: written; input: read
    const char *residual;
    int64_t ld_pre, ld_res;
    float *d_bias;               // weights
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void *base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t offset, void *dst)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)dst, 16, (int)offset, 0, 0, 0);
}
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// A descriptor's records, and a lane offset past them: such a load asks for nothing and brings zeros.  256 rows are at most
// kMostExpertPitch values apart, so that every offset that is meant lies below.
constexpr uint32_t kRecords = 0x80000000u, kNowhere = 0xffffff00u;

// ---- which tile a workgroup takes ---------------------------------------------------------------
struct Placed {
    int group, row0, rows, nt;
};
// Row tiles are counted group by group, each with n_tiles column tiles.  Workgroup b runs on XCD b % 8; an XCD takes an eighth of
// the tiles there are, one after the other.  Every wavefront finds its tile by itself, four groups to a lane; rows = 0
// where there are fewer tiles than workgroups.
template <int BM>
__device__ __forceinline__ Placed place(const GemmArgs &a, int n_tiles)
{
    const int lane = threadIdx.x & 63;
    const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
    auto tile_of = [&](int64_t tiles) {
        const int64_t total = tiles * n_tiles, share = (total + 7) / 8, id = xcd * share + local;
        return local < share && id < total ? (int)id : -1;
    };
    if (!a.offsets) {
        const int id = tile_of((a.M + BM - 1) / BM);
        if (id < 0) return Placed{0, 0, 0, 0};
        const int row0 = id / n_tiles * BM;
        return Placed{0, row0, min(BM, a.M - row0), id % n_tiles};
    }
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.offsets, (uint32_t)(a.groups + 1) * 4);   // entries past the last one come as zeros
    int at[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) at[i] = max(0, min(a.M, (int)__builtin_amdgcn_raw_buffer_load_b32(r, lane * 16 + i * 4, 0, 0)));
    int tiles = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) tiles += (max(0, at[i + 1] - at[i]) + BM - 1) / BM;
    int upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(upto, d);
        upto += lane >= d ? v : 0;
    }
    const int id = tile_of(__builtin_amdgcn_readlane(upto, 63));
    if (id < 0) return Placed{0, 0, 0, 0};
    const int mt = id / n_tiles;
    const int owner = __builtin_ctzll(__ballot(upto > mt));
    int left = mt - (upto - tiles), group = 0, row0 = 0, rows = 0;
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

// ---- operand tiles in LDS -----------------------------------------------------------------------
// 64 values of c at a time, by loads of 1 KiB that go straight into LDS, lane i's 16 bytes to 16 i.
//   ALONG   c along a row: rows of 128 bytes, piece p of row r at place p ^ (r / 2 & 7), so that neither the loads nor the
//           reads of one piece of 32 rows meet in a bank
//   ACROSS  64 rows of c, each with the tile's columns; the 64-byte chunk of 32 columns that a fragment takes is moved
//           by the row, so that the four rows of a transposing read lie in four quarters of the banks
template <bool ACROSS, int ROWS>
struct Tile {
    static constexpr int kBytes = ROWS * 128;
    static constexpr int kPitch = ACROSS ? ROWS * 2 : 128;
    static constexpr int kLoads = kBytes / 1024;
    static __device__ __forceinline__ int turn(int r) { return kPitch >= 256 ? r & 3 : kPitch == 128 ? r >> 1 & 1 : 0; }
    // Byte offset of a lane's piece of load `w` from the tile's first value, and its c; `rows` of the tile are there.
    static __device__ __forceinline__ void lane_at(int w, int lane, int rows, uint32_t pitch, uint32_t &offset, int &c)
    {
        if constexpr (ACROSS) {
            const int at = w * 1024 + lane * 16, r = at / kPitch, b = at % kPitch;
            const int col = ((b / 64 ^ turn(r)) * 64 + b % 64) / 2;
            c = r;
            offset = col < rows ? (uint32_t)r * pitch + col * 2 : kNowhere;
        } else {
            const int r = w * 8 + (lane >> 3), piece = (lane & 7) ^ (r >> 1 & 7);
            c = piece * 8;
            offset = r < rows ? (uint32_t)r * pitch + piece * 16 : kNowhere;
        }
    }
    // Byte offset of a lane's part of the fragment of 32 rows from row 32 m and 16 c from 16 q: lane l has row l % 32, c 8 (l / 32) .. + 7.
    static __device__ __forceinline__ bf16x8 fragment(const char *tile, int lane, int m, int q)
    {
        if constexpr (ACROSS) {
            // Sixteen lanes read four rows of c, 16 columns each, and get a column each.
            const int g = lane >> 4, r = 8 * (g >> 1) + (lane >> 2 & 3);
            const char *at = tile + (16 * q + r) * kPitch + (m ^ turn(r)) * 64 + (g & 1) * 32 + (lane & 3) * 8;
            typedef __attribute__((address_space(3))) s16x4 lds4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 4 * kPitch));   // turn(r + 4) is turn(r)
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int r = lane & 31;
            return *reinterpret_cast<const bf16x8 *>(tile + (m * 32 + r) * 128 + ((2 * q + (lane >> 5)) ^ (r >> 1 & 7)) * 16);
        }
    }
};

// ---- epilogue -----------------------------------------------------------------------------------
constexpr float kLog2e = 1.44269504088896340736f, kGelu = 0.79788456080286535588f, kGelu3 = 0.044715f;
// exp(-u) and 1 / (1 + exp(-u))
struct Sigmoid {
    float e, s;
};
__device__ __forceinline__ Sigmoid sigmoid(float u)
{
    const float e = __builtin_amdgcn_exp2f(-u * kLog2e);
    return Sigmoid{e, __builtin_amdgcn_rcpf(1.f + e)};
}
// Both activations are v sigmoid(u): u = v, or for GELU in its form with tanh twice the tanh's argument.
__device__ __forceinline__ float gelu_u(float v) { return 2 * kGelu * (v + kGelu3 * v * v * v); }
__device__ __forceinline__ float activated(float v, int act)
{
    if (act == kActRelu) return v <= 0.f ? 0.f : v;          // NaN stays
    if (act == kActNone) return v;
    const float s = sigmoid(act == kActSilu ? v : gelu_u(v)).s;
    return s == 0.f ? 0.f : v * s;                           // also at -infinity
}
// s + v s (1 - s) du/dv, with 1 - s = exp(-u) s, which loses nothing where s is close to 1.  Beyond +-80 (SiLU) and +-9 (GELU) the slope is 0 or 1 to
// within 2^-80; there the powers of v and exp(-u) would give infinity times 0.
__device__ __forceinline__ float slope(float v, int act)
{
    if (act == kActNone) return 1.f;
    if (act == kActRelu) return v > 0.f ? 1.f : v <= 0.f ? 0.f : v;
    const float most = act == kActSilu ? 80.f : 9.f;
    v = v > most ? most : v < -most ? -most : v;
    const Sigmoid g = sigmoid(act == kActSilu ? v : gelu_u(v));
    const float du = act == kActSilu ? 1.f : 2 * kGelu * (1.f + 3 * kGelu3 * v * v);
    return g.s + v * (g.e * g.s) * g.s * du;
}

struct F8 {
    float v[8];
};
__device__ __forceinline__ F8 widen(bf16x8 x)
{
    F8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = (float)x[i];
    return f;
}
__device__ __forceinline__ F8 read8(const char *base, int64_t at, bool f32)
{
    if (!f32) return widen(*reinterpret_cast<const bf16x8 *>(base + at * 2));
    const f32x4 lo = *reinterpret_cast<const f32x4 *>(base + at * 4), hi = *reinterpret_cast<const f32x4 *>(base + at * 4 + 16);
    return F8{{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}};
}
__device__ __forceinline__ void write8(char *base, int64_t at, bool f32, const F8 &f)
{
    if (f32) {
        __builtin_nontemporal_store(f32x4{f.v[0], f.v[1], f.v[2], f.v[3]}, reinterpret_cast<f32x4 *>(base + at * 4));
        __builtin_nontemporal_store(f32x4{f.v[4], f.v[5], f.v[6], f.v[7]}, reinterpret_cast<f32x4 *>(base + at * 4 + 16));
        return;
    }
    bf16x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)f.v[i];
    __builtin_nontemporal_store(x, reinterpret_cast<bf16x8 *>(base + at * 2));
}

// A workgroup's tile: WI x WJ wavefronts, each MI x NJ blocks of 32 x 32; the sum over c in turns of 64 WC, which WC wavefronts share;
// S stages of tiles in LDS.
template <Job JOB, int WI, int WJ, int WC, int MI, int NJ, int S>
struct Shape {
    static constexpr bool kAcrossA = JOB == Job::weights, kAcrossB = JOB != Job::product;
    static constexpr int kWaves = WI * WJ * WC, kThreads = kWaves * 64;
    static constexpr int BM = 32 * MI * WI, BN = 32 * NJ * WJ;
    typedef Tile<kAcrossA, BM> A;
    typedef Tile<kAcrossB, BN> B;
    static constexpr int kPart = A::kBytes + B::kBytes;                    // 64 values of c
    static constexpr int kStage = WC * kPart;
    static constexpr int kLoadsA = WC * A::kLoads / kWaves, kLoadsB = WC * B::kLoads / kWaves;   // of a wavefront and stage
    static_assert(WC * A::kLoads % kWaves == 0 && WC * B::kLoads % kWaves == 0, "loads are dealt evenly");
    static constexpr int kTurnPitch = NJ * 128 + 16;
    static constexpr int kTurn = kWaves * 32 * kTurnPitch;
    static constexpr int kLds = S * kStage > kTurn ? S * kStage : kTurn;
    static_assert(WC == 1 || (WI == 1 && WJ == 1 && MI == 1), "parts of a sum");
};

// Where the operands and the result of a tile lie.
struct Work {
    const char *a, *b;           // the tile's first row, at c = 0
    uint32_t pitch_a, pitch_b;   // bytes
    int rows_a, rows_b, c;       // rows of the tile that are there, length of the sum
    int i0, j0;                  // first row and column of the result
    int group;
};

template <class Sh, Job JOB, int WI, int WJ, int WC, int MI, int NJ, int S>
__device__ __forceinline__ void take_tile(const GemmArgs &g, const Work &w, char *lds)
{
    typedef typename Sh::A A;
    typedef typename Sh::B B;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wc = wave % WC, wj = wave / WC % WJ, wi = wave / (WC * WJ);

    uint32_t off_a[Sh::kLoadsA], off_b[Sh::kLoadsB];
    int c_a[Sh::kLoadsA], c_b[Sh::kLoadsB];
#pragma unroll
    for (int i = 0; i < Sh::kLoadsA; ++i) {
        const int at = i * Sh::kWaves + wave;
        A::lane_at(at % A::kLoads, lane, w.rows_a, w.pitch_a, off_a[i], c_a[i]);
    }
#pragma unroll
    for (int i = 0; i < Sh::kLoadsB; ++i) {
        const int at = i * Sh::kWaves + wave;
        B::lane_at(at % B::kLoads, lane, w.rows_b, w.pitch_b, off_b[i], c_b[i]);
    }
    const int64_t step_a = Sh::kAcrossA ? (int64_t)64 * w.pitch_a : 128, step_b = Sh::kAcrossB ? (int64_t)64 * w.pitch_b : 128;
    const int stages = (w.c + 64 * WC - 1) / (64 * WC);
    auto load = [&](int stage, int slot) {
        char *dst = lds + slot * Sh::kStage;
#pragma unroll
        for (int i = 0; i < Sh::kLoadsA; ++i) {
            const int at = i * Sh::kWaves + wave, part = at / A::kLoads, step = stage * WC + part, c0 = step * 64;
            const bool in = c0 < w.c;                         // a step past the end asks for nothing
            const __amdgpu_buffer_rsrc_t r = make_rsrc(w.a + (in ? step * step_a : 0), kRecords);
            load_to_lds(r, in && c0 + c_a[i] < w.c ? off_a[i] : kNowhere, dst + part * Sh::kPart + at % A::kLoads * 1024);
        }
#pragma unroll
        for (int i = 0; i < Sh::kLoadsB; ++i) {
            const int at = i * Sh::kWaves + wave, part = at / B::kLoads, step = stage * WC + part, c0 = step * 64;
            const bool in = c0 < w.c;
            const __amdgpu_buffer_rsrc_t r = make_rsrc(w.b + (in ? step * step_b : 0), kRecords);
            load_to_lds(r, in && c0 + c_b[i] < w.c ? off_b[i] : kNowhere, dst + part * Sh::kPart + A::kBytes + at % B::kLoads * 1024);
        }
    };

    f32x16 acc[MI][NJ];
#pragma unroll
    for (int m = 0; m < MI; ++m)
#pragma unroll
        for (int n = 0; n < NJ; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[m][n][r] = 0;
    float bias_part[MI] = {};                                 // weights: sums of dy's columns, this wavefront's share of c
    const bool sum_bias = JOB == Job::weights && g.d_bias && w.j0 == 0;
    auto multiply = [&](int slot) {
        const char *ta = lds + slot * Sh::kStage + wc * Sh::kPart, *tb = ta + A::kBytes;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            bf16x8 fa[MI], fb[NJ];
#pragma unroll
            for (int m = 0; m < MI; ++m) fa[m] = A::fragment(ta, lane, m * WI + wi, q);
#pragma unroll
            for (int n = 0; n < NJ; ++n) fb[n] = B::fragment(tb, lane, n * WJ + wj, q);
#pragma unroll
            for (int m = 0; m < MI; ++m)
#pragma unroll
                for (int n = 0; n < NJ; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[n], fa[m], acc[m][n], 0, 0, 0);
            if (JOB == Job::weights && sum_bias && q % WJ == wj) {
#pragma unroll
                for (int m = 0; m < MI; ++m) {
                    const F8 f = widen(fa[m]);
                    bias_part[m] += ((f.v[0] + f.v[1]) + (f.v[2] + f.v[3])) + ((f.v[4] + f.v[5]) + (f.v[6] + f.v[7]));
                }
            }
        }
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s) load(s, s);
    int slot = 0;
    for (int t = 0; t < stages; ++t) {
        wait_loads<(S - 2) * (Sh::kLoadsA + Sh::kLoadsB)>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        load(t + S - 1, slot ? slot - 1 : S - 1);
        multiply(slot);
        slot = slot == S - 1 ? 0 : slot + 1;
    }
    wait_loads<0>();                                          // the last loads still write LDS
    __syncthreads();

    // A lane holds four times four columns of one row of a block; through LDS, in fp32, to eight consecutive columns of a row, so that
    // what is read and written beside the result goes by whole lines.  Parts of a sum are added here, in a fixed order.
    const bool out32 = g.out32;
#pragma unroll
    for (int m = 0; m < MI; ++m) {
        char *turn = lds + wave * 32 * Sh::kTurnPitch;
#pragma unroll
        for (int n = 0; n < NJ; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 *>(turn + (lane & 31) * Sh::kTurnPitch + (n * 32 + q * 8 + half * 4) * 4) =
                    f32x4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
        if (WC > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
        constexpr int kPieces = 32 * NJ * 4, kTakers = 64 * WC;
        for (int p = WC > 1 ? tid : lane; p < kPieces; p += kTakers) {
            const int r = p / (NJ * 4), c8 = p % (NJ * 4);
            const int i = w.i0 + (m * WI + wi) * 32 + r, jn = c8 / 4, j = w.j0 + (jn * WJ + wj) * 32 + c8 % 4 * 8;
            if (i - w.i0 >= w.rows_a || j - w.j0 >= w.rows_b) continue;
            const char *src = WC > 1 ? lds : turn;
            F8 f;
#pragma unroll
            for (int e = 0; e < 8; ++e) f.v[e] = 0;
#pragma unroll
            for (int part = 0; part < WC; ++part) {
                const f32x4 *at = reinterpret_cast<const f32x4 *>(src + (part * 32 + r) * Sh::kTurnPitch + c8 * 32);
#pragma unroll
                for (int e = 0; e < 4; ++e) f.v[e] += at[0][e], f.v[4 + e] += at[1][e];
            }
            if constexpr (JOB == Job::product) {
                if (g.bias) {
                    const F8 b = read8((const char *)g.bias, (int64_t)w.group * g.N + j, true);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f.v[e] += b.v[e];
                }
                if (g.pre) write8(g.pre, (int64_t)i * g.ld_pre + j, false, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) f.v[e] = activated(f.v[e], g.activation);
                if (g.residual) {
                    const F8 s = read8(g.residual, (int64_t)i * g.ld_res + j, out32);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f.v[e] += s.v[e];
                }
                write8(g.out, (int64_t)i * g.ldo + j, out32, f);
            } else if constexpr (JOB == Job::input) {
                if (g.pre) {
                    const F8 s = read8(g.pre, (int64_t)i * g.ld_pre + j, false);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f.v[e] *= slope(s.v[e], g.activation);
                }
                write8(g.out, (int64_t)i * g.ldo + j, out32, f);
            } else {
                write8(g.out, w.group * g.out_group + (int64_t)i * g.ldo + j, out32, f);
            }
        }
        if (WC > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
    }
    if (JOB == Job::weights && sum_bias) {                    // the wavefronts' shares of a column, in a fixed order
        __syncthreads();
        float *part = reinterpret_cast<float *>(lds);         // [WJ][2][BM]
#pragma unroll
        for (int m = 0; m < MI; ++m) part[(wj * 2 + half) * Sh::BM + (m * WI + wi) * 32 + (lane & 31)] = bias_part[m];
        __syncthreads();
        for (int i = tid; i < Sh::BM; i += Sh::kThreads) {
            if (i >= w.rows_a) continue;
            float sum = 0;
            for (int p = 0; p < 2 * WJ; ++p) sum += part[p * Sh::BM + i];
            g.d_bias[(int64_t)w.group * g.N + w.i0 + i] = sum;
        }
    }
}

template <Job JOB, int WI, int WJ, int WC, int MI, int NJ, int S>
__global__ __launch_bounds__(WI *WJ *WC * 64) void expert_gemm_tiles(const GemmArgs g)
{
    typedef Shape<JOB, WI, WJ, WC, MI, NJ, S> Sh;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    Work w;
    if constexpr (JOB == Job::weights) {
        const int ti = (g.N + Sh::BM - 1) / Sh::BM, tj = (g.K + Sh::BN - 1) / Sh::BN;
        const int tile = blockIdx.x % (ti * tj), group = blockIdx.x / (ti * tj);
        const int from = g.offsets ? max(0, min(g.M, g.offsets[group])) : 0, to = g.offsets ? max(0, min(g.M, g.offsets[group + 1])) : g.M;
        w.group = group, w.i0 = tile / tj * Sh::BM, w.j0 = tile % tj * Sh::BN;
        w.a = g.a + ((int64_t)from * g.lda + w.i0) * 2, w.b = g.b + ((int64_t)from * g.ldb + w.j0) * 2;
        w.rows_a = min(Sh::BM, g.N - w.i0), w.rows_b = min(Sh::BN, g.K - w.j0), w.c = max(0, to - from);
    } else {
        const int cols = JOB == Job::product ? g.N : g.K;
        const Placed at = place<Sh::BM>(g, (cols + Sh::BN - 1) / Sh::BN);
        if (at.rows == 0) return;
        w.group = at.group, w.i0 = at.row0, w.j0 = at.nt * Sh::BN;
        w.a = g.a + (int64_t)at.row0 * g.lda * 2;
        w.b = g.b + (at.group * g.b_group + (JOB == Job::product ? w.j0 * g.ldb : (int64_t)w.j0)) * 2;
        w.rows_a = at.rows, w.rows_b = min(Sh::BN, cols - w.j0), w.c = JOB == Job::product ? g.K : g.N;
    }
    w.pitch_a = (uint32_t)g.lda * 2, w.pitch_b = (uint32_t)g.ldb * 2;
    take_tile<Sh, JOB, WI, WJ, WC, MI, NJ, S>(g, w, lds);
}

template <Job JOB, int WI, int WJ, int WC, int MI, int NJ, int S>
int launch_shape(const GemmArgs &g, hipStream_t st)
{
    typedef Shape<JOB, WI, WJ, WC, MI, NJ, S> Sh;
    static LdsGrant grant;
    const void *kernel = (const void *)expert_gemm_tiles<JOB, WI, WJ, WC, MI, NJ, S>;
    const int e = allow_lds(grant, kernel, Sh::kLds);
    if (e) return e;
    int64_t grid;
    if (JOB == Job::weights) {
        grid = (int64_t)g.groups * ((g.N + Sh::BM - 1) / Sh::BM) * ((g.K + Sh::BN - 1) / Sh::BN);
    } else {
        const int cols = JOB == Job::product ? g.N : g.K;
        const int64_t tiles = g.M / Sh::BM + (g.groups < g.M ? g.groups : g.M);
        grid = (tiles * ((cols + Sh::BN - 1) / Sh::BN) + 7) / 8 * 8;
    }
    expert_gemm_tiles<JOB, WI, WJ, WC, MI, NJ, S><<<(uint32_t)grid, Sh::kThreads, Sh::kLds, st>>>(g);
    return (int)hipGetLastError();
}

GemmArgs args_of(const ExpertGemmShape &s, const int32_t *offsets, int32_t M)
{
    GemmArgs g{};
    g.offsets = offsets, g.M = M, g.groups = s.groups, g.N = s.N, g.K = s.K, g.out32 = s.out32, g.activation = s.activation;
    return g;
}

}  // namespace

int launch_expert_gemm(const ExpertGemmShape &s, const void *x, int64_t ldx, int32_t M, const void *w, const int32_t *offsets, const float *bias,
                       void *pre, int64_t ld_pre, const void *residual, int64_t ld_res, void *y, int64_t ldy, hipStream_t st)
{
    GemmArgs g = args_of(s, offsets, M);
    g.a = (const char *)x, g.lda = ldx, g.b = (const char *)w, g.ldb = s.K, g.b_group = (int64_t)s.N * s.K;
    g.bias = bias, g.pre = (char *)pre, g.ld_pre = ld_pre, g.residual = (const char *)residual, g.ld_res = ld_res;
    g.out = (char *)y, g.ldo = ldy;
    return launch_shape<Job::product, 2, 2, 1, 2, 2, 2>(g, st);
}

int launch_expert_gemm_input(const ExpertGemmShape &s, const void *dy, int64_t ld_dy, int32_t M, const void *w, const int32_t *offsets, const void *pre,
                             int64_t ld_pre, void *dx, int64_t ld_dx, hipStream_t st)
{
    GemmArgs g = args_of(s, offsets, M);
    g.a = (const char *)dy, g.lda = ld_dy, g.b = (const char *)w, g.ldb = s.K, g.b_group = (int64_t)s.N * s.K;
    g.pre = (char *)const_cast<void *>(pre), g.ld_pre = ld_pre;
    g.out = (char *)dx, g.ldo = ld_dx;
    return launch_shape<Job::input, 2, 2, 1, 2, 2, 2>(g, st);
}

int launch_expert_gemm_weights(const ExpertGemmShape &s, const void *dy, int64_t ld_dy, const void *x, int64_t ldx, int32_t M, const int32_t *offsets,
                               void *dw, float *d_bias, void *, hipStream_t st)
{
    GemmArgs g = args_of(s, offsets, M);
    g.a = (const char *)dy, g.lda = ld_dy, g.b = (const char *)x, g.ldb = ldx;
    g.out = (char *)dw, g.ldo = s.K, g.out_group = (int64_t)s.N * s.K, g.d_bias = d_bias;
    return launch_shape<Job::weights, 2, 2, 1, 2, 2, 2>(g, st);
}

}  // namespace sida
