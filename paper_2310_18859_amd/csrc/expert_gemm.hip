// Grouped products of plain bf16 experts, forward and backward, for the rows r of group g (sums in fp32, one rounding at the end):
//     product   v = W_g x[r] + b_g,  y[r] = act(v) + residual[r]             sum over K
//     input     dx[r] = (W_g^T dy[r]) act'(pre[r])                           sum over N
//     weights   dW_g = sum_r dy[r] x[r]^T,  db_g = sum_r dy[r]               sum over the group's rows
// One tile routine serves the three: C[i,j] = sum_c A[i,c] B[j,c], where an operand lies with c along its rows in memory (x, dy, and W in
// the product) or with c across them (W in `input`, both operands in `weights`).
//
// What bounds it, 32768 rows over 64 experts of 4096 x 1024 (Zipf 1.0), bf16: 2.7e11 operations are 196 us at 1.4 PFLOP/s, which a large library product
// reaches here; bytes in and out are as many.  Measured: product with bias, GELU and the values in front of it kept 414 to 432 us, the input's gradient 417 to
// 448, the weights' 449 to 478, by the card.  The matrix cores are busy 32, 31 and 26 % of the cycles (64 % of those of 8192 cubed): a workgroup has the compute unit
// to itself, which multiplies nothing while a tile's results leave, so that bytes and products overlap in part only; the weights' gradient deals its tiles out
// unevenly besides (groups_by_rows).  The compute clock falls to 1.6 to 2.0 GHz under them.  One card: 64 groups of 512 rows, without extras, 287, 260 and 355 us (product,
// input's, weights' gradient), the library's batched product of the same 281; one matrix of 32768 x 4096 x 1024 takes the library 232, 221 and 321, the kernels
// here 266, 235 and 302.
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

enum class Job { product, input, weights, parts };           // parts: the weights' gradient of `chunk` rows at a time, to be added up

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
    int chunk, parts;            // parts: rows of a part, and parts at most, more than which only offsets that do not ascend would make
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void *base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}
// 16 bytes a lane straight into LDS: lane i's land at dst + 16 i.  Written out, because the compiler waits for all that it knows to be on its way to LDS
// in front of each transposing read (8192 cubed, the input's gradient: 1089 us against 947); it has no register as its result, and waits that the compiler
// counts without it wait longer, never shorter.  The pause: M0, and scalar registers that a vector instruction wrote, are not there at once, and inside the
// statement the compiler does not see to that.
__device__ __forceinline__ i32x4 lds_source(const char *base, uint32_t bytes)
{
    return i32x4{(int)(uint32_t)(uint64_t)base, (int)((uint64_t)base >> 32 & 0xffff), (int)bytes, 0x00020000};
}
__device__ __forceinline__ void load_to_lds(i32x4 source, uint32_t offset, uint32_t dst)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(offset), "s"(source) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// A uniform value that the compiler cannot see through: it makes one copy of the code that depends on it, not one for each value.
__device__ __forceinline__ int hidden(int v)
{
    v = __builtin_amdgcn_readfirstlane(v);
    asm("" : "+s"(v));
    return v;
}
// What is the same in all lanes, in scalar registers whatever the compiler makes of where it comes from: a descriptor out of vector registers
// costs a loop around its access.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const char *uniform(const char *p)
{
    const uint64_t v = (uint64_t)p;
    return (const char *)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}
// A value that the compiler cannot see through: what follows from it is worked out where it is used, rather than held in registers all the time.
__device__ __forceinline__ int anew(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}
// A descriptor's records, and a lane offset past them: such a load asks for nothing and brings zeros.  256 rows are at most
// kMostExpertPitch bytes apart, so that every offset that is meant lies below.
constexpr uint32_t kRecords = 0x80000000u, kNowhere = 0xffffff00u;

// ---- which tiles a workgroup takes --------------------------------------------------------------
// A tile: where its operands and its result lie.
struct Work {
    const char *a, *b;           // the tile's first row, at c = 0
    int rows_a, rows_b, c;       // rows of the tile that are there, length of the sum
    int i0, j0;                  // first row and column of the result
    int group, to;               // to (weights): which of the result's matrices, the group's or the part's
};

// Where the groups begin, four of them to a lane.
struct Groups {
    int at[5];
    __device__ __forceinline__ explicit Groups(const GemmArgs &g)
    {
        const int lane = threadIdx.x & 63;
        if (!g.offsets) {
#pragma unroll
            for (int i = 0; i < 5; ++i) at[i] = i || lane ? g.M : 0;
        } else {
            const __amdgpu_buffer_rsrc_t r = make_rsrc(g.offsets, (uint32_t)(g.groups + 1) * 4);   // entries past the last one come as zeros
#pragma unroll
            for (int i = 0; i < 5; ++i) at[i] = max(0, min(g.M, (int)__builtin_amdgcn_raw_buffer_load_b32(r, lane * 16 + i * 4, 0, 0)));
        }
    }
    // The rows of a group, the same in all lanes.
    __device__ __forceinline__ void rows(int group, int &from, int &n) const
    {
        int begin = 0, end = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            begin = (group & 3) == i ? at[i] : begin;
            end = (group & 3) == i ? at[i + 1] : end;
        }
        from = __builtin_amdgcn_readlane(begin, group >> 2);
        n = max(0, __builtin_amdgcn_readlane(end, group >> 2) - from);
    }
};

// Row tiles of `tall` rows are counted group by group; a lane knows how many there are up to its last group.
struct RowTiles : Groups {
    int tall, upto, total;
    __device__ __forceinline__ RowTiles(const GemmArgs &g, int tall_) : Groups(g), tall(tall_)
    {
        const int lane = threadIdx.x & 63;
        upto = tiles();
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(upto, d);
            upto += lane >= d ? v : 0;
        }
        total = __builtin_amdgcn_readlane(upto, 63);
    }
    __device__ __forceinline__ int tiles_of(int i) const { return (max(0, at[i + 1] - at[i]) + tall - 1) / tall; }
    __device__ __forceinline__ int tiles() const { return tiles_of(0) + tiles_of(1) + tiles_of(2) + tiles_of(3); }
    // Of row tile mt: its group, first row and number of rows.
    __device__ __forceinline__ void find(int mt, int &group_of, int &row0_of, int &rows_of) const
    {
        const int owner = __builtin_ctzll(__ballot(upto > mt));
        int left = mt - (upto - tiles()), group = 0, row0 = 0, rows = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = tiles_of(i);
            if (left >= 0 && left < n) {
                group = (threadIdx.x & 63) * 4 + i;
                row0 = at[i] + left * tall;
                rows = min(tall, at[i + 1] - row0);
            }
            left -= n;
        }
        group_of = __builtin_amdgcn_readlane(group, owner);
        row0_of = __builtin_amdgcn_readlane(row0, owner);
        rows_of = __builtin_amdgcn_readlane(rows, owner);
    }
    // Of a group: its first row tile and how many it has.
    __device__ __forceinline__ void of(int group, int &first, int &n) const
    {
        int before = upto - tiles(), mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            before += i < (group & 3) ? tiles_of(i) : 0;
            mine = i == (group & 3) ? tiles_of(i) : mine;
        }
        first = __builtin_amdgcn_readlane(before, group >> 2);
        n = __builtin_amdgcn_readlane(mine, group >> 2);
    }
};

// The groups by their number of rows, the largest first; the lower of equal ones: a tile's cost is its group's rows (weights), and workgroups that take their last
// tiles at about the same time are to have short ones then.  Four to a lane, a byte each.  It does not even out what they have altogether, as they take
// tiles in fixed turns (Items): of 64 groups of 4096 x 1024 with 32768 rows (Zipf 1.0) the same two XCDs get the largest of every four, 198 stages a workgroup,
// where the mean is 138 and the least 104 (449 to 478 us, by the card).  Even groups have 135 each (355 to 374 us).
template <int THREADS>
__device__ __forceinline__ uint32_t groups_by_rows(const Groups &groups, int n_groups, char *lds)
{
    int *rows = reinterpret_cast<int *>(lds);                 // [256]
    uint8_t *order = reinterpret_cast<uint8_t *>(lds + 1024); // [256]
    const int tid = threadIdx.x;
    if (tid < 64) {
#pragma unroll
        for (int i = 0; i < 4; ++i) rows[tid * 4 + i] = max(0, groups.at[i + 1] - groups.at[i]);
    }
    __syncthreads();
    for (int i = tid; i < n_groups; i += THREADS) {
        const int mine = rows[i];
        int rank = 0;
        for (int j = 0; j < n_groups; ++j) {
            const int n = rows[j];
            rank += n > mine || (n == mine && j < i) ? 1 : 0;
        }
        order[rank] = (uint8_t)i;
    }
    __syncthreads();
    const uint32_t mine = reinterpret_cast<const uint32_t *>(order)[tid & 63];
    __syncthreads();
    return mine;
}

// ---- operand tiles in LDS -----------------------------------------------------------------------
// KB values of c at a time, by loads of 1 KiB that go straight into LDS, lane i's 16 bytes to 16 i.
//   ALONG   c along a row: rows of 2 KB bytes, their 16-byte pieces moved by the row, so that neither the loads nor the reads of
//           one piece of 32 rows meet in a bank
//   ACROSS  KB rows of c, each with the tile's columns; the 64-byte chunk of 32 columns that a fragment takes is moved
//           by the row, so that the four rows of a transposing read lie in four quarters of the banks
// No bank conflict is left in any of the three products.  KB = 64: segments of 64 bytes (KB = 32) would ask L2 twice as often.
template <bool ACROSS, int ROWS, int KB>
struct Tile {
    static constexpr int kBytes = ROWS * KB * 2;
    static constexpr int kPitch = ACROSS ? ROWS * 2 : KB * 2;
    static constexpr int kLoads = kBytes / 1024;
    static __device__ __forceinline__ int turn(int r)
    {
        if (ACROSS) return kPitch >= 256 ? r & 3 : kPitch == 128 ? r >> 1 & 1 : 0;
        return KB == 64 ? r >> 1 & 7 : r >> 2 & 3;
    }
    // Byte offset of a lane's piece of load `w` from the tile's first value, and its c; `rows` of the tile are there.
    static __device__ __forceinline__ void lane_at(int w, int lane, int rows, uint32_t pitch, uint32_t &offset, int &c)
    {
        const int at = w * 1024 + lane * 16, r = at / kPitch, b = at % kPitch;
        if constexpr (ACROSS) {
            const int col = ((b / 64 ^ turn(r)) * 64 + b % 64) / 2;
            c = r;
            offset = col < rows ? (uint32_t)r * pitch + col * 2 : kNowhere;
        } else {
            const int piece = b / 16 ^ turn(r);
            c = piece * 8;
            offset = r < rows ? (uint32_t)r * pitch + piece * 16 : kNowhere;
        }
    }
    // A lane's part of the fragment of 32 rows from row 32 m and 16 c from 16 q: lane l has row l % 32, c 8 (l / 32) .. + 7.
    static __device__ __forceinline__ bf16x8 fragment(const char *tile, int lane, int m, int q)
    {
        if constexpr (ACROSS) {
            // Sixteen lanes read four rows of c, 16 columns each, and get a column each.
            const int g = lane >> 4, r = 8 * (g >> 1) + (lane >> 2 & 3);
            const char *at = tile + (16 * q + r) * kPitch + (m ^ turn(r)) * 64 + (g & 1) * 32 + (lane & 3) * 8;
            typedef __attribute__((address_space(3))) s16x4 lds4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 4 * kPitch + ((m ^ turn(r + 4)) - (m ^ turn(r))) * 64));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int r = lane & 31;
            return *reinterpret_cast<const bf16x8 *>(tile + (m * 32 + r) * kPitch + ((2 * q + (lane >> 5)) ^ turn(r)) * 16);
        }
    }
};

// ---- epilogue -----------------------------------------------------------------------------------
constexpr float kLog2e = 1.44269504088896340736f, kGelu = 0.79788456080286535588f, kGelu3 = 0.044715f;
// Both smooth activations are v sigmoid(u): u = v, or for GELU in its form with tanh twice the tanh's argument.  One way through the code for the two:
// -u log2 e = v (c0 + c1 v^2), du/dv = d0 + d1 v^2.
struct Act {
    int kind;                    // kActNone, kActRelu, or else smooth
    float c0, c1, d0, d1, most;
    __device__ __forceinline__ explicit Act(int act)
    {
        const bool gelu = act == kActGelu;
        kind = act;
        c0 = gelu ? -2 * kGelu * kLog2e : -kLog2e, c1 = gelu ? -2 * kGelu * kGelu3 * kLog2e : 0.f;
        d0 = gelu ? 2 * kGelu : 1.f, d1 = gelu ? 2 * kGelu * 3 * kGelu3 : 0.f;
        most = gelu ? 9.f : 80.f;
    }
    __device__ __forceinline__ float smooth(float v) const
    {
        const float v2 = fminf(v * v, 1e30f);                // 0 times infinity would be NaN
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * (c0 + c1 * v2)));
        return s == 0.f ? 0.f : v * s;                       // also at -infinity
    }
    // s + v s (1 - s) du/dv, with 1 - s = exp(-u) s, which loses nothing where s is close to 1.  Beyond +-80 (SiLU) and +-9 (GELU) the slope is 0 or 1 to
    // within 2^-80; there the powers of v and exp(-u) would give infinity times 0.
    __device__ __forceinline__ float smooth_slope(float v) const
    {
        v = v > most ? most : v < -most ? -most : v;         // NaN stays
        const float e = __builtin_amdgcn_exp2f(v * (c0 + c1 * (v * v))), s = __builtin_amdgcn_rcpf(1.f + e);
        return s + v * (e * s) * s * (d0 + d1 * (v * v));
    }
};
__device__ __forceinline__ float relu_of(float v) { return v <= 0.f ? 0.f : v; }                     // NaN stays
__device__ __forceinline__ float relu_slope(float v) { return v > 0.f ? 1.f : v <= 0.f ? 0.f : v; }  // the same

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
__device__ __forceinline__ void activate(const Act &act, int kind, F8 &f)
{
    if (kind >= kActGelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = act.smooth(f.v[e]);
    } else if (kind == kActRelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = relu_of(f.v[e]);
    }
}
__device__ __forceinline__ void times_slope(const Act &act, int kind, F8 &f, const F8 &pre)
{
    if (kind >= kActGelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] *= act.smooth_slope(pre.v[e]);
    } else if (kind == kActRelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] *= relu_slope(pre.v[e]);
    }
}
// Eight values from `at`, in values; kNone: none (zeros, nothing stored).
constexpr uint32_t kNone = kNowhere;
__device__ __forceinline__ F8 read8(__amdgpu_buffer_rsrc_t r, uint32_t at, bool f32)
{
    if (!f32) return widen(__builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(at == kNone ? kNowhere : at * 2), 0, 0)));
    const int from = (int)(at == kNone ? kNowhere : at * 4);
    const f32x4 lo = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, from, 0, 0));
    const f32x4 hi = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, from, 16, 0));
    return F8{{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}};
}
__device__ __forceinline__ void write8(__amdgpu_buffer_rsrc_t r, uint32_t at, bool f32, const F8 &f)
{
    typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
    if (f32) {
        const int to = (int)(at == kNone ? kNowhere : at * 4);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{f.v[0], f.v[1], f.v[2], f.v[3]}), r, to, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{f.v[4], f.v[5], f.v[6], f.v[7]}), r, to, 16, 0);
        return;
    }
    bf16x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)f.v[i];
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, (int)(at == kNone ? kNowhere : at * 2), 0, 0);
}

// A workgroup's tile: WI x WJ wavefronts, each MI x NJ blocks of 32 x 32 (rows' blocks dealt in turn, so that a short tile keeps all busy);
// SA and SB stages of KB values of c of the two operands in LDS.
template <Job JOB, int WI, int WJ, int MI, int NJ, int SA, int SB, int KB>
struct Shape {
    static constexpr bool kAcrossA = JOB == Job::weights || JOB == Job::parts, kAcrossB = JOB != Job::product;
    static constexpr int kWaves = WI * WJ, kThreads = kWaves * 64;
    static constexpr int BM = 32 * MI * WI, BN = 32 * NJ * WJ;
    typedef Tile<kAcrossA, BM, KB> A;
    typedef Tile<kAcrossB, BN, KB> B;
    static_assert(A::kLoads % kWaves == 0 && B::kLoads % kWaves == 0, "loads are dealt evenly");
    static_assert(kWaves % 4 == 0, "a lane has the same piece in all of its loads along c");
    static constexpr int kLoadsA = A::kLoads / kWaves, kLoadsB = B::kLoads / kWaves;   // of a wavefront and stage
    // The operand that is further ahead, by one stage, is asked for behind the other, so that waiting for that leaves it out.
    static constexpr bool kLeadB = SB > SA;
    static constexpr int S = SA < SB ? SA : SB, kMost = SA > SB ? SA : SB;
    static_assert(S >= 2 && kMost - S <= 1, "stages");
    static constexpr int kLater = (S - 2) * (kLoadsA + kLoadsB) + (SA > SB ? kLoadsA : SB > SA ? kLoadsB : 0);   // loads behind the ones waited for
    static constexpr int kLds = SA * A::kBytes + SB * B::kBytes;
    static constexpr int kPerUnit = kLds <= 80 * 1024 ? 2 : 1;                          // workgroups to a compute unit
};

// One operand's loads: a ring of S stages in LDS, and where the next stage comes from.  A lane's offsets are from where a stage begins in memory; along c its
// first value of c says whether a stage that is not whole, the last one of a tile, has something for it; across c the descriptor ends with the last row.
template <class T, bool ACROSS, int S, int KB, int WAVES>
struct Ring {
    static constexpr int kLoads = T::kLoads / WAVES;
    uint32_t off[kLoads], lds_at, pitch;
    int c;
    const char *from = nullptr;
    int left = 0, to_load = 0, slot = 0;                      // values of c, and stages, of the tile that are still to be asked for
    i32x4 source;
    uint32_t dst;
    __device__ __forceinline__ Ring(uint32_t lds, uint32_t pitch_, int wave) : lds_at(lds + wave * 1024), pitch(pitch_) {}
    __device__ __forceinline__ void begin(const char *tile, int rows, int length, int stages, int lane, int wave)
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) T::lane_at(i * WAVES + wave, lane, rows, pitch, off[i], c);
        from = tile, left = length, to_load = stages;
    }
    __device__ __forceinline__ void end() { left = 0, to_load = INT32_MAX; }              // asks for nothing from now on
    __device__ __forceinline__ void prepare()
    {
        if (!ACROSS && (left & (KB - 1)) && left < KB) {      // the tile's last stage, and not a whole one (a comparison at each load instead: 2 to 3 %)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) off[i] = c < left ? off[i] : kNowhere;
        }
        source = lds_source(from, (uint32_t)uniform((int)(ACROSS ? (uint32_t)min(left, KB) * pitch : left ? kRecords : 0)));
        dst = lds_at + slot * T::kBytes;
        left -= min(left, KB);
        from += left > 0 ? (ACROSS ? (int64_t)KB * pitch : KB * 2) : 0;
        --to_load;
        slot = slot == S - 1 ? 0 : slot + 1;
    }
    __device__ __forceinline__ void load(int i) { load_to_lds(source, off[i], dst + i * WAVES * 1024); }
};

template <int I>
struct Int {
    static constexpr int value = I;
};

// A workgroup walks over its tiles, and treats them as one stream of stages: while one stage is multiplied, the next ones are on their way, those of
// the next tile too, so that neither the results of a tile nor the search for the next one keep loads waiting.  Every tile has as many stages as there are
// in LDS at least, so that the stream is never more than one tile ahead.
//
// The shapes.  256 x 256 (eight wavefronts of 128 x 64; two stages of A, three of B, all of the 160 KiB): a value brought in goes into 256 products,
// a fragment read from LDS into 2.7 matrix instructions on average, with 128 x 128 (four wavefronts of 64 x 64, two workgroups to a compute unit that cover each
// other's results) into 128 and 2: 258 and 315 us for 64 groups of 512 rows, input's gradient of 4096 x 1024.  But it takes many tiles to fill 256 compute units
// evenly.  Wavefronts of 128 x 128 spill.
// 32 x 128 and 64 x 256 are for groups of few rows, which are bound by bringing the experts' matrices in (1111 rows over 64 experts of 1024 x 2048, input's
// gradient: 61 us at best for 45 of bytes).  The rule and its measurements: expert_rule.h.
template <Job JOB, int WI, int WJ, int MI, int NJ, int SA, int SB, int KB>
__global__ __launch_bounds__(WI *WJ * 64, (Shape<JOB, WI, WJ, MI, NJ, SA, SB, KB>::kWaves * Shape<JOB, WI, WJ, MI, NJ, SA, SB, KB>::kPerUnit / 4)) void expert_gemm_tiles(const GemmArgs g)
{
    typedef Shape<JOB, WI, WJ, MI, NJ, SA, SB, KB> Sh;
    typedef typename Sh::A A;
    typedef typename Sh::B B;
    constexpr int S = Sh::S;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wj = wave % WJ, wi = wave / WJ;
    const int cols = JOB == Job::product ? g.N : g.K, col_tiles = (cols + Sh::BN - 1) / Sh::BN;

    // ---- the tiles
    constexpr bool kWeights = Sh::kAcrossA;
    const int tiles_i = kWeights ? (g.N + Sh::BM - 1) / Sh::BM : 0;
    std::conditional_t<JOB == Job::weights, Groups, RowTiles> rows = [&] {
        if constexpr (JOB == Job::weights) return Groups(g);
        else return RowTiles(g, JOB == Job::parts ? g.chunk : Sh::BM);
    }();
    uint32_t order = 0;
    int64_t total;
    if constexpr (JOB == Job::weights) {
        order = groups_by_rows<Sh::kThreads>(rows, g.groups, lds);
        total = (int64_t)g.groups * tiles_i * col_tiles;
    } else {
        total = (int64_t)(JOB == Job::parts ? min(rows.total, g.parts) * tiles_i : rows.total) * col_tiles;
    }
    Items items(total, gridDim.x, kItemsInARow, blockIdx.x);
    // Zeros for a tile of a group without rows: no stages are spent on it.
    auto clear = [&](const Work &w) {
        const int of = g.out32 ? 4 : 8, pieces = w.rows_b / of;
        char *to = g.out + (w.to * g.out_group + (int64_t)w.i0 * g.ldo + w.j0) * (g.out32 ? 4 : 2);
        for (int p = tid; p < w.rows_a * pieces; p += Sh::kThreads)
            *reinterpret_cast<i32x4 *>(to + ((int64_t)(p / pieces) * g.ldo + p % pieces * of) * (g.out32 ? 4 : 2)) = i32x4{0, 0, 0, 0};
        if (g.d_bias && w.j0 == 0)
            for (int i = tid; i < w.rows_a; i += Sh::kThreads) g.d_bias[(int64_t)w.to * g.N + w.i0 + i] = 0.f;
    };
    auto next_item = [&](Work &w) {
        const int id = items.next();
        if (id < 0) return false;
        if constexpr (kWeights) {
            const int at = id / (tiles_i * col_tiles), tile = id % (tiles_i * col_tiles);
            int from;
            if constexpr (JOB == Job::weights) {
                w.to = w.group = __builtin_amdgcn_readlane(order, at >> 2) >> (at & 3) * 8 & 255;
                rows.rows(w.group, from, w.c);
            } else {
                w.to = at;
                rows.find(at, w.group, from, w.c);
            }
            w.i0 = tile / col_tiles * Sh::BM, w.j0 = tile % col_tiles * Sh::BN;
            w.a = g.a + ((int64_t)from * g.lda + w.i0) * 2, w.b = g.b + ((int64_t)from * g.ldb + w.j0) * 2;
            w.rows_a = min(Sh::BM, g.N - w.i0);
        } else {
            w.to = 0;
            // A matrix of its own (one group) is walked four rows of tiles at a time: an XCD's 32 tiles are 4 x 8 of them rather than 1 x 32, and L2 is asked for
            // fewer lines that it has not got (8192 cubed: 1018 to 967 us; 32768 rows, 4096 x 1024, input's gradient: 300 to 293).  With 64 groups of
            // a few rows of tiles each it makes no difference (415 and 416 us, Zipf 1.0).
            const int together = g.groups == 1 ? 4 : 1, before = id / (together * col_tiles) * together, at = id - before * col_tiles;
            const int tall = min(together, rows.total - before);
            rows.find(before + at % tall, w.group, w.i0, w.rows_a);
            w.j0 = at / tall * Sh::BN;
            w.a = g.a + (int64_t)w.i0 * g.lda * 2;
            w.b = g.b + (w.group * g.b_group + (JOB == Job::product ? w.j0 * g.ldb : (int64_t)w.j0)) * 2;
            w.c = JOB == Job::product ? g.K : g.N;
        }
        w.rows_b = min(Sh::BN, cols - w.j0);
        w = Work{uniform(w.a), uniform(w.b), uniform(w.rows_a), uniform(w.rows_b), uniform(w.c), uniform(w.i0), uniform(w.j0), uniform(w.group), uniform(w.to)};
        return true;
    };
    auto next = [&](Work &w) {
        while (true) {
            if (!next_item(w)) return false;
            if (JOB != Job::weights || w.c > 0) return true;
            clear(w);
        }
    };
    auto stages_of = [&](const Work &w) { return max(Sh::kMost, (w.c + KB - 1) / KB); };

    // ---- loads
    const uint32_t lds_at = (uint32_t)uniform((int)(uintptr_t)(__attribute__((address_space(3))) char *)lds);
    Ring<A, Sh::kAcrossA, SA, KB, Sh::kWaves> ra(lds_at, (uint32_t)g.lda * 2, wave);
    Ring<B, Sh::kAcrossB, SB, KB, Sh::kWaves> rb(lds_at + SA * A::kBytes, (uint32_t)g.ldb * 2, wave);
    Work ahead;                                               // the tile that is loaded
    bool more = true;
    auto begin_a = [&] {
        if (!Sh::kLeadB) more = next(ahead);
        const int l = anew(lane);
        if (more) ra.begin(ahead.a, ahead.rows_a, ahead.c, stages_of(ahead), l, wave);
        else ra.end();
    };
    auto begin_b = [&] {
        if (Sh::kLeadB) more = next(ahead);
        const int l = anew(lane);
        if (more) rb.begin(ahead.b, ahead.rows_b, ahead.c, stages_of(ahead), l, wave);
        else rb.end();
    };
    // The next stage of each operand; the leading one finds the next tile.
    auto prepare_a = [&] {
        if (ra.to_load == 0) begin_a();
        ra.prepare();
    };
    auto prepare_b = [&] {
        if (rb.to_load == 0) begin_b();
        rb.prepare();
    };
    auto prepare = [&] {
        if (Sh::kLeadB) prepare_b(), prepare_a();
        else prepare_a(), prepare_b();
    };
    constexpr int kLoads = Sh::kLoadsA + Sh::kLoadsB;
    auto load = [&](int i) {                                  // the leading operand's behind the other's
        if (Sh::kLeadB) {
            if (i < Sh::kLoadsA) ra.load(i);
            else rb.load(i - Sh::kLoadsA);
        } else {
            if (i < Sh::kLoadsB) rb.load(i);
            else ra.load(i - Sh::kLoadsB);
        }
    };

    if (Sh::kLeadB) begin_b(), begin_a();
    else begin_a(), begin_b();
    if (!more) return;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        prepare();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(i);
    }
    if constexpr (SA > S) {
        ra.prepare();
#pragma unroll
        for (int i = 0; i < Sh::kLoadsA; ++i) ra.load(i);
    }
    if constexpr (SB > S) {
        rb.prepare();
#pragma unroll
        for (int i = 0; i < Sh::kLoadsB; ++i) rb.load(i);
    }
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    int slot_a = 0, slot_b = 0;

    // A tile of which this wavefront has `blocks` blocks of rows.
    auto take = [&](const Work &w, auto blocks, auto with_bias) {
        constexpr int MB = decltype(blocks)::value, MR = MB ? MB : 1, Q = KB / 16;
        const int stages = stages_of(w), whole = (w.c + KB - 1) / KB;                         // those that hold something
        f32x16 acc[MR][NJ];
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int n = 0; n < NJ; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][n][r] = 0;
        // Sums of dy's columns (weights, the tiles of the first columns of x); of the wavefronts that have the same rows the one with column m % WJ sums block m.
        constexpr bool BIAS = decltype(with_bias)::value;
        constexpr int kShare = (MR + WJ - 1) / WJ;
        float bias_part[kShare] = {};

        // Fragments of 16 values of c are read one step of products ahead, the first ones of a stage behind the barrier that says that the stage is
        // there; that stands in front of the last products of the stage before, so that nobody waits for LDS with idle matrix cores.
        bf16x8 fa[2][MR], fb[2][NJ];
        auto fetch = [&](int q, int to) {
            if constexpr (MB > 0) {
                const char *ta = lds + slot_a * A::kBytes, *tb = lds + SA * A::kBytes + slot_b * B::kBytes;
#pragma unroll
                for (int n = 0; n < NJ; ++n) fb[to][n] = B::fragment(tb, lane, wj * NJ + n, q);
#pragma unroll
                for (int m = 0; m < MB; ++m) fa[to][m] = A::fragment(ta, lane, m * WI + wi, q);
            }
        };
        // One block of rows' products of a step.
        auto block = [&](int q, int m) {
            const int of = q & 1;
#pragma unroll
            for (int n = 0; n < NJ; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[of][n], fa[of][m], acc[m][n], 0, 0, 0);
        };
        // A wavefront's share is read for it a second time: its number is not known to the compiler, and registers have no index.
        auto add_bias = [&](int q) {
            if constexpr (BIAS && MB > 0) {
                const char *ta = lds + slot_a * A::kBytes;
#pragma unroll
                for (int k = 0; k < kShare; ++k) {
                    const int m = wj + k * WJ;
                    const F8 f = widen(A::fragment(ta, lane, (m < MB ? m : 0) * WI + wi, q));
                    bias_part[k] += ((f.v[0] + f.v[1]) + (f.v[2] + f.v[3])) + ((f.v[4] + f.v[5]) + (f.v[6] + f.v[7]));
                }
            }
        };
        // The next stage is there, and nobody reads this one any more.  The first S stages of a tile are there when it begins: they are waited for in front of
        // the stores of the tile before, so that no wait for them is one for stores.
        int there = S - 1;                                    // stages that are, besides the one that is multiplied
        auto arrived = [&] {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            there = hidden(there - 1);
            if (there < 0) wait_loads<Sh::kLater>();
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        auto go_on = [&] {                                    // to the next stage
            slot_a = slot_a == SA - 1 ? 0 : slot_a + 1;
            slot_b = slot_b == SB - 1 ? 0 : slot_b + 1;
            prepare();
            arrived();
        };
        if (whole > 0) fetch(0, 0);
#pragma clang loop unroll(disable)
        for (int t = 0; t < whole; ++t) {
#pragma unroll
            for (int q = 0; q < Q - 1; ++q) {
                fetch(q + 1, q + 1 & 1);
#pragma unroll
                for (int m = 0; m < MB; ++m) block(q, m);
                add_bias(q);
                __builtin_amdgcn_sched_barrier(0);
            }
            add_bias(Q - 1);
            go_on();
            if (t + 1 < whole) fetch(0, 0);                   // the next tile's first are read when it begins
            // The loads of the stage that takes this one's place, between the products of its last step.
            constexpr int kEach = (kLoads + MR - 1) / MR;
#pragma unroll
            for (int m = 0; m < MR; ++m) {
#pragma unroll
                for (int i = m * kEach; i < (m + 1) * kEach && i < kLoads; ++i) load(i);
                if (MB > 0) block(Q - 1, m);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma clang loop unroll(disable)
        for (int t = whole; t < stages; ++t) {                // stages that hold nothing: sums shorter than the ring (a check in the loop above costs 2 to 6%)
            go_on();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load(i);
        }

        // ---- results.  A lane holds four times four consecutive columns of one row of a block, lane ^ 32 the four beside them.  Two exchanges, between
        // halves and between quarters of the wavefront, leave it with eight consecutive columns of one row of the block's upper half and eight of the lower:
        // four lanes hold 64 consecutive bytes in bf16, which is what is read and written beside them, too.
        const Act act(g.activation);
        const int size = g.out32 ? 4 : 2;
        // What a call has beside the result; the compiler is kept from making a copy of all this for each of the possibilities.
        int has_bias = g.bias != nullptr, has_pre = g.pre != nullptr, has_residual = g.residual != nullptr, out32 = g.out32, kind = act.kind;
        const __amdgpu_buffer_rsrc_t ro = make_rsrc(g.out + ((kWeights ? w.to * g.out_group : 0) + (int64_t)w.i0 * g.ldo + w.j0) * size, kRecords);
        const __amdgpu_buffer_rsrc_t rp = make_rsrc(g.pre + ((int64_t)w.i0 * g.ld_pre + w.j0) * 2, kRecords);
        const __amdgpu_buffer_rsrc_t rr = make_rsrc(g.residual + ((int64_t)w.i0 * g.ld_res + w.j0) * size, kRecords);
        const __amdgpu_buffer_rsrc_t rbias = make_rsrc(g.bias + (JOB == Job::product ? (int64_t)w.group * g.N + w.j0 : 0), kRecords);
        const int l = anew(lane), quarter = l >> 4;
        const int col0 = wj * NJ * 32 + (quarter & 1) * 16 + (quarter >> 1) * 8;              // of block n: + 32 n
        auto row_of = [&](int m, int half) { return (m * WI + wi) * 32 + half * 16 + (l & 15); };
        auto place = [&](int m, int n, int half, int64_t ld) {                                // in values
            const int i = row_of(m, half), j = col0 + n * 32;
            return i < w.rows_a && j < w.rows_b ? i * (uint32_t)ld + j : kNone;
        };
        // Beside the result is read: the bias of the tile's columns, and for each row `pre` (input, a block of rows ahead) or the residual.
        F8 bias[NJ];
        if (JOB == Job::product && has_bias) {
#pragma unroll
            for (int n = 0; n < NJ; ++n) bias[n] = read8(rbias, col0 + n * 32 < w.rows_b ? (uint32_t)(col0 + n * 32) : kNone, true);
        }
        constexpr int kAhead = JOB == Job::input ? 1 : 0;     // blocks of rows (a product's bias has the registers of a second one)
        i32x4 beside[kAhead + 1][NJ * 2], beside_high[JOB == Job::product ? NJ * 2 : 1];
        const int reads = JOB == Job::input ? has_pre : has_residual;
        auto ask = [&](int m) {
            if (kWeights || !reads) return;
#pragma unroll
            for (int p = 0; p < NJ * 2; ++p) {
                if constexpr (JOB == Job::input) {
                    const uint32_t at = place(m, p / 2, p % 2, g.ld_pre);
                    beside[m & kAhead][p] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rp, (int)(at == kNone ? kNowhere : at * 2), 0, 0));
                } else {
                    const uint32_t at = place(m, p / 2, p % 2, g.ld_res);
                    beside[m & kAhead][p] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, (int)(at == kNone ? kNowhere : at * size), 0, 0));
                    if (g.out32) beside_high[p] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, (int)(at == kNone ? kNowhere : at * 4), 16, 0));
                }
            }
        };
        if constexpr (MB > 0 && kAhead > 0) ask(0);
        wait_loads<0>();
#pragma unroll
        for (int m = 0; m < MB; ++m) {
            if (m + kAhead < MB) ask(m + kAhead);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < NJ; ++n) {
                F8 f[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float lo = acc[m][n][h * 8 + e], hi = acc[m][n][h * 8 + 4 + e];
                        const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi), false, false);
                        const uint32_t first = both[0], second = both[1];
                        f[h].v[e] = __builtin_bit_cast(float, first);
                        f[h].v[4 + e] = __builtin_bit_cast(float, second);
                    }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float lo = f[0].v[e], hi = f[1].v[e];
                    const auto both = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi), false, false);
                    const uint32_t first = both[0], second = both[1];
                    f[0].v[e] = __builtin_bit_cast(float, first);
                    f[1].v[e] = __builtin_bit_cast(float, second);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    has_bias = hidden(has_bias), has_pre = hidden(has_pre), has_residual = hidden(has_residual), out32 = hidden(out32), kind = hidden(kind);
                    F8 &v = f[h];
                    if constexpr (JOB == Job::product) {
                        if (has_bias) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) v.v[e] += bias[n].v[e];
                        }
                        if (has_pre) write8(rp, place(m, n, h, g.ld_pre), false, v);
                        activate(act, kind, v);
                        if (has_residual) {
                            const i32x4 low = beside[m & kAhead][n * 2 + h];
                            F8 s = widen(__builtin_bit_cast(bf16x8, low));
                            if (out32) {
                                const f32x4 a = __builtin_bit_cast(f32x4, low), b = __builtin_bit_cast(f32x4, beside_high[n * 2 + h]);
                                s = F8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e) v.v[e] += s.v[e];
                        }
                    } else if constexpr (JOB == Job::input) {
                        if (has_pre) {
                            const i32x4 low = beside[m & kAhead][n * 2 + h];
                            times_slope(act, kind, v, widen(__builtin_bit_cast(bf16x8, low)));
                        }
                    }
                    write8(ro, place(m, n, h, g.ldo), out32, v);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if constexpr (BIAS && MB > 0) {
#pragma unroll
            for (int k = 0; k < kShare; ++k) {
                const float sum = bias_part[k] + __shfl_xor(bias_part[k], 32);
                const int m = wj + k * WJ, i = (m * WI + wi) * 32 + (l & 31);
                if (m < MB && l < 32 && i < w.rows_a) g.d_bias[(int64_t)w.to * g.N + w.i0 + i] = sum;
            }
        }
    };
    auto take_blocks = [&](const Work &w, auto with_bias) {
        const int blocks = ((w.rows_a + 31) / 32 - wi + WI - 1) / WI;
        if (blocks <= 0) take(w, Int<0>(), with_bias);
        else if (MI == 1 || blocks == 1) take(w, Int<1>(), with_bias);
        else if (MI == 2 || blocks == 2) take(w, Int<(MI < 2 ? MI : 2)>(), with_bias);
        else if (MI == 3 || blocks == 3) take(w, Int<(MI < 3 ? MI : 3)>(), with_bias);
        else take(w, Int<MI>(), with_bias);
    };
    while (true) {
        const Work w = ahead;
        if (kWeights && g.d_bias && w.j0 == 0) take_blocks(w, std::bool_constant<kWeights>());
        else take_blocks(w, std::false_type());
        if (!more) break;
    }
}

// Few rows, few tiles: what counts is how long the way through the sum is.  A workgroup takes 32 rows and 32 columns, and its eight wavefronts share the
// sum, 64 values of c at a time in turn, each with a ring of its own in LDS and no barrier; their parts meet in LDS and are added in a fixed order.
// One row through an expert of 4096 x 1024: 6.2 us at best (a call 8.5, of 32 x 128 tiles 12.0; 8.4 MB, 1.4 us of bytes), the ways to memory of offsets, operands and bias after one another.
constexpr int kFewWaves = 8, kFewStages = 2;
template <Job JOB>
__global__ __launch_bounds__(kFewWaves * 64) void expert_gemm_few(const GemmArgs g)
{
    constexpr bool kAcross = JOB == Job::input;
    typedef Tile<false, 32, 64> A;
    typedef Tile<kAcross, 32, 64> B;
    constexpr int kStage = A::kBytes + B::kBytes, kLoads = A::kLoads, kPitch = 36;
    static_assert(A::kLoads == B::kLoads, "loads");
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cols = JOB == Job::product ? g.N : g.K, col_tiles = (cols + 31) / 32, length = JOB == Job::product ? g.K : g.N;
    const RowTiles rows(g, 32);
    Items items((int64_t)rows.total * col_tiles, gridDim.x, kFewInARow, blockIdx.x);   // a workgroup takes one
    const int id = items.next();
    if (id < 0) return;
    int group, i0, n_rows;
    rows.find(id / col_tiles, group, i0, n_rows);
    const int j0 = id % col_tiles * 32, n_cols = min(32, cols - j0);
    const uint32_t pitch_a = (uint32_t)g.lda * 2, pitch_b = (uint32_t)g.ldb * 2;
    const char *a = uniform(g.a + (int64_t)i0 * g.lda * 2);
    const char *b = uniform(g.b + (group * g.b_group + (JOB == Job::product ? j0 * g.ldb : (int64_t)j0)) * 2);
    uint32_t off_a[kLoads], off_b[kLoads];
    int c_a[kLoads], c_b[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        A::lane_at(i, lane, n_rows, pitch_a, off_a[i], c_a[i]);
        B::lane_at(i, lane, n_cols, pitch_b, off_b[i], c_b[i]);
    }
    char *mine = lds + wave * kFewStages * kStage;
    const uint32_t at = (uint32_t)uniform((int)(uintptr_t)(__attribute__((address_space(3))) char *)mine);
    auto load = [&](int s) {                                  // this wavefront's stage s; past the end it asks for nothing
        const int c0 = (s * kFewWaves + wave) * 64, there = max(0, min(64, length - c0));
        const i32x4 from_a = lds_source(a + (there ? c0 * 2 : 0), (uint32_t)uniform(there ? (int)kRecords : 0));
        const i32x4 from_b = lds_source(b + (there ? (kAcross ? c0 * (int64_t)pitch_b : c0 * 2) : 0), (uint32_t)uniform((int)(kAcross ? there * pitch_b : there ? kRecords : 0)));
        const uint32_t dst = at + s % kFewStages * kStage;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            load_to_lds(from_a, c_a[i] < there ? off_a[i] : kNowhere, dst + i * 1024);
            load_to_lds(from_b, kAcross || c_b[i] < there ? off_b[i] : kNowhere, dst + A::kBytes + i * 1024);
        }
    };
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0;
    const int stages = (length + kFewWaves * 64 - 1) / (kFewWaves * 64);
#pragma unroll
    for (int s = 0; s < kFewStages; ++s) load(s);
    for (int s = 0; s < stages; ++s) {
        wait_loads<(kFewStages - 1) * 2 * kLoads>();
        __builtin_amdgcn_sched_barrier(0);
        const char *tile = mine + s % kFewStages * kStage;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(B::fragment(tile + A::kBytes, lane, 0, q), A::fragment(tile, lane, 0, q), acc, 0, 0, 0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // read before it is written again
        __builtin_amdgcn_sched_barrier(0);
        load(s + kFewStages);
    }
    wait_loads<0>();
    __syncthreads();
    float *parts = reinterpret_cast<float *>(lds);            // [wavefronts][32 rows][kPitch]
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4 *>(parts + (wave * 32 + (lane & 31)) * kPitch + q * 8 + (lane >> 5) * 4) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    const int r = tid >> 2, j = tid % 4 * 8;
    if (r >= n_rows || j >= n_cols) return;
    F8 f{};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        const f32x4 *from = reinterpret_cast<const f32x4 *>(parts + (w * 32 + r) * kPitch + j);
        const f32x4 lo = from[0], hi = from[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) f.v[e] += lo[e], f.v[4 + e] += hi[e];
    }
    const Act act(g.activation);
    const int size = g.out32 ? 4 : 2;
    const __amdgpu_buffer_rsrc_t rp = make_rsrc(g.pre + ((int64_t)i0 * g.ld_pre + j0) * 2, kRecords);
    if constexpr (JOB == Job::product) {
        if (g.bias) {
            const F8 bias = read8(make_rsrc(g.bias + (int64_t)group * g.N + j0, kRecords), j, true);
#pragma unroll
            for (int e = 0; e < 8; ++e) f.v[e] += bias.v[e];
        }
        if (g.pre) write8(rp, r * (uint32_t)g.ld_pre + j, false, f);
        activate(act, act.kind, f);
        if (g.residual) {
            const F8 res = read8(make_rsrc(g.residual + ((int64_t)i0 * g.ld_res + j0) * size, kRecords), r * (uint32_t)g.ld_res + j, g.out32);
#pragma unroll
            for (int e = 0; e < 8; ++e) f.v[e] += res.v[e];
        }
    } else {
        if (g.pre) times_slope(act, act.kind, f, read8(rp, r * (uint32_t)g.ld_pre + j, false));
    }
    write8(make_rsrc(g.out + ((int64_t)i0 * g.ldo + j0) * size, kRecords), r * (uint32_t)g.ldo + j, g.out32, f);
}

// The parts of each group's gradient, added in their order; 0 for a group without rows.  Four values to a thread, eight parts asked for at a time; what lies
// behind a matrix's last values are the biases.  4 experts of 520 x 264 and 32 parts: 5.2 us, 20 MB and a launch.
constexpr int kAddThreads = 256, kAddAhead = 8;
__global__ __launch_bounds__(kAddThreads) void expert_weights_add(const GemmArgs g, const float *parts, const float *bias_parts)
{
    const RowTiles rows(g, g.chunk);
    const int64_t pieces = (int64_t)g.N * g.K / 4, all = pieces + (g.d_bias ? g.N / 4 : 0);
    const int64_t blocks = (all + kAddThreads - 1) / kAddThreads;
    const int group = (int)(blockIdx.x / blocks);
    const int64_t p = blockIdx.x % blocks * kAddThreads + threadIdx.x;
    int first, n;
    rows.of(group, first, n);
    n = min(n, g.parts - first);
    if (p >= all) return;
    const bool is_bias = p >= pieces;
    const int64_t step = is_bias ? g.N : (int64_t)g.N * g.K, at = (is_bias ? p - pieces : p) * 4;
    const float *from = (is_bias ? bias_parts : parts) + first * step + at;
    f32x4 sum = {0, 0, 0, 0};
    for (int c = 0; c < n; c += kAddAhead) {
        f32x4 v[kAddAhead];
#pragma unroll
        for (int i = 0; i < kAddAhead; ++i) v[i] = *reinterpret_cast<const f32x4 *>(from + min(c + i, n - 1) * step);
#pragma unroll
        for (int i = 0; i < kAddAhead; ++i)
            if (c + i < n) sum += v[i];
    }
    if (is_bias) {
        *reinterpret_cast<f32x4 *>(g.d_bias + (int64_t)group * g.N + at) = sum;
    } else if (g.out32) {
        *reinterpret_cast<f32x4 *>(g.out + (group * g.out_group + at) * 4) = sum;
    } else {
        typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
        bf16x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (__bf16)sum[e];
        *reinterpret_cast<bf16x4 *>(g.out + (group * g.out_group + at) * 2) = x;
    }
}

template <Job JOB, int WI, int WJ, int MI, int NJ, int SA, int SB, int KB>
int launch_shape(const GemmArgs &g, hipStream_t st)
{
    typedef Shape<JOB, WI, WJ, MI, NJ, SA, SB, KB> Sh;
    static LdsGrant grant;
    const void *kernel = (const void *)expert_gemm_tiles<JOB, WI, WJ, MI, NJ, SA, SB, KB>;
    const int e = allow_lds(grant, kernel, Sh::kLds);
    if (e) return e;
    int64_t tiles;                                            // at most
    if (Sh::kAcrossA) {
        const int64_t matrices = JOB == Job::parts ? g.parts : g.groups;
        tiles = matrices * ((g.N + Sh::BM - 1) / Sh::BM) * ((g.K + Sh::BN - 1) / Sh::BN);
    } else {
        const int cols = JOB == Job::product ? g.N : g.K;
        tiles = (int64_t)(g.M / Sh::BM + (g.groups < g.M ? g.groups : g.M)) * ((cols + Sh::BN - 1) / Sh::BN);
    }
    const int64_t most = Sh::kPerUnit * stream_compute_units(st), grid = tiles < most ? (tiles + 7) / 8 * 8 : most;
    expert_gemm_tiles<JOB, WI, WJ, MI, NJ, SA, SB, KB><<<(uint32_t)grid, Sh::kThreads, Sh::kLds, st>>>(g);
    return (int)hipGetLastError();
}

template <Job JOB>
int launch_few(const GemmArgs &g, hipStream_t st)
{
    static LdsGrant grant;
    constexpr int kBytes = kFewWaves * kFewStages * 8192;
    const int e = allow_lds(grant, (const void *)expert_gemm_few<JOB>, kBytes);
    if (e) return e;
    const int cols = JOB == Job::product ? g.N : g.K;
    expert_gemm_few<JOB><<<(uint32_t)expert_few_grid(g.M, g.groups, cols), kFewWaves * 64, kBytes, st>>>(g);
    return (int)hipGetLastError();
}

// Rows through experts, forward or back, by the shape that the rule picks.
template <Job JOB>
int launch_rows_job(const GemmArgs &g, hipStream_t st)
{
    const int cols = JOB == Job::product ? g.N : g.K, length = JOB == Job::product ? g.K : g.N;
    switch (expert_tiles(g.M, g.groups, cols, length, JOB == Job::input)) {
    case ExpertTiles::few: return launch_few<JOB>(g, st);
    case ExpertTiles::rows32: return launch_shape<JOB, 1, 4, 1, 1, 4, 4, 64>(g, st);
    case ExpertTiles::rows64: return launch_shape<JOB, 1, 4, 2, 2, 2, 2, 64>(g, st);
    case ExpertTiles::square128: return launch_shape<JOB, 2, 2, 2, 2, 2, 3, 64>(g, st);
    case ExpertTiles::rows256: break;
    }
    return launch_shape<JOB, 2, 4, 4, 2, 2, 3, 64>(g, st);
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
    return launch_rows_job<Job::product>(g, st);
}

int launch_expert_gemm_input(const ExpertGemmShape &s, const void *dy, int64_t ld_dy, int32_t M, const void *w, const int32_t *offsets, const void *pre,
                             int64_t ld_pre, void *dx, int64_t ld_dx, hipStream_t st)
{
    GemmArgs g = args_of(s, offsets, M);
    g.a = (const char *)dy, g.lda = ld_dy, g.b = (const char *)w, g.ldb = s.K, g.b_group = (int64_t)s.N * s.K;
    g.pre = (char *)const_cast<void *>(pre), g.ld_pre = ld_pre;
    g.out = (char *)dx, g.ldo = ld_dx;
    return launch_rows_job<Job::input>(g, st);
}

int launch_expert_gemm_weights(const ExpertGemmShape &s, const void *dy, int64_t ld_dy, const void *x, int64_t ldx, int32_t M, const int32_t *offsets,
                               void *dw, float *d_bias, void *ws, hipStream_t st)
{
    GemmArgs g = args_of(s, offsets, M);
    g.a = (const char *)dy, g.lda = ld_dy, g.b = (const char *)x, g.ldb = ldx;
    g.out = (char *)dw, g.ldo = s.K, g.out_group = (int64_t)s.N * s.K, g.d_bias = d_bias;
    g.chunk = expert_weights_chunk(M, s.groups, s.N, s.K);
    if (g.chunk == 0) {
        if (expert_weights_small(s.groups, s.N, s.K)) return launch_shape<Job::weights, 2, 2, 2, 2, 2, 3, 64>(g, st);
        return launch_shape<Job::weights, 2, 4, 4, 2, 2, 3, 64>(g, st);
    }
    g.parts = (int)expert_weights_parts(M, s.groups, g.chunk);
    GemmArgs p = g;                                           // the parts, in fp32, behind one another; then their sums of dy
    p.out = (char *)ws, p.out32 = 1;
    p.d_bias = d_bias ? (float *)ws + (int64_t)g.parts * s.N * s.K : nullptr;
    const int e = launch_shape<Job::parts, 2, 2, 2, 2, 2, 3, 64>(p, st);
    if (e) return e;
    const int64_t pieces = (int64_t)s.N * s.K / 4 + (d_bias ? s.N / 4 : 0);
    expert_weights_add<<<(uint32_t)(s.groups * ((pieces + kAddThreads - 1) / kAddThreads)), kAddThreads, 0, st>>>(g, (const float *)ws, p.d_bias);
    return (int)hipGetLastError();
}

}  // namespace sida
