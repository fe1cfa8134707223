// The way of tokens to their experts and back, as a routed layer that is trained takes it.  Pair p = t k + j is token t's j-th expert:
//     sort      places[p] = offsets[e] + number of earlier pairs of p's expert e;  -1 without a part (id outside [0,E), gate 0)
//     rows      rows[places[p]] = x[t]
//     sum       y[t] = residual[t] + sum_j gates[p] rows[places[p]]                    (without gates: the gradient of `rows`)
//     backward  d_rows[places[p]] = gates[p] dy[t],   d_gates[p] = dy[t] . rows[places[p]]
// Places alone lead both ways: a token's row is read once and goes to, or comes from, its k places, so no pass needs the
// inverse order.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "expert_rule.h"
#include "kernels.h"

namespace sida {

namespace {

constexpr int kMostE = 256;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;

struct SortArgs {
    const int32_t *ids;
    const float *gates;          // may be NULL
    int pairs, E, chunk;         // pairs of a workgroup: a multiple of 1024
    int32_t *offsets, *places;
    int32_t *hist;               // [chunks][E]
};

// The expert of pair p, -1 without a part.
__device__ __forceinline__ int expert_of(const SortArgs &a, int64_t p)
{
    const int id = a.ids[p];
    const float gate = a.gates ? a.gates[p] : 1.f;
    return (uint32_t)id < (uint32_t)a.E && gate != 0.f ? id : -1;
}

__global__ __launch_bounds__(kSortThreads) void expert_sort_count(const SortArgs a)
{
    __shared__ int hist[kMostE];
    const int tid = threadIdx.x;
    if (tid < kMostE) hist[tid] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * a.chunk, end = min(from + a.chunk, (int64_t)a.pairs);
    for (int64_t p = from + tid; p < end; p += kSortThreads) {
        const int e = expert_of(a, p);
        if (e >= 0) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    if (tid < a.E) a.hist[(size_t)blockIdx.x * a.E + tid] = hist[tid];
}

// Bound by the way to memory and back, a few times over, as there are 256 KiB of pairs for 32768 tokens: 3.0 us at best for 128 pairs in one launch, 3.8 and 4.6
// for 65536 in two.  No second pass over floating-point or atomic places: a pair's place follows from the pairs in front of it, so that bits repeat.
// A workgroup places the pairs of its chunk; each wavefront has a sixteenth of them, in order, 64 at a time.  A pair's place is the first
// one of its expert, the expert's pairs in earlier chunks and wavefronts, in earlier turns of this one, and in lower lanes, which nine
// ballots find.  ONE: there is one chunk, which counts for itself.
template <bool ONE>
__global__ __launch_bounds__(kSortThreads) void expert_sort_place(const SortArgs a)
{
    __shared__ int count[kSortWaves][kMostE];                // pairs of a wavefront, then the next place for them
    __shared__ int before[4][kMostE], all[4][kMostE];        // quarters of the chunks: those in front of this one, and all
    __shared__ int wave_total[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int e = tid & (kMostE - 1), quarter = tid / kMostE;
    for (int i = tid; i < kSortWaves * kMostE; i += kSortThreads) (&count[0][0])[i] = 0;
    __syncthreads();
    const int per = a.chunk / kSortWaves;
    const int64_t from = (int64_t)blockIdx.x * a.chunk + (int64_t)wave * per, end = min(from + per, (int64_t)a.pairs);
    for (int64_t p = from + lane; p < end; p += 64) {
        const int mine = expert_of(a, p);
        if (mine >= 0) atomicAdd(&count[wave][mine], 1);
    }
    int b = 0, n = 0;
    if (!ONE && e < a.E) {
        const int chunks = gridDim.x;
        for (int c0 = quarter; c0 < chunks; c0 += 32) {
            int v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = c0 + 4 * i < chunks ? a.hist[(size_t)(c0 + 4 * i) * a.E + e] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n += v[i];
                b += c0 + 4 * i < (int)blockIdx.x ? v[i] : 0;
            }
        }
    }
    before[quarter][e] = b;
    all[quarter][e] = n;
    __syncthreads();
    int total = 0, in_front = 0, mine[kSortWaves];
    if (tid < kMostE) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) mine[w] = count[w][tid];
        if (ONE) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) total += mine[w];
        } else {
            total = all[0][tid] + all[1][tid] + all[2][tid] + all[3][tid];
            in_front = before[0][tid] + before[1][tid] + before[2][tid] + before[3][tid];
        }
    }
    int upto = total;
    if (tid < kMostE) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(upto, d);
            upto += lane >= d ? v : 0;
        }
        if (lane == 63) wave_total[wave] = upto;
    }
    __syncthreads();
    if (tid < kMostE) {
        for (int w = 0; w < wave; ++w) upto += wave_total[w];
        int next = upto - total;
        if (blockIdx.x == 0) {
            if (tid < a.E) a.offsets[tid] = next;
            if (tid == a.E - 1) a.offsets[a.E] = upto;
        }
        next += in_front;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            count[w][tid] = next;
            next += mine[w];
        }
    }
    __syncthreads();
    for (int64_t p0 = from; p0 < end; p0 += 64) {
        const int64_t p = p0 + lane;
        const int mine = p < end ? expert_of(a, p) : -1;
        uint64_t same = __ballot(mine >= 0);
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const uint64_t set = __ballot(mine >> bit & 1);
            same &= mine >> bit & 1 ? set : ~set;
        }
        const int lower = __popcll(same & ((uint64_t)1 << lane) - 1);
        int place = -1;
        if (mine >= 0) place = count[wave][mine] + lower;
        __builtin_amdgcn_wave_barrier();
        if (mine >= 0 && lower == 0) count[wave][mine] = place + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (p < end) a.places[p] = place;
    }
}

// ---- rows ---------------------------------------------------------------------------------------
// Bound by bytes where there are many tokens, and by the way to memory and back where there are few: what a token's pairs read is asked for together,
// KM pairs and kDepth pieces of a row at a time.  32768 tokens of 1024 bf16 values, two experts each, at best: out 28 us (182 MB with a tenth without a part, 6.5 TB/s, as L2
// and the cache behind it keep some), sum 45 us (256 MB, 5.7 TB/s), back 55 us (303 MB, 5.5 TB/s); a copy of a large matrix reaches 5.2.
struct RowsArgs {
    const int32_t *places;
    const float *gates;          // may be NULL: ones
    const void *x;               // tokens: x, or dy
    const void *rows;            // expert rows that are read
    const void *residual;        // may be NULL
    void *to_rows, *y;
    float *d_gates;              // may be NULL
    int64_t ld_x, ld_rows, ld_res, ld_to_rows, ld_y;   // values between rows
    int T, M, k, d;              // expert rows there are, values of a row
    int lanes_log2;              // lanes of a token, or of a pair
};

constexpr int kRowsThreads = 256, kDepth = 2;

// A piece of a row: BYTES of values of type V, at any address of ALIGN bytes.
template <class V, int BYTES, int ALIGN>
struct Piece {
    static constexpr int kOf = BYTES / (int)sizeof(V);
    typedef __attribute__((ext_vector_type(kOf))) V Vec;
    typedef Vec __attribute__((aligned(ALIGN))) Any;
    static __device__ __forceinline__ Vec get(const V *p) { return *reinterpret_cast<const Any *>(p); }
    static __device__ __forceinline__ void put(V *p, Vec v)
    {
        if constexpr (ALIGN == 16) __builtin_nontemporal_store(v, reinterpret_cast<Vec *>(p));   // whole lines, past L2's replacement
        else *reinterpret_cast<Any *>(p) = v;
    }
    static __device__ __forceinline__ float at(const Vec &v, int i) { return (float)v[i]; }
    static __device__ __forceinline__ void set(Vec &v, int i, float f) { v[i] = (V)f; }
};
template <class V, int ALIGN>
struct Piece<V, (int)sizeof(V), ALIGN> {
    static constexpr int kOf = 1;
    typedef V Vec;
    static __device__ __forceinline__ V get(const V *p) { return *p; }
    static __device__ __forceinline__ void put(V *p, V v) { *p = v; }
    static __device__ __forceinline__ float at(V v, int) { return (float)v; }
    static __device__ __forceinline__ void set(V &v, int, float f) { v = (V)f; }
};

// Lanes of a token (or pair): `sub` of 2^lanes_log2, so that short rows share a wavefront.
struct Lanes {
    int64_t t;
    int sub, lanes;
};
__device__ __forceinline__ Lanes lanes_of(const RowsArgs &a)
{
    const int64_t at = (int64_t)blockIdx.x * kRowsThreads + threadIdx.x;
    return Lanes{at >> a.lanes_log2, (int)at & ((1 << a.lanes_log2) - 1), 1 << a.lanes_log2};
}
// A place; -1 also for one past the rows there are.
__device__ __forceinline__ int place_at(const RowsArgs &a, int64_t p)
{
    const int at = a.places[p];
    return (uint32_t)at < (uint32_t)a.M ? at : -1;
}
// The pieces of a row: of 16 bytes, and what is left of it in the smallest pieces that its alignment allows.
template <class V, int ALIGN, class Use>
__device__ __forceinline__ void each_piece(int d, Use &&use)
{
    constexpr int kOf = 16 / (int)sizeof(V);
    if constexpr (ALIGN >= 4) {
        use(Piece<V, 16, ALIGN>(), 0, d / kOf);
        if constexpr (ALIGN < 16) use(Piece<V, 4, 4>(), d / kOf * kOf, d % kOf / (4 / (int)sizeof(V)));
    } else {
        use(Piece<V, (int)sizeof(V), ALIGN>(), 0, d);
    }
}

template <class V, int ALIGN, int KM>
__global__ __launch_bounds__(kRowsThreads) void expert_rows_out(const RowsArgs a)
{
    const Lanes me = lanes_of(a);
    if (me.t >= a.T) return;
    const V *x = (const V *)a.x + me.t * a.ld_x;
    V *to[KM];
#pragma unroll
    for (int j = 0; j < KM; ++j) {
        const int at = j < a.k ? place_at(a, me.t * a.k + j) : -1;
        to[j] = at >= 0 ? (V *)a.to_rows + (int64_t)at * a.ld_to_rows : nullptr;
    }
    each_piece<V, ALIGN>(a.d, [&](auto piece, int from, int pieces) {
        typedef decltype(piece) P;
        for (int i0 = me.sub; i0 < pieces; i0 += me.lanes * kDepth) {
            typename P::Vec v[kDepth];
#pragma unroll
            for (int u = 0; u < kDepth; ++u) {
                const int i = i0 + u * me.lanes;
                v[u] = P::get(x + from + (i < pieces ? i : i0) * P::kOf);
            }
#pragma unroll
            for (int u = 0; u < kDepth; ++u)
                if (i0 + u * me.lanes < pieces)
#pragma unroll
                    for (int j = 0; j < KM; ++j)
                        if (to[j]) P::put(to[j] + from + (i0 + u * me.lanes) * P::kOf, v[u]);
        }
    });
}

template <class V, int ALIGN, int KM>
__global__ __launch_bounds__(kRowsThreads) void expert_rows_sum(const RowsArgs a)
{
    const Lanes me = lanes_of(a);
    if (me.t >= a.T) return;
    const V *from_row[KM];
    float gate[KM];
    bool part[KM];
#pragma unroll
    for (int j = 0; j < KM; ++j) {
        const int at = j < a.k ? place_at(a, me.t * a.k + j) : -1;
        part[j] = at >= 0;
        from_row[j] = (const V *)a.rows + (int64_t)max(at, 0) * a.ld_rows;
        gate[j] = a.gates && part[j] ? a.gates[me.t * a.k + j] : 1.f;
    }
    each_piece<V, ALIGN>(a.d, [&](auto piece, int from, int pieces) {
        typedef decltype(piece) P;
        for (int i = me.sub; i < pieces; i += me.lanes) {
            const int at = from + i * P::kOf;
            typename P::Vec v[KM], res{};
#pragma unroll
            for (int j = 0; j < KM; ++j)
                if (part[j]) v[j] = P::get(from_row[j] + at);
            if (a.residual) res = P::get((const V *)a.residual + me.t * a.ld_res + at);
            float sum[P::kOf] = {};
#pragma unroll
            for (int j = 0; j < KM; ++j)
                if (part[j])
#pragma unroll
                    for (int q = 0; q < P::kOf; ++q) sum[q] += gate[j] * P::at(v[j], q);
            typename P::Vec out;
#pragma unroll
            for (int q = 0; q < P::kOf; ++q) P::set(out, q, a.residual ? sum[q] + P::at(res, q) : sum[q]);
            P::put((V *)a.y + me.t * a.ld_y + at, out);
        }
    });
}

// A pair to a group of lanes: with a token to it its pairs would wait for one another (999 tokens of 601 fp32 values, three each: 14.0 us in place of 6.9, of
// which the pieces of 16 bytes at 4-byte boundaries are a part).
template <class V, int ALIGN>
__global__ __launch_bounds__(kRowsThreads) void expert_rows_back(const RowsArgs a)
{
    const Lanes me = lanes_of(a);
    if (me.t >= (int64_t)a.T * a.k) return;
    const int at = place_at(a, me.t);
    float dot = 0;
    if (at >= 0) {
        const float gate = a.gates ? a.gates[me.t] : 1.f;
        const V *dy = (const V *)a.x + me.t / a.k * a.ld_x, *row = (const V *)a.rows + (int64_t)at * a.ld_rows;
        V *to = (V *)a.to_rows + (int64_t)at * a.ld_to_rows;
        each_piece<V, ALIGN>(a.d, [&](auto piece, int from, int pieces) {
            typedef decltype(piece) P;
            for (int i0 = me.sub; i0 < pieces; i0 += me.lanes * kDepth) {
                typename P::Vec g[kDepth], r[kDepth];
#pragma unroll
                for (int u = 0; u < kDepth; ++u) {
                    const int i = i0 + u * me.lanes, value = from + (i < pieces ? i : i0) * P::kOf;
                    g[u] = P::get(dy + value);
                    if (a.d_gates) r[u] = P::get(row + value);
                }
#pragma unroll
                for (int u = 0; u < kDepth; ++u) {
                    const int i = i0 + u * me.lanes;
                    if (i >= pieces) break;
                    typename P::Vec out;
#pragma unroll
                    for (int q = 0; q < P::kOf; ++q) {
                        const float f = P::at(g[u], q);
                        if (a.d_gates) dot += f * P::at(r[u], q);
                        P::set(out, q, gate * f);
                    }
                    P::put(to + from + i * P::kOf, out);
                }
            }
        });
    }
    if (a.d_gates) {
        for (int d = 1; d < me.lanes; d *= 2) dot += __shfl_xor(dot, d);
        if (me.sub == 0) a.d_gates[me.t] = dot;
    }
}

enum class RowsWay { out, sum, back };
template <class V, int ALIGN>
int launch_way(RowsArgs &a, RowsWay way, hipStream_t st)
{
    const int64_t of = way == RowsWay::back ? (int64_t)a.T * a.k : a.T;
    a.lanes_log2 = rows_lanes_log2(ALIGN >= 4 ? a.d * (int)sizeof(V) / 16 : a.d, of);
    const uint32_t grid = (uint32_t)(((of << a.lanes_log2) + kRowsThreads - 1) / kRowsThreads);
    auto by_pairs = [&](auto one, auto two, auto four, auto eight) {
        if (a.k == 1) one<<<grid, kRowsThreads, 0, st>>>(a);
        else if (a.k == 2) two<<<grid, kRowsThreads, 0, st>>>(a);
        else if (a.k <= 4) four<<<grid, kRowsThreads, 0, st>>>(a);
        else eight<<<grid, kRowsThreads, 0, st>>>(a);
    };
    switch (way) {
    case RowsWay::out: by_pairs(expert_rows_out<V, ALIGN, 1>, expert_rows_out<V, ALIGN, 2>, expert_rows_out<V, ALIGN, 4>, expert_rows_out<V, ALIGN, 8>); break;
    case RowsWay::sum: by_pairs(expert_rows_sum<V, ALIGN, 1>, expert_rows_sum<V, ALIGN, 2>, expert_rows_sum<V, ALIGN, 4>, expert_rows_sum<V, ALIGN, 8>); break;
    case RowsWay::back: expert_rows_back<V, ALIGN><<<grid, kRowsThreads, 0, st>>>(a); break;
    }
    return (int)hipGetLastError();
}
// By the alignment of all rows' beginnings and ends: 16 bytes, 4, or single bf16 values.
int launch_rows(RowsArgs &a, RowsWay way, bool fp32, size_t ends, hipStream_t st)
{
    if (fp32) return ends % 16 == 0 ? launch_way<float, 16>(a, way, st) : launch_way<float, 4>(a, way, st);
    if (ends % 16 == 0) return launch_way<__bf16, 16>(a, way, st);
    return ends % 4 == 0 ? launch_way<__bf16, 4>(a, way, st) : launch_way<__bf16, 2>(a, way, st);
}
size_t ends_of(const void *p, int64_t ld, size_t size) { return (size_t)(uintptr_t)p | (size_t)ld * size; }

}  // namespace

int launch_expert_sort(const int32_t *ids, const float *gates, int64_t pairs, int32_t E, int32_t *offsets, int32_t *places, void *ws,
                       hipStream_t st)
{
    SortArgs a{};
    a.ids = ids, a.gates = gates, a.pairs = (int)pairs, a.E = E, a.offsets = offsets, a.places = places, a.hist = (int32_t *)ws;
    a.chunk = expert_sort_chunk(pairs);
    const int chunks = expert_sort_chunks(pairs);
    if (chunks == 1) {
        expert_sort_place<true><<<1, kSortThreads, 0, st>>>(a);
        return (int)hipGetLastError();
    }
    expert_sort_count<<<chunks, kSortThreads, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
    expert_sort_place<false><<<chunks, kSortThreads, 0, st>>>(a);
    return (int)hipGetLastError();
}

int launch_expert_rows(const ExpertRowsShape &s, const void *x, int64_t ld_x, const int32_t *places, void *rows, int64_t ld_rows, hipStream_t st)
{
    RowsArgs a{};
    a.places = places, a.x = x, a.to_rows = rows, a.ld_x = ld_x, a.ld_to_rows = ld_rows, a.T = s.T, a.M = s.M, a.k = s.k, a.d = s.d;
    const size_t size = s.fp32 ? 4 : 2;
    return launch_rows(a, RowsWay::out, s.fp32, ends_of(x, ld_x, size) | ends_of(rows, ld_rows, size) | s.d * size, st);
}

int launch_expert_sum(const ExpertRowsShape &s, const void *rows, int64_t ld_rows, const int32_t *places, const float *gates, const void *residual,
                      int64_t ld_res, void *y, int64_t ld_y, hipStream_t st)
{
    RowsArgs a{};
    a.places = places, a.gates = gates, a.rows = rows, a.residual = residual, a.y = y, a.ld_rows = ld_rows, a.ld_res = ld_res, a.ld_y = ld_y;
    a.T = s.T, a.M = s.M, a.k = s.k, a.d = s.d;
    const size_t size = s.fp32 ? 4 : 2;
    return launch_rows(a, RowsWay::sum, s.fp32,
                       ends_of(rows, ld_rows, size) | ends_of(y, ld_y, size) | (residual ? ends_of(residual, ld_res, size) : 0) | s.d * size, st);
}

int launch_expert_sum_backward(const ExpertRowsShape &s, const void *dy, int64_t ld_dy, const void *rows, int64_t ld_rows, const int32_t *places,
                               const float *gates, void *d_rows, int64_t ld_d, float *d_gates, hipStream_t st)
{
    RowsArgs a{};
    a.places = places, a.gates = gates, a.x = dy, a.rows = rows, a.to_rows = d_rows, a.d_gates = d_gates;
    a.ld_x = ld_dy, a.ld_rows = ld_rows, a.ld_to_rows = ld_d, a.T = s.T, a.M = s.M, a.k = s.k, a.d = s.d;
    const size_t size = s.fp32 ? 4 : 2;
    return launch_rows(a, RowsWay::back, s.fp32,
                       ends_of(dy, ld_dy, size) | ends_of(d_rows, ld_d, size) | (d_gates ? ends_of(rows, ld_rows, size) : 0) | s.d * size, st);
}

}  // namespace sida
