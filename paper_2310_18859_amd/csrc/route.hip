// The router: SoftMax of a token's expert logits, its top_k experts and their gates, tokens per expert and the balance loss
//     loss = E * sum_e f_e P_e,   f_e = counts[e] / (n k),   P_e = sum_t p[t,e] / n
// and the gradient of the logits.
//
// Sixteen lanes share a token, at most 16 logits each (E <= 256): a token's maximum and sums are four exchanges inside a row of
// 16 lanes (full-rate register moves), four tokens to a wavefront.  With a wavefront to a token the six exchanges, two of
// them through LDS, would cost more than the logits themselves.  All logits of a token are in registers at once, so every
// pass reads them once.  exp(v - m) is 2^((v - m) log2 e), the difference first: m log2 e on its own would overflow where all logits
// are the type's lowest value.
//
// Small batches are bound by the launch.  Large ones, forward: about 10 vector instructions for a logit and 6 more for each expert a token
// has, which are most of the time where a token has many (107351 tokens of 239 bf16 logits, 8 experts each: 54 us for 58 MB; 26.5 million
// instructions, 43 us if each SIMD issues one in four cycles at 2.4 GHz), and about half of it otherwise, the rest being loads and exchanges that
// are waited for with two rounds of tokens to a workgroup (32768 of 256 fp32 logits, 3 each: 13 us for 34 MB, 6.8 us of instructions;
// 40000 of 129 bf16 logits, 1 each: 10.5 and 5.8).  The sums of the workgroups are another 4.2 to 4.7 us.  Backward, about 14 for a logit, by
// bytes: 262144 of 128 fp32 logits, 270 MB in 47 us, 5.7 TB/s.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "kernels.h"

namespace sida {

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int kLanes = 16;                     // lanes per token
constexpr int kRouteThreads = 1024, kRouteRows = kRouteThreads / kLanes;
constexpr int kRouteWaves = kRouteThreads / 64;
constexpr int kMostE = 256;
constexpr int kRouteBlocks = 256;              // workgroups whose sums the second launch adds: one per compute unit
constexpr float kLog2e = 1.44269504088896340736f;

// Value of the lane N places on in the row of 16 lanes, around its end.
template <int N>
__device__ __forceinline__ float turned(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, true));
}
template <int N>
__device__ __forceinline__ int turned(int v)
{
    return __builtin_amdgcn_mov_dpp(v, 0x120 + N, 0xf, 0xf, true);
}
// Each lane of the row gets the same bits: at every step the two sides add the same two numbers.
__device__ __forceinline__ float row_sum(float v)
{
    v += turned<8>(v);
    v += turned<4>(v);
    v += turned<2>(v);
    return v + turned<1>(v);
}
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, turned<8>(v));
    v = fmaxf(v, turned<4>(v));
    v = fmaxf(v, turned<2>(v));
    return fmaxf(v, turned<1>(v));
}
__device__ __forceinline__ int row_min(int v)
{
    v = min(v, turned<8>(v));
    v = min(v, turned<4>(v));
    v = min(v, turned<2>(v));
    return min(v, turned<1>(v));
}
__device__ __forceinline__ int row_sum(int v)
{
    v += turned<8>(v);
    v += turned<4>(v);
    v += turned<2>(v);
    return v + turned<1>(v);
}

// A lane's logits: J loads of VEC values; load j of lane `sub` starts at column (j * 16 + sub) * VEC.  Places past E hold -infinity.
template <class T, int VEC, int J>
struct Row {
    static constexpr int V = VEC * J;
    typedef __attribute__((ext_vector_type(VEC))) T Vec;
    float v[V];
    static __device__ __forceinline__ int column(int sub, int i) { return ((i / VEC) * kLanes + sub) * VEC + i % VEC; }
    // As they lie in memory, without a branch or a conversion that would wait for them (one load for each value, as where E is odd, would be
    // waited for one by one: 40000 tokens of 129 bf16 logits, 14.7 us against 17.8); lanes past E read the first columns.
    struct Raw {
        Vec x[J];
        __device__ __forceinline__ void load(const T *row, int sub, int E)
        {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int c = (j * kLanes + sub) * VEC;
                x[j] = *reinterpret_cast<const Vec *>(row + (c < E ? c : 0));   // E is a multiple of VEC
            }
        }
    };
    __device__ __forceinline__ void take(const Raw &raw, int sub, int E)
    {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[j * VEC + i] = (j * kLanes + sub) * VEC < E ? (float)raw.x[j][i] : -INFINITY;
    }
    __device__ __forceinline__ void store(T *row, int sub, int E) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = (j * kLanes + sub) * VEC;
            if (c < E) {
                if constexpr (VEC == 1) {
                    row[c] = (T)v[j];
                } else {
                    Vec x;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) x[i] = (T)v[j * VEC + i];
                    __builtin_nontemporal_store(x, reinterpret_cast<Vec *>(row + c));
                }
            }
        }
    }
    // The largest logit that is a number, in every lane of the token; -infinity where there is none.
    __device__ __forceinline__ float largest() const
    {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) m = fmaxf(m, v[i]);
        return row_max(m);
    }
    // Whether all logits are -infinity, given the largest.
    __device__ __forceinline__ bool nothing(float m) const
    {
        if (m != -INFINITY) return false;
        int nan = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) nan |= v[i] != v[i];
        return row_sum(nan) == 0;
    }
};

__device__ __forceinline__ float power(float v, float m) { return __builtin_amdgcn_exp2f((v - m) * kLog2e); }

// What the second launch's workgroups leave for the last of them; the first launch sets `arrived` to 0.
struct RouteTail {
    float term[8];
    int count[8];
    int arrived;
};
static_assert(sizeof(RouteTail) <= kRouteTailBytes, "workspace");

struct RouteArgs {
    const void *logits;
    const uint8_t *mask;
    int64_t ld, ld_d;
    int T, E, k, normalize;
    int32_t *ids;
    float *gates;
    int32_t *counts;
    float *loss;
    float *part_p;               // [workgroups][part_ld], part_ld = E filled up to 16 bytes
    int32_t *part_n;             // the same
    int part_ld;
    RouteTail *tail;
    const float *d_gates, *d_loss;
    void *d_logits;
};

// The loss from sum_e counts[e] sum_t p[t,e] and the sum of the counts, n k.
__device__ __forceinline__ float loss_of(const RouteArgs &a, float term, int total)
{
    const float all = (float)total, tokens = all / a.k;
    return total ? (float)a.E * (term / all / tokens) : 0.f;
}

template <class T, int VEC, int J>
__global__ __launch_bounds__(kRouteThreads) void route_rows(const RouteArgs a)
{
    typedef Row<T, VEC, J> R;
    __shared__ float p_part[kRouteWaves][kMostE];
    __shared__ int n_part[kMostE];
    __shared__ float sums[8];
    const int tid = threadIdx.x, sub = tid & (kLanes - 1), lane = tid & 63, wave = tid >> 6;
    for (int e = tid; e < kMostE; e += kRouteThreads) n_part[e] = 0;
    __syncthreads();
    float p_acc[R::V];
#pragma unroll
    for (int i = 0; i < R::V; ++i) p_acc[i] = 0;
    const int64_t step = (int64_t)gridDim.x * kRouteRows;
    typename R::Raw next;
    uint8_t next_in;
    auto ask = [&](int64_t t) {
        const T *row = (const T *)a.logits + t * a.ld;
        next.load(row, sub, a.E);
        next_in = *(a.mask ? a.mask + t : (const uint8_t *)row);   // no branch here either: a load behind one is waited for at once
    };
    int64_t t = (int64_t)blockIdx.x * kRouteRows + tid / kLanes;
    if (t < a.T) ask(t);
    for (; t < a.T; t += step) {
        R r;
        r.take(next, sub, a.E);
        const bool in = !a.mask || next_in;
        if (t + step < a.T) ask(t + step);                   // while this token is dealt with
        const float m = r.largest();
        const bool part = in && !r.nothing(m);
        float e[R::V], sum = 0;
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            e[i] = power(r.v[i], m);
            sum += e[i];
        }
        const float inv = 1.f / row_sum(sum);
        if (part) {
#pragma unroll
            for (int i = 0; i < R::V; ++i) p_acc[i] += e[i] * inv;
        }
        // The experts, one after the other: the largest logit left, the lowest column that has it.  A chosen logit becomes
        // NaN, which no maximum takes.
        int my_id = 0;
        float my_gate = 0, gate_sum = 0, top = m;
        for (int j = 0; j < a.k; ++j) {
            if (j) top = r.largest();
            int id = INT32_MAX;
#pragma unroll
            for (int i = R::V - 1; i >= 0; --i) id = r.v[i] == top ? R::column(sub, i) : id;
            id = row_min(id);
            if (id >= a.E) {                                 // only NaN are left: the lowest column not chosen yet
                uint32_t taken = 0;                          // bit i: place i is chosen
                for (int q = 0; q < j; ++q) {
                    const int before = __shfl(my_id, (lane & ~(kLanes - 1)) + q);
#pragma unroll
                    for (int i = 0; i < R::V; ++i) taken |= R::column(sub, i) == before ? 1u << i : 0u;
                }
                id = INT32_MAX;
#pragma unroll
                for (int i = R::V - 1; i >= 0; --i)
                    if (!(taken >> i & 1) && R::column(sub, i) < a.E) id = R::column(sub, i);
                id = row_min(id);
            }
            const float gate = power(top, m) * inv;
            gate_sum += gate;
            if (sub == j) {
                my_id = id;
                my_gate = gate;
            }
            if (j + 1 < a.k) {
#pragma unroll
                for (int i = 0; i < R::V; ++i) r.v[i] = R::column(sub, i) == id ? NAN : r.v[i];
            }
        }
        if (sub < a.k) {
            if (a.normalize) my_gate /= gate_sum;
            a.ids[t * a.k + sub] = my_id;
            a.gates[t * a.k + sub] = part ? my_gate : 0.f;
            if (part) atomicAdd(&n_part[my_id], 1);
        }
    }
    // The four tokens of a wavefront, then the wavefronts, in a fixed order.
#pragma unroll
    for (int i = 0; i < R::V; ++i) {
        p_acc[i] += __shfl_xor(p_acc[i], 16);
        p_acc[i] += __shfl_xor(p_acc[i], 32);
        if (lane < kLanes) p_part[wave][R::column(sub, i)] = p_acc[i];
    }
    __syncthreads();
    float p = 0;
    int n = 0;
    if (tid < a.E) {
#pragma unroll
        for (int w = 0; w < kRouteWaves; ++w) p += p_part[w][tid];
        n = n_part[tid];
    }
    if (gridDim.x > 1) {
        if (tid < a.E) {
            a.part_p[(size_t)blockIdx.x * a.part_ld + tid] = p;
            a.part_n[(size_t)blockIdx.x * a.part_ld + tid] = n;
        }
        if (blockIdx.x == 0 && tid == 0) a.tail->arrived = 0;
        return;
    }
    float term = p * (float)n;
    int total = n;
    if (tid < kMostE) {
        if (tid < a.E) a.counts[tid] = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            term += __shfl_xor(term, d);
            total += __shfl_xor(total, d);
        }
        if (lane == 0) {
            sums[wave] = term;
            sums[4 + wave] = __builtin_bit_cast(float, total);
        }
    }
    __syncthreads();
    if (tid == 0) {
        total = 0;
        for (int w = 0; w < 4; ++w) total += __builtin_bit_cast(int, sums[4 + w]);
        *a.loss = loss_of(a, sums[0] + sums[1] + (sums[2] + sums[3]), total);
    }
}

// Adds the workgroups' sums.  A workgroup takes 32 experts, 8 threads with 16-byte loads to a row of sums: they were written through other
// XCDs' caches, and one compute unit alone would wait 9.4 us for the 512 KiB of 256 experts (4.7 us this way).  The
// workgroup that is the last to arrive, whichever it is, adds the eight terms of the loss in their order.
constexpr int kFinishE = 32, kFinishThreads = 512, kFinishSlices = kFinishThreads / (kFinishE / 4), kFinishLoads = kRouteBlocks / kFinishSlices;
__global__ __launch_bounds__(kFinishThreads) void route_finish(const RouteArgs a, int workgroups)
{
    __shared__ f32x4 p_part[kFinishSlices][kFinishE / 4];
    __shared__ i32x4 n_part[kFinishSlices][kFinishE / 4];
    __shared__ float p_sum[kFinishThreads / kFinishE][kFinishE];
    __shared__ int n_sum[kFinishThreads / kFinishE][kFinishE];
    const int tid = threadIdx.x, c4 = tid % (kFinishE / 4), slice = tid / (kFinishE / 4), from = blockIdx.x * kFinishE + c4 * 4;
    f32x4 p[kFinishLoads];
    i32x4 n[kFinishLoads];
#pragma unroll
    for (int i = 0; i < kFinishLoads; ++i) {
        const int b = i * kFinishSlices + slice;
        const bool in = b < workgroups && from < a.part_ld;
        p[i] = in ? *reinterpret_cast<const f32x4 *>(a.part_p + (size_t)b * a.part_ld + from) : f32x4{0, 0, 0, 0};
        n[i] = in ? *reinterpret_cast<const i32x4 *>(a.part_n + (size_t)b * a.part_ld + from) : i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 1; i < kFinishLoads; ++i) {
        p[0] += p[i];
        n[0] += n[i];
    }
    p_part[slice][c4] = p[0];
    n_part[slice][c4] = n[0];
    __syncthreads();
    constexpr int kParts = kFinishThreads / kFinishE, kPer = kFinishSlices / kParts;
    const int mine = tid % kFinishE, part = tid / kFinishE;
    float sum = 0;
    int count = 0;
#pragma unroll
    for (int s = 0; s < kPer; ++s) {
        sum += p_part[part * kPer + s][mine / 4][mine % 4];
        count += n_part[part * kPer + s][mine / 4][mine % 4];
    }
    p_sum[part][mine] = sum;
    n_sum[part][mine] = count;
    __syncthreads();
    if (tid >= 64) return;
    sum = 0;
    count = 0;
    const int e = blockIdx.x * kFinishE + tid;
    if (tid < kFinishE && e < a.E) {
#pragma unroll
        for (int s = 0; s < kParts; ++s) {
            sum += p_sum[s][tid];
            count += n_sum[s][tid];
        }
        a.counts[e] = count;
    }
    float term = sum * (float)count;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        term += __shfl_xor(term, d);
        count += __shfl_xor(count, d);
    }
    if (tid) return;
    RouteTail *t = a.tail;
    __hip_atomic_store(&t->term[blockIdx.x], term, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&t->count[blockIdx.x], count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__hip_atomic_fetch_add(&t->arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 != (int)gridDim.x) return;
    term = 0;
    count = 0;
    for (int i = 0; i < (int)gridDim.x; ++i) {
        term += __hip_atomic_load(&t->term[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        count += __hip_atomic_load(&t->count[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    *a.loss = loss_of(a, term, count);
}

constexpr int kBackThreads = 256, kBackRows = kBackThreads / kLanes;
template <class T, int VEC, int J>
__global__ __launch_bounds__(kBackThreads) void route_back_rows(const RouteArgs a)
{
    typedef Row<T, VEC, J> R;
    const int tid = threadIdx.x, sub = tid & (kLanes - 1), lane = tid & 63;
    // What is read of a token: its logits, and in lane j its j-th expert and the gradient of its gate (36000 tokens of 128 bf16 logits, 8
    // experts each, 12.9 us; every lane loading every one of them, one behind the other, 19.7).
    typename R::Raw next;
    uint8_t next_in;
    int next_id = -1;
    float next_dg = 0;
    auto ask = [&](int64_t t) {
        const T *row = (const T *)a.logits + t * a.ld;
        next.load(row, sub, a.E);
        next_in = *(a.mask ? a.mask + t : (const uint8_t *)row);
        if (a.d_gates && sub < a.k) {
            next_id = a.ids[t * a.k + sub];
            next_dg = a.d_gates[t * a.k + sub];
        }
    };
    const int64_t step = (int64_t)gridDim.x * kBackRows;
    int64_t t = (int64_t)blockIdx.x * kBackRows + tid / kLanes;
    if (t < a.T) ask(t);
    // What the loss adds to an expert's column: d_loss E/n counts/(n k), n k being the sum of all counts.
    float pull[R::V];
    int all = 0;
#pragma unroll
    for (int i = 0; i < R::V; ++i) {
        const int c = R::column(sub, i), at = a.counts[c < a.E ? c : 0], n = c < a.E ? at : 0;
        all += n;
        pull[i] = (float)n;
    }
    all = row_sum(all);
    const float nk = (float)all, coef = a.d_loss && all ? *a.d_loss * (float)a.E * (float)a.k / nk / nk : 0.f;
#pragma unroll
    for (int i = 0; i < R::V; ++i) pull[i] *= coef;
    for (; t < a.T; t += step) {
        R r;
        r.take(next, sub, a.E);
        const bool in = !a.mask || next_in;
        const int my_id = (uint32_t)next_id < (uint32_t)a.E ? next_id : -1;   // a place past E is no expert's
        const float my_dg = next_dg;
        const T my_logit = ((const T *)a.logits + t * a.ld)[my_id >= 0 ? my_id : 0];
        if (t + step < a.T) ask(t + step);                   // while this token is dealt with
        const float m = r.largest();
        const bool part = in && !r.nothing(m);
        float p[R::V], sum = 0;
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            p[i] = power(r.v[i], m);
            sum += p[i];
        }
        const float inv = 1.f / row_sum(sum);
        float d[R::V];
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            p[i] *= inv;
            d[i] = pull[i];
        }
        if (a.d_gates) {
            float my_g = my_dg;
            if (a.normalize) {                               // dg_i - sum_j dg_j gate_j, over the sum of the chosen p
                const float q = my_id >= 0 ? power((float)my_logit, m) * inv : 0.f;
                const float scale = 1.f / row_sum(q);
                my_g = (my_dg - row_sum(my_id >= 0 ? my_dg * q : 0.f) * scale) * scale;
            }
            for (int j = 0; j < a.k; ++j) {
                const int from = (lane & ~(kLanes - 1)) + j, id = __shfl(my_id, from);
                const float g = __shfl(my_g, from);
#pragma unroll
                for (int i = 0; i < R::V; ++i) d[i] += R::column(sub, i) == id ? g : 0.f;
            }
        }
        float dot = 0;
#pragma unroll
        for (int i = 0; i < R::V; ++i) dot += p[i] * d[i];
        dot = row_sum(dot);
#pragma unroll
        for (int i = 0; i < R::V; ++i) r.v[i] = part ? p[i] * (d[i] - dot) : 0.f;
        r.store((T *)a.d_logits + t * a.ld_d, sub, a.E);
    }
}

template <class T, int VEC, int J>
int launch_forward(const RouteArgs &a, hipStream_t st)
{
    const int grid = route_workgroups(a.T);
    route_rows<T, VEC, J><<<grid, kRouteThreads, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && grid > 1) {
        route_finish<<<(a.E + kFinishE - 1) / kFinishE, kFinishThreads, 0, st>>>(a, grid);
        e = hipGetLastError();
    }
    return (int)e;
}
template <class T, int VEC, int J>
int launch_back(const RouteArgs &a, hipStream_t st)
{
    const int64_t need = ((int64_t)a.T + kBackRows - 1) / kBackRows;
    route_back_rows<T, VEC, J><<<(int)(need < 8192 ? need : 8192), kBackThreads, 0, st>>>(a);
    return (int)hipGetLastError();
}

// Picks the loads per lane.  16-byte loads where every row starts on a 16-byte boundary and E is a multiple of a load's values.
template <class T, class Use>
int by_width(const RouteArgs &a, bool wide, Use &&use)
{
    constexpr int VEC = 16 / sizeof(T);
    if (wide) {
        const int j = (a.E + kLanes * VEC - 1) / (kLanes * VEC);
        if (j <= 1) return use(std::integral_constant<int, VEC>(), std::integral_constant<int, 1>());
        if (j <= 2) return use(std::integral_constant<int, VEC>(), std::integral_constant<int, 2>());
        if constexpr (VEC == 4) return use(std::integral_constant<int, VEC>(), std::integral_constant<int, 4>());
    }
    const int j = (a.E + kLanes - 1) / kLanes;
    if (j <= 2) return use(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
    if (j <= 4) return use(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
    if (j <= 8) return use(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
    return use(std::integral_constant<int, 1>(), std::integral_constant<int, 16>());
}
template <class T>
bool rows_wide(const void *p, int64_t ld, int E)
{
    return (((uintptr_t)p | (uintptr_t)ld * sizeof(T)) % 16) == 0 && E % (16 / sizeof(T)) == 0;
}
template <class T>
int forward_typed(const RouteArgs &a, hipStream_t st)
{
    return by_width<T>(a, rows_wide<T>(a.logits, a.ld, a.E),
                       [&](auto vec, auto j) { return launch_forward<T, decltype(vec)::value, decltype(j)::value>(a, st); });
}
template <class T>
int back_typed(const RouteArgs &a, hipStream_t st)
{
    return by_width<T>(a, rows_wide<T>(a.logits, a.ld, a.E) && rows_wide<T>(a.d_logits, a.ld_d, a.E),
                       [&](auto vec, auto j) { return launch_back<T, decltype(vec)::value, decltype(j)::value>(a, st); });
}

}  // namespace

// Up to kRouteOne tokens one workgroup does everything: the second launch costs more than its rounds of 64 tokens.
constexpr int kRouteOne = 256;
int route_workgroups(int32_t T)
{
    if (T <= kRouteOne) return 1;
    const int need = (int)(((int64_t)T + kRouteRows - 1) / kRouteRows);
    return need < kRouteBlocks ? need : kRouteBlocks;
}

int launch_route(const RouteShape &s, const void *logits, int64_t ld, int32_t T, const uint8_t *mask, int32_t *ids, float *gates,
                 int32_t *counts, float *loss, void *ws, hipStream_t st)
{
    RouteArgs a{};
    a.logits = logits, a.ld = ld, a.T = T, a.E = s.E, a.k = s.top_k, a.normalize = s.normalize, a.mask = mask;
    a.ids = ids, a.gates = gates, a.counts = counts, a.loss = loss;
    a.tail = (RouteTail *)ws;
    a.part_p = (float *)((char *)ws + kRouteTailBytes);
    a.part_ld = (s.E + 3) / 4 * 4;
    a.part_n = (int32_t *)(a.part_p + (size_t)route_workgroups(T) * a.part_ld);
    return s.fp32 ? forward_typed<float>(a, st) : forward_typed<__bf16>(a, st);
}

int launch_route_backward(const RouteShape &s, const void *logits, int64_t ld, int32_t T, const uint8_t *mask, const int32_t *ids,
                          const int32_t *counts, const float *d_gates, const float *d_loss, void *d_logits, int64_t ld_d,
                          hipStream_t st)
{
    RouteArgs a{};
    a.logits = logits, a.ld = ld, a.T = T, a.E = s.E, a.k = s.top_k, a.normalize = s.normalize, a.mask = mask;
    a.ids = const_cast<int32_t *>(ids), a.counts = const_cast<int32_t *>(counts);
    a.d_gates = d_gates, a.d_loss = d_loss, a.d_logits = d_logits, a.ld_d = ld_d;
    return s.fp32 ? back_typed<float>(a, st) : back_typed<__bf16>(a, st);
}

}  // namespace sida
