// Balance loss of a mixture of experts (see bagua_hip.h): statistics over all workers' tokens, loss, and gradient of the logits.
//
// A row of logits lies in L = 2^i lanes of a wave, VEC * NV elements in each, so that a wave holds 64 / L rows at a time; a row's
// maximum and sums are exchanges among those lanes.  The last lanes of a row that does not fill them read its last elements once
// more (in bounds, whatever the length): these are left out of the sums by a factor of 0, and where they are stored both lanes
// store the same bits.
#include <cmath>

#include "elements.hpp"

#pragma clang fp contract(off)

namespace bagua {

constexpr int kBalanceWaves = 16;            // of a workgroup of the forward pass
constexpr unsigned kBalanceGroups = kCus;    // most workgroups of the forward pass: the last one adds up their sums
constexpr int kGradWaves = 4;

struct Workers {
    const void* logits[BAGUA_MAX_WORKERS];
    const void* ids[BAGUA_MAX_WORKERS];      // of the backward pass: where the gradients go
    const uint8_t* mask[BAGUA_MAX_WORKERS];
    uint32_t tokens[BAGUA_MAX_WORKERS];
    uint32_t first_unit[BAGUA_MAX_WORKERS + 1];   // a unit: the rows that a wave holds at a time
    uint32_t k;
};

template <typename T, int N>
struct Raw;   // N elements as they are in memory, with the alignment of one
template <typename T>
struct Raw<T, 1> {
    typedef T v __attribute__((ext_vector_type(1), aligned(sizeof(T))));
};
template <typename T>
struct Raw<T, 8> {
    typedef T v __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

// op over the L lanes of a row, in every one of them.
template <int L, typename F>
__device__ __forceinline__ float lanes_reduce(float v, const F& op)
{
    if (L >= 2) v = op(v, dpp<kXor1>(v));
    if (L >= 4) v = op(v, dpp<kXor2>(v));
    if (L >= 8) v = op(v, dpp<kHalfMirror>(v));
    if (L >= 16) v = op(v, dpp<kMirror>(v));
    if (L >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if (L >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}

// What a lane holds of a row.
template <int TYPE, int VEC, int L, int NV>
struct Row {
    typedef typename Elem<TYPE>::one one;
    typedef typename Raw<one, VEC>::v raw;
    static constexpr int kRows = kWave / L;       // rows of a unit
    raw q[NV];

    // Elements of vector j of the lane: from at(j) on; slot(j): what it would be if the row filled the lanes.
    static __device__ __forceinline__ int slot(int j) { return (j * L + static_cast<int>(threadIdx.x % L)) * VEC; }
    static __device__ __forceinline__ int at(int j, int experts) { return min(slot(j), experts - VEC); }

    __device__ __forceinline__ void load(const one* row, int experts, bool there)
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            q[j] = raw(0);
            if (there) q[j] = __builtin_nontemporal_load(reinterpret_cast<const raw*>(row + at(j, experts)));
        }
    }
    // e = exp(x - max) of the lane's elements; the value: 1 / sum of the row's.
    __device__ __forceinline__ float exponentials(const float (&own)[NV][VEC], float (&e)[NV][VEC]) const
    {
        float most = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                e[j][i] = Elem<TYPE>::widen(q[j][i]);
                most = fmaxf(most, e[j][i]);
            }
        most = lanes_reduce<L>(most, OpMaxF());
        constexpr float kLog2e = 1.44269504088896340736f;
        if (TYPE != BAGUA_F16 && __any(fabsf(most) > 0x1p126f)) {
            // a largest one that leaves fp32 when it is multiplied: the type's lowest number (or -infinity) throughout a row
            const float top = most == -INFINITY ? 0.0f : most;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) e[j][i] = __builtin_amdgcn_exp2f((e[j][i] - top) * kLog2e);
        } else {
            const float shift = most == -INFINITY ? 0.0f : -most * kLog2e;    // its rounding is the same factor on all of a row
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) e[j][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(e[j][i], kLog2e, shift));
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum = __builtin_fmaf(e[j][i], own[j][i], sum);
        sum = lanes_reduce<L>(sum, OpAddF());
        const float r = __builtin_amdgcn_rcpf(sum);
        return sum == 0.0f ? 0.0f : __builtin_fmaf(__builtin_fmaf(-sum, r, 1.0f), r, r);
    }
    static __device__ __forceinline__ void owned(int experts, float (&own)[NV][VEC])
    {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) own[j][i] = j < NV / 2 || at(j, experts) + i >= slot(j) ? 1.0f : 0.0f;   // (rows are longer than half the lanes)
    }
};

// The token of a lane's row in unit `unit` (wave-uniform): of worker w, its index there, and whether it is one that counts.
struct Token {
    uint32_t w, t;
    bool exists, counts;
};
template <int ROWS, int L>
__device__ __forceinline__ Token token_of(const Workers& ws, uint32_t unit, uint32_t units)
{
    Token k{0, 0, unit < units, false};
    if (!k.exists) return k;
    while (ws.first_unit[k.w + 1] <= unit) ++k.w;     // first_unit[k] = units
    k.t = (unit - ws.first_unit[k.w]) * ROWS + (threadIdx.x & 63) / L;
    k.exists = k.t < ws.tokens[k.w];
    const uint8_t* mask = ws.mask[k.w];
    k.counts = k.exists && (!mask || mask[k.t] != 0);
    return k;
}

struct BalanceOut {
    int32_t* counts;
    float *prob, *loss, *weight;
    double alpha;
    int experts, top_k;
};

// Loss and weights from the sums, by one workgroup; thread i has experts i, i + THREADS, ...  `part`: one double per wave.
template <int THREADS, typename COUNT, typename PROB>
__device__ __forceinline__ void balance_loss(const BalanceOut& o, int32_t tokens, const COUNT& count, const PROB& prob, double* part)
{
    const double n = tokens;
    const double scale = tokens > 0 ? o.alpha * o.experts / (static_cast<double>(o.top_k) * n * n) : 0.0;
    double sum = 0.0;
    for (int e = threadIdx.x; e < o.experts; e += THREADS) {
        const double w = scale * count(e);
        o.weight[e] = static_cast<float>(w);
        if (tokens > 0) sum += w * prob(e);
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < THREADS / kWave; ++w) sum += part[w];
    o.loss[0] = static_cast<float>(sum);
}

// The forward pass.  Dynamic LDS: float sums[experts], then uint32 counters[(experts + 1) << lg]: 2^lg copies of each, one of which a
// lane adds to, so that popular experts are not waited for.  Workspace: counter (64 bytes), then every workgroup's sums and counts.
template <int TYPE, int VEC, int L, int NV, int UNROLL>
__global__ void __launch_bounds__(kWave * kBalanceWaves)
k_balance_stats(Workers ws, size_t ld, size_t ids_ld, int id_bytes, uint32_t units, uint32_t per_k, int lg, uint32_t* workspace, BalanceOut o)
{
    typedef Row<TYPE, VEC, L, NV> R;
    extern __shared__ float sums[];
    __shared__ double part[kBalanceWaves];
    __shared__ bool last;
    const int experts = o.experts, lane = threadIdx.x & 63, wave = wave_index();
    uint32_t* counters = reinterpret_cast<uint32_t*>(sums + experts);
    for (int i = threadIdx.x; i < (experts + 1) << lg; i += kWave * kBalanceWaves) counters[i] = 0;
    for (int i = threadIdx.x; i < experts; i += kWave * kBalanceWaves) sums[i] = 0.0f;
    __syncthreads();

    float own[NV][VEC], acc[NV][VEC];
    R::owned(experts, own);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[j][i] = 0.0f;
    const uint32_t waves = gridDim.x * kBalanceWaves;
    uint32_t tokens = 0;
    for (uint32_t unit = blockIdx.x * kBalanceWaves + wave; unit < units; unit += UNROLL * waves) {
        Token k[UNROLL];
        R row[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) k[u] = token_of<R::kRows, L>(ws, unit + u * waves, units);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            row[u].load(static_cast<const typename R::one*>(ws.logits[k[u].w]) + k[u].t * ld, experts, k[u].counts);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float e[NV][VEC];
            float inverse = row[u].exponentials(own, e);
            inverse = k[u].counts ? inverse : 0.0f;         // (rows that do not count were read as zeros)
            tokens += __popcll(__ballot(k[u].counts && lane % L == 0));
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[j][i] = __builtin_fmaf(e[j][i], inverse, acc[j][i]);
        }
    }

    // the choices: one per thread, worker after worker
    for (uint32_t w = 0; w < ws.k; ++w) {
        const uint32_t choices = ws.tokens[w] * static_cast<uint32_t>(o.top_k);
        for (uint32_t i = blockIdx.x * (kWave * kBalanceWaves) + threadIdx.x; i < choices; i += gridDim.x * (kWave * kBalanceWaves)) {
            uint32_t t = per_k ? __umulhi(i, per_k) : i;       // i / top_k, or one more (below 2^31)
            if (t * static_cast<uint32_t>(o.top_k) > i) --t;
            if (ws.mask[w] && ws.mask[w][t] == 0) continue;
            const size_t at = t * ids_ld + (i - t * static_cast<uint32_t>(o.top_k));
            const int64_t id = id_bytes == 8 ? static_cast<const int64_t*>(ws.ids[w])[at] : static_cast<const int32_t*>(ws.ids[w])[at];
            if (static_cast<uint64_t>(id) < static_cast<uint64_t>(experts))
                atomicAdd(counters + (static_cast<uint32_t>(id) << lg) + (lane & ((1 << lg) - 1)), 1u);
        }
    }
    if (lane == 0 && tokens) atomicAdd(counters + (experts << lg), tokens);

    // rows of one wave, then the waves one after another
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
#pragma unroll
            for (int s = L; s < kWave; s <<= 1) acc[j][i] += __shfl_xor(acc[j][i], s);
        }
    for (int w = 0; w < kBalanceWaves; ++w) {
        if (w == wave && lane < L) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (own[j][i] != 0.0f) sums[R::at(j, experts) + i] += acc[j][i];
        }
        __syncthreads();
    }
    float* prob = reinterpret_cast<float*>(workspace + 16);
    uint32_t* count = workspace + 16 + gridDim.x * experts;
    auto sum_of = [&](int e) {
        uint32_t c = 0;
        for (int r = 0; r < 1 << lg; ++r) c += counters[(e << lg) + r];
        return c;
    };
    for (int e = threadIdx.x; e <= experts; e += kWave * kBalanceWaves) {
        if (e < experts) __hip_atomic_store(prob + blockIdx.x * experts + e, sums[e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(count + blockIdx.x * (experts + 1) + e, sum_of(e), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0)
        last = __hip_atomic_fetch_add(workspace, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();

    // The groups' sums, by as many threads per expert as there are, in a fixed order.
    __shared__ double slice_sum[kWave * kBalanceWaves];
    __shared__ uint32_t slice_count[kWave * kBalanceWaves];
    int width = 1;                                          // threads of a slice, a power of two
    while (width < experts + 1 && width < kWave * kBalanceWaves) width *= 2;
    const int slices = kWave * kBalanceWaves / width, slice = threadIdx.x / width;
    for (int e0 = 0; e0 <= experts; e0 += width) {
        const int e = e0 + threadIdx.x % width;
        double s = 0.0;
        uint32_t c = 0;
        if (e <= experts) {
#pragma unroll 8
            for (uint32_t g = slice; g < gridDim.x; g += slices) {
                if (e < experts) s += __hip_atomic_load(prob + g * experts + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                c += __hip_atomic_load(count + g * (experts + 1) + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        slice_sum[threadIdx.x] = s;
        slice_count[threadIdx.x] = c;
        __syncthreads();
        if (slice == 0 && e <= experts) {
            for (int i = 1; i < slices; ++i) {
                s += slice_sum[i * width + threadIdx.x];
                c += slice_count[i * width + threadIdx.x];
            }
            o.counts[e] = static_cast<int32_t>(c);
            if (e < experts) {
                o.prob[e] = static_cast<float>(s);
                sums[e] = static_cast<float>(s);
            }
            counters[e] = c;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) __hip_atomic_store(workspace, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next call
    if (o.loss)
        balance_loss<kWave * kBalanceWaves>(o, static_cast<int32_t>(counters[experts]), [&](int e) { return static_cast<double>(counters[e]); },
                                            [&](int e) { return static_cast<double>(sums[e]); }, part);
}

__global__ void __launch_bounds__(256)
k_balance_loss(const int32_t* __restrict__ counts, const float* __restrict__ prob, BalanceOut o)
{
    __shared__ double part[4];
    balance_loss<256>(o, counts[o.experts], [&](int e) { return static_cast<double>(counts[e]); },
                      [&](int e) { return static_cast<double>(prob[e]); }, part);
}

// The backward pass: the probabilities are formed again from the logits, which are read anyway.
template <int TYPE, int VEC, int L, int NV, int UNROLL>
__global__ void __launch_bounds__(kWave * kGradWaves)
k_balance_grad(Workers ws, size_t ld, size_t ld_out, uint32_t units, int experts, const float* __restrict__ weight, const float* __restrict__ upstream)
{
    typedef Row<TYPE, VEC, L, NV> R;
    typedef typename R::one one;
    const uint32_t waves = gridDim.x * kGradWaves;
    const float up = upstream ? upstream[0] : 1.0f;
    float own[NV][VEC], g[NV][VEC];
    R::owned(experts, own);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[j][i] = weight[R::at(j, experts) + i];
    for (uint32_t unit = blockIdx.x * kGradWaves + wave_index(); unit < units; unit += UNROLL * waves) {
        Token k[UNROLL];
        R row[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) k[u] = token_of<R::kRows, L>(ws, unit + u * waves, units);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) row[u].load(static_cast<const one*>(ws.logits[k[u].w]) + k[u].t * ld, experts, k[u].counts);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float e[NV][VEC], dot = 0.0f;
            const float inverse = row[u].exponentials(own, e);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) dot = __builtin_fmaf(e[j][i], g[j][i] * own[j][i], dot);
            dot = lanes_reduce<L>(dot, OpAddF()) * inverse;
            const float scale = inverse * up;
            one* out = static_cast<one*>(const_cast<void*>(ws.ids[k[u].w])) + k[u].t * ld_out;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                typename R::raw q;
#pragma unroll
                for (int i = 0; i < VEC; ++i) q[i] = Elem<TYPE>::narrow(k[u].counts ? (e[j][i] * scale) * (g[j][i] - dot) : 0.0f);
                if (k[u].exists) __builtin_nontemporal_store(q, reinterpret_cast<typename R::raw*>(out + R::at(j, experts)));
            }
        }
    }
}

// Calls f with the layout of a row of `experts` elements: {VEC, L, NV, rows of a wave that are in flight together}.
template <int VEC_, int L_, int NV_, int UNROLL_>
struct Layout {
    static constexpr int VEC = VEC_, L = L_, NV = NV_, UNROLL = UNROLL_;
};
template <typename F>
inline void with_layout(int experts, const F& f)
{
    if (experts < 8) {
        if (experts <= 1) f(Layout<1, 1, 1, 4>());
        else if (experts <= 2) f(Layout<1, 2, 1, 4>());
        else if (experts <= 4) f(Layout<1, 4, 1, 4>());
        else f(Layout<1, 8, 1, 4>());
    } else if (experts <= 8) f(Layout<8, 1, 1, 4>());
    else if (experts <= 16) f(Layout<8, 2, 1, 4>());
    else if (experts <= 32) f(Layout<8, 4, 1, 4>());
    else if (experts <= 64) f(Layout<8, 8, 1, 4>());
    else if (experts <= 128) f(Layout<8, 16, 1, 4>());
    else if (experts <= 256) f(Layout<8, 32, 1, 4>());
    else if (experts <= 512) f(Layout<8, 64, 1, 4>());
    else if (experts <= 1024) f(Layout<8, 64, 2, 2>());
    else f(Layout<8, 64, 4, 1>());
}
template <typename F>
inline void with_type(int dtype, const F& f)
{
    if (dtype == BAGUA_F32) f(std::integral_constant<int, BAGUA_F32>());
    else if (dtype == BAGUA_BF16) f(std::integral_constant<int, BAGUA_BF16>());
    else f(std::integral_constant<int, BAGUA_F16>());
}

// Arguments that both passes have, and the workers' table.  rows: of a unit.
inline int balance_check(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts, Workers& ws)
{
    if (!logits || !tokens || !type_ok(dtype) || k < 1 || k > BAGUA_MAX_WORKERS || experts < 1 || ld < static_cast<size_t>(experts)) return BAGUA_ERR_INVALID_ARG;
    if (experts > BAGUA_MAX_EXPERTS || ld > static_cast<size_t>(1) << 40) return BAGUA_ERR_UNSUPPORTED;
    for (int w = 0; w < k; ++w) {
        if (tokens[w] && !logits[w]) return BAGUA_ERR_INVALID_ARG;
        if (tokens[w] > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    }
    ws = Workers{};
    ws.k = static_cast<uint32_t>(k);
    for (int w = 0; w < k; ++w) {
        ws.logits[w] = logits[w];
        ws.tokens[w] = static_cast<uint32_t>(tokens[w]);
    }
    return BAGUA_OK;
}
inline bool units_of(Workers& ws, int rows)
{
    uint64_t units = 0;
    for (uint32_t w = 0; w < ws.k; ++w) {
        ws.first_unit[w] = static_cast<uint32_t>(units);
        units += (ws.tokens[w] + static_cast<uint32_t>(rows) - 1) / static_cast<uint32_t>(rows);
        if (units > kMaxGrid) return false;
    }
    for (uint32_t w = ws.k; w <= BAGUA_MAX_WORKERS; ++w) ws.first_unit[w] = static_cast<uint32_t>(units);
    return true;
}
inline size_t matrix_bytes(size_t rows, size_t ld, size_t columns, size_t element) { return rows ? ((rows - 1) * ld + columns) * element : 0; }

}  // namespace bagua

using namespace bagua;

extern "C" size_t bagua_balance_workspace_bytes(int experts)
{
    if (experts < 1 || experts > BAGUA_MAX_EXPERTS) return 0;
    return (64 + kBalanceGroups * (2 * static_cast<size_t>(experts) + 1) * sizeof(uint32_t) + 15) & ~static_cast<size_t>(15);
}

extern "C" int bagua_balance_stats(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts,
                                   const void* const* ids, int id_bytes, size_t ids_ld, int top_k, const uint8_t* const* mask,
                                   int32_t* counts, float* prob, double alpha, float* loss, float* weight, void* workspace,
                                   size_t workspace_bytes, void* stream)
{
    Workers ws;
    const int bad = balance_check(dtype, logits, ld, tokens, k, experts, ws);
    if (bad) return bad;
    if (!ids || (id_bytes != 4 && id_bytes != 8) || top_k < 1 || top_k > experts || ids_ld < static_cast<size_t>(top_k) || !counts || !prob ||
        !workspace || !loss != !weight || !(std::fabs(alpha) < INFINITY))
        return BAGUA_ERR_INVALID_ARG;
    if (ids_ld > static_cast<size_t>(1) << 40) return BAGUA_ERR_UNSUPPORTED;
    if (workspace_bytes < bagua_balance_workspace_bytes(experts)) return BAGUA_ERR_INVALID_ARG;
    size_t choices = 0;
    RangeCheck rc;
    for (int w = 0; w < k; ++w) {
        if (tokens[w] == 0) continue;
        if (!ids[w] || (mask && !mask[w])) return BAGUA_ERR_INVALID_ARG;
        if (!aligned_to(logits[w], type_bytes(dtype)) || !aligned_to(ids[w], static_cast<size_t>(id_bytes))) return BAGUA_ERR_ALIGNMENT;
        choices += tokens[w] * static_cast<size_t>(top_k);
        rc.reads(logits[w], matrix_bytes(tokens[w], ld, static_cast<size_t>(experts), type_bytes(dtype)));
        rc.reads(ids[w], matrix_bytes(tokens[w], ids_ld, static_cast<size_t>(top_k), static_cast<size_t>(id_bytes)));
        if (mask) rc.reads(mask[w], tokens[w]);
        ws.ids[w] = ids[w];
        ws.mask[w] = mask ? mask[w] : nullptr;
    }
    if (choices > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    const size_t e = static_cast<size_t>(experts);
    rc.writes(counts, (e + 1) * sizeof(int32_t));
    rc.writes(prob, e * sizeof(float));
    rc.writes(loss, sizeof(float));
    rc.writes(weight, e * sizeof(float));
    rc.writes(workspace, bagua_balance_workspace_bytes(experts));
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned16(workspace) || !aligned4(counts) || !aligned4(prob) || !aligned4(loss) || !aligned4(weight)) return BAGUA_ERR_ALIGNMENT;
    const BalanceOut out{counts, prob, loss, weight, alpha, experts, top_k};
    const uint32_t per_k = top_k == 1 ? 0 : static_cast<uint32_t>((0x100000000ull + static_cast<uint64_t>(top_k) - 1) / static_cast<uint64_t>(top_k));
    int lg = 5;                                             // copies of a counter: what fits 16 KiB
    while (lg > 0 && ((e + 1) << lg) > 4096) --lg;
    const size_t lds = (e + ((e + 1) << lg)) * sizeof(float);
    int status = BAGUA_OK;
    with_layout(experts, [&](auto layout) {
        typedef decltype(layout) Lay;
        if (!units_of(ws, kWave / Lay::L)) {
            status = BAGUA_ERR_UNSUPPORTED;
            return;
        }
        const uint32_t units = ws.first_unit[BAGUA_MAX_WORKERS];
        const size_t work = std::max<size_t>((units + kBalanceWaves - 1) / kBalanceWaves, (choices + 8 * kWave * kBalanceWaves - 1) / (8 * kWave * kBalanceWaves));
        const dim3 grid(static_cast<unsigned>(std::min<size_t>(std::max<size_t>(work, 1), kBalanceGroups))), block(kWave * kBalanceWaves);
        with_type(dtype, [&](auto type) {
            launch_kernel(k_balance_stats<decltype(type)::value, Lay::VEC, Lay::L, Lay::NV, Lay::UNROLL>, grid, block, lds, static_cast<hipStream_t>(stream),
                          ws, ld, ids_ld, id_bytes, units, per_k, lg, static_cast<uint32_t*>(workspace), out);
        });
        status = launch_status();
    });
    return status;
}

extern "C" int bagua_balance_loss(const int32_t* counts, const float* prob, int experts, int top_k, double alpha, float* loss, float* weight, void* stream)
{
    if (!counts || !prob || !loss || !weight || experts < 1 || top_k < 1 || top_k > experts || !(std::fabs(alpha) < INFINITY)) return BAGUA_ERR_INVALID_ARG;
    if (experts > BAGUA_MAX_EXPERTS) return BAGUA_ERR_UNSUPPORTED;
    const size_t e = static_cast<size_t>(experts);
    RangeCheck rc;
    rc.reads(counts, (e + 1) * sizeof(int32_t));
    rc.reads(prob, e * sizeof(float));
    rc.writes(loss, sizeof(float));
    rc.writes(weight, e * sizeof(float));
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(counts) || !aligned4(prob) || !aligned4(loss) || !aligned4(weight)) return BAGUA_ERR_ALIGNMENT;
    const BalanceOut out{nullptr, nullptr, loss, weight, alpha, experts, top_k};
    launch_kernel(k_balance_loss, dim3(1), dim3(256), 0, static_cast<hipStream_t>(stream), counts, prob, out);
    return launch_status();
}

extern "C" int bagua_balance_grad(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts,
                                  const uint8_t* const* mask, const float* weight, const float* upstream, void* const* dlogits, size_t ld_out,
                                  void* stream)
{
    Workers ws;
    const int bad = balance_check(dtype, logits, ld, tokens, k, experts, ws);
    if (bad) return bad;
    if (!weight || !dlogits || ld_out < static_cast<size_t>(experts)) return BAGUA_ERR_INVALID_ARG;
    if (ld_out > static_cast<size_t>(1) << 40) return BAGUA_ERR_UNSUPPORTED;
    const size_t element = type_bytes(dtype), e = static_cast<size_t>(experts);
    RangeCheck rc;
    for (int w = 0; w < k; ++w) {
        if (tokens[w] == 0) continue;
        if (!dlogits[w] || (mask && !mask[w])) return BAGUA_ERR_INVALID_ARG;
        if (!aligned_to(logits[w], element) || !aligned_to(dlogits[w], element)) return BAGUA_ERR_ALIGNMENT;
        rc.reads(logits[w], matrix_bytes(tokens[w], ld, e, element));
        rc.writes(dlogits[w], matrix_bytes(tokens[w], ld_out, e, element));
        if (mask) rc.reads(mask[w], tokens[w]);
        ws.ids[w] = dlogits[w];
        ws.mask[w] = mask ? mask[w] : nullptr;
    }
    rc.reads(weight, e * sizeof(float));
    rc.reads(upstream, sizeof(float));
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(weight) || !aligned4(upstream)) return BAGUA_ERR_ALIGNMENT;
    int status = BAGUA_OK;
    with_layout(experts, [&](auto layout) {
        typedef decltype(layout) Lay;
        if (!units_of(ws, kWave / Lay::L)) {
            status = BAGUA_ERR_UNSUPPORTED;
            return;
        }
        const uint32_t units = ws.first_unit[BAGUA_MAX_WORKERS];
        if (units == 0) return;
        const dim3 grid(std::min<uint32_t>((units + kGradWaves - 1) / kGradWaves, kCus * 8)), block(kWave * kGradWaves);
        with_type(dtype, [&](auto type) {
            launch_kernel(k_balance_grad<decltype(type)::value, Lay::VEC, Lay::L, Lay::NV, Lay::UNROLL>, grid, block, 0, static_cast<hipStream_t>(stream), ws, ld,
                          ld_out, units, experts, weight, upstream);
        });
        status = launch_status();
    });
    return status;
}
