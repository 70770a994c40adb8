// Many tensors in one launch: the global gradient norm with its clipping factor, and the AdamW step (see bagua_hip.h).
//
// A plan cuts every tensor into tiles of kTile elements, counted from the tensor's first one, and gives for every tile the
// tensor that it belongs to; a wave takes one row of 256 elements of a tile, one access of four elements per lane and array.
// Tensors need the alignment of their elements only: the accesses are declared so, and the hardware takes them at any address.
#include <cmath>
#include <new>
#include <vector>

#include "batch.hpp"
#include "elements.hpp"

#pragma clang fp contract(off)

namespace bagua {

constexpr int kTensorTile = 1024;
constexpr int kTileRows = kTensorTile / kRow;
constexpr unsigned kNormGroups = 2048;    // most workgroups of the norm: eight waves of four on every SIMD
constexpr unsigned kNormWaves = 4;

struct TensorEntry {
    uint64_t grad, param, m, v, m_scale, v_scale, copy, numel;
    uint32_t first_tile, index;
    float decay;
    uint32_t unused;
};
static_assert(sizeof(TensorEntry) == 80, "the table is a whole number of 16-byte words");

// The plan's workspace: [counter, padding | partial sums of the norm | entries | tensor of every tile].
constexpr size_t kPartialsAt = 64, kEntriesAt = kPartialsAt + kNormGroups * sizeof(double);
struct TensorPlanView {
    uint32_t* counter;
    double* partial;
    const TensorEntry* entry;
    const uint32_t* tile_tensor;
};
inline TensorPlanView tensor_plan_view(const bagua_tensor_plan_t* p)
{
    unsigned char* w = static_cast<unsigned char*>(p->workspace);
    return TensorPlanView{reinterpret_cast<uint32_t*>(w), reinterpret_cast<double*>(w + kPartialsAt),
                          reinterpret_cast<const TensorEntry*>(w + kEntriesAt),
                          reinterpret_cast<const uint32_t*>(w + kEntriesAt + static_cast<size_t>(p->tensors) * sizeof(TensorEntry))};
}

// ---------------------------------------------------------------- four elements of a row
// `remain`: valid elements from the row's start on (wave-uniform).  Absent ones read as 0.
template <int TYPE>
__device__ __forceinline__ f4 load_four(const typename Elem<TYPE>::one* row, int lane, int remain)
{
    typedef Elem<TYPE> E;
    const int e = lane * 4;
    if (remain >= kRow) return E::load(row + e);
    f4 r = f4{0.f, 0.f, 0.f, 0.f};
    if (e + 0 < remain) r.x = E::widen(row[e + 0]);
    if (e + 1 < remain) r.y = E::widen(row[e + 1]);
    if (e + 2 < remain) r.z = E::widen(row[e + 2]);
    if (e + 3 < remain) r.w = E::widen(row[e + 3]);
    return r;
}
template <int TYPE>
__device__ __forceinline__ void store_four(typename Elem<TYPE>::one* row, int lane, int remain, f4 v)
{
    typedef Elem<TYPE> E;
    const int e = lane * 4;
    if (remain >= kRow) {
        E::store(row + e, v);
    } else {
        if (e + 0 < remain) row[e + 0] = E::narrow(v.x);
        if (e + 1 < remain) row[e + 1] = E::narrow(v.y);
        if (e + 2 < remain) row[e + 2] = E::narrow(v.z);
        if (e + 3 < remain) row[e + 3] = E::narrow(v.w);
    }
}
__device__ __forceinline__ uint32_t load_four_codes(const uint8_t* row, int lane, int remain)
{
    if (remain >= kRow) return __builtin_nontemporal_load(reinterpret_cast<const u32u*>(row + lane * 4));
    return load_codes_row(row, lane, remain);
}
__device__ __forceinline__ void store_four_codes(uint8_t* row, int lane, int remain, uint32_t w)
{
    if (remain >= kRow) __builtin_nontemporal_store(static_cast<u32u>(w), reinterpret_cast<u32u*>(row + lane * 4));
    else store_codes_row(row, lane, remain, w, 0);
}

// ---------------------------------------------------------------- E4M3 codes with a scale
typedef float f2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ f4 widen_codes(uint32_t w, float scale)
{
    const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    return f4{lo.x * scale, lo.y * scale, hi.x * scale, hi.y * scale};
}
// Scale of a block whose largest magnitude is `most`, and its reciprocal; a block that is (nearly) zero has neither.
struct Scale {
    float scale, inverse;
};
__device__ __forceinline__ Scale scale_of(float most)
{
    const float s = most * static_cast<float>(1.0 / 448.0);
    return s >= 0x1p-126f ? Scale{s, 1.0f / s} : Scale{0.0f, 0.0f};
}
__device__ __forceinline__ uint32_t nearest_codes(f4 y)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y.x, y.y, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y.z, y.w, w, true));
}
// y >= 0 times 2^-120 has E4M3's exponent field in the low bits of fp32's own (and its subnormals where fp32 has them), so
// the bits above the 20 lowest are the code, and what lies below them is how far y is on the way to the next one.
__device__ __forceinline__ uint32_t random_code(float y, float r, uint32_t random)
{
    uint32_t c = (__float_as_uint(y * 0x1p-120f) + (random >> 12)) >> 20;
    c = c < 1 ? 1 : c > 126 ? 126 : c;
    c = r == r ? c : 127;                 // what is no number stays none
    return r == 0.0f ? 0 : c;
}

__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}
constexpr uint32_t kGolden = 0x9E3779B9u;
__device__ __forceinline__ uint32_t turned(uint32_t h, int by) { return by == 0 ? h : __builtin_amdgcn_alignbit(h, h, 32 - by); }
__device__ __forceinline__ uint16_t random_bf16(float x, uint32_t random)
{
    return static_cast<uint16_t>((__float_as_uint(x) + (random >> 16)) >> 16);
}

// ---------------------------------------------------------------- AdamW
struct AdamArgs {
    const float* clip;
    float beta1, omb1, beta2, omb2, root, eps, rate, decay;   // root: 1/sqrt(1-beta2^t), rate: lr/(1-beta1^t), decay: lr*weight_decay
    uint32_t seed, rows;
};

__device__ __forceinline__ float max4(f4 x) { return fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)); }
__device__ __forceinline__ f4 abs4(f4 x) { return f4{fabsf(x.x), fabsf(x.y), fabsf(x.z), fabsf(x.w)}; }

// G, P, C: types of gradient, parameter and copy (C < 0: none).
template <int G, int P, int C, int BITS>
__global__ void __launch_bounds__(kWave * kRowWaves)
k_adamw(const TensorEntry* __restrict__ entries, const uint32_t* __restrict__ tile_tensor, AdamArgs a)
{
    const uint32_t row = blockIdx.x * kRowWaves + wave_index();
    if (row >= a.rows) return;
    const uint32_t tile = row / kTileRows;
    const TensorEntry d = entries[tile_tensor[tile]];
    const size_t e0 = static_cast<size_t>(tile - d.first_tile) * kTensorTile + (row % kTileRows) * kRow;
    if (e0 >= d.numel) return;
    float factor = 1.0f;
    if (a.clip) {
        if (!(fabsf(a.clip[0]) < INFINITY)) return;
        factor = a.clip[1];
    }
    const int lane = threadIdx.x & 63;
    const int remain = d.numel - e0 < static_cast<size_t>(kRow) ? static_cast<int>(d.numel - e0) : kRow;
    typedef typename Elem<P>::one param_t;
    param_t* pp = table_ptr<param_t>(d.param) + e0;

    f4 p = load_four<P>(pp, lane, remain);
    f4 g = load_four<G>(table_ptr<const typename Elem<G>::one>(d.grad) + e0, lane, remain);
    f4 m, v;
    if (BITS == 32) {
        m = load_four<BAGUA_F32>(table_ptr<const float>(d.m) + e0, lane, remain);
        v = load_four<BAGUA_F32>(table_ptr<const float>(d.v) + e0, lane, remain);
    } else {
        const size_t block = e0 / kRow;
        m = widen_codes(load_four_codes(table_ptr<const uint8_t>(d.m) + e0, lane, remain), table_ptr<const float>(d.m_scale)[block]);
        const f4 r = widen_codes(load_four_codes(table_ptr<const uint8_t>(d.v) + e0, lane, remain), table_ptr<const float>(d.v_scale)[block]);
        v = r * r;
    }
    if (a.clip) g = g * factor;
    m = m * a.beta1 + g * a.omb1;
    v = v * a.beta2 + (g * g) * a.omb2;
    const f4 r = f4{sqrtf(v.x), sqrtf(v.y), sqrtf(v.z), sqrtf(v.w)};
    const f4 u = m / (r * a.root + a.eps);
    p = p - (u * a.rate + p * (d.decay * a.decay));

    uint32_t h = 0;
    if (BITS == 8 || P == BAGUA_BF16)
        h = mix((static_cast<uint32_t>(e0 / 4) + lane) * kGolden + mix(d.index * kGolden + a.seed));
    if (BITS == 32) {
        store_four<BAGUA_F32>(table_ptr<float>(d.m) + e0, lane, remain, m);
        store_four<BAGUA_F32>(table_ptr<float>(d.v) + e0, lane, remain, v);
    } else {
        // the absent elements of a last row hold 0
        const Scale ms = scale_of(wave_reduce(max4(abs4(m)), OpMaxF())), vs = scale_of(wave_reduce(max4(r), OpMaxF()));
        const f4 y = r * vs.inverse;
        const uint32_t w = random_code(y.x, r.x, turned(h, 0)) | random_code(y.y, r.y, turned(h, 8)) << 8 |
                           random_code(y.z, r.z, turned(h, 16)) << 16 | random_code(y.w, r.w, turned(h, 24)) << 24;
        store_four_codes(table_ptr<uint8_t>(d.m) + e0, lane, remain, nearest_codes(m * ms.inverse));
        store_four_codes(table_ptr<uint8_t>(d.v) + e0, lane, remain, w);
        if (lane == 0) {
            table_ptr<float>(d.m_scale)[e0 / kRow] = ms.scale;
            table_ptr<float>(d.v_scale)[e0 / kRow] = vs.scale;
        }
    }
    if constexpr (P == BAGUA_BF16) {
        const uint32_t h2 = mix(h + kGolden);
        const h4 q = h4{random_bf16(p.x, turned(h2, 0)), random_bf16(p.y, turned(h2, 8)), random_bf16(p.z, turned(h2, 16)), random_bf16(p.w, turned(h2, 24))};
        const int e = lane * 4;
        if (remain >= kRow) {
            __builtin_nontemporal_store(static_cast<h4e>(q), reinterpret_cast<h4e*>(pp + e));
        } else {
            if (e + 0 < remain) pp[e + 0] = q.x;
            if (e + 1 < remain) pp[e + 1] = q.y;
            if (e + 2 < remain) pp[e + 2] = q.z;
            if (e + 3 < remain) pp[e + 3] = q.w;
        }
    } else {
        store_four<P>(pp, lane, remain, p);
    }
    if constexpr (C >= 0) store_four<C>(table_ptr<typename Elem<C>::one>(d.copy) + e0, lane, remain, p);
}

// ---------------------------------------------------------------- norm
// Squares are exact in 64 bits and their sum loses nothing that an fp32 result could show, whatever the order; 64-bit additions
// run at half the rate of fp32 ones, a twentieth of what the loads leave time for.  Each workgroup sums every gridDim-th tile;
// the workgroup that finishes last adds the groups' sums in ascending order.
template <int G>
__global__ void __launch_bounds__(kWave * kNormWaves)
k_grad_norm(TensorPlanView plan, uint32_t tiles, double scale, double max_norm, float* __restrict__ out)
{
    const int lane = threadIdx.x & 63, wave = wave_index();
    double sum = 0.0;
    for (uint32_t tile = blockIdx.x * kNormWaves + wave; tile < tiles; tile += gridDim.x * kNormWaves) {
        const TensorEntry d = plan.entry[plan.tile_tensor[tile]];
        const size_t e0 = static_cast<size_t>(tile - d.first_tile) * kTensorTile;
        const typename Elem<G>::one* g = table_ptr<const typename Elem<G>::one>(d.grad) + e0;
        const size_t left = d.numel - e0;
        f4 x[kTileRows];
        if (left >= kTensorTile) {
#pragma unroll
            for (int i = 0; i < kTileRows; ++i) x[i] = Elem<G>::load(g + i * kRow + lane * 4);
        } else {
#pragma unroll
            for (int i = 0; i < kTileRows; ++i) x[i] = load_four<G>(g + i * kRow, lane, static_cast<int>(left) - i * kRow);
        }
#pragma unroll
        for (int i = 0; i < kTileRows; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const double y = static_cast<double>(x[i][j]);
                sum = __builtin_fma(y, y, sum);
            }
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
    __shared__ double part[kNormWaves];
    __shared__ bool last;
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) publish(plan.partial + blockIdx.x, (part[0] + part[1]) + (part[2] + part[3]));
    if (!last_to_arrive(plan.counter, &last)) return;
    sum = 0.0;
#pragma unroll 8
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kWave * kNormWaves) sum += plan.partial[i];
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    __hip_atomic_store(plan.counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next call
    const double n = scale * sqrt((part[0] + part[1]) + (part[2] + part[3]));
    const float norm = static_cast<float>(n);
    out[0] = norm;
    const double c = max_norm / (n + 1e-6);
    out[1] = fabsf(norm) < INFINITY ? static_cast<float>(scale * (c < 1.0 ? c : 1.0)) : 0.0f;
}

inline size_t tiles_of(size_t numel) { return numel / kTensorTile + (numel % kTensorTile != 0); }
constexpr size_t kMaxTiles = kMaxGrid / kTileRows;   // one launch of single-wave rows holds them

inline size_t tensor_plan_bytes(size_t T, size_t tiles)
{
    return (kEntriesAt + T * sizeof(TensorEntry) + tiles * sizeof(uint32_t) + 15) & ~static_cast<size_t>(15);
}

}  // namespace bagua

using namespace bagua;

extern "C" size_t bagua_tensor_plan_bytes(const size_t* numel, size_t T)
{
    if (!numel || T == 0 || T > 0xfffffff0u) return 0;
    size_t tiles = 0;
    for (size_t t = 0; t < T && tiles <= kMaxTiles; ++t) tiles += tiles_of(numel[t]);
    return tiles > kMaxTiles ? 0 : tensor_plan_bytes(T, tiles);
}

extern "C" int bagua_tensor_plan(const size_t* numel, size_t T, const void* const* grad, int grad_type, void* const* param,
                                 int param_type, void* const* m, void* const* v, int state_bits, float* const* m_scale,
                                 float* const* v_scale, void* const* copy, int copy_type, const float* decay, void* workspace,
                                 size_t workspace_bytes, bagua_tensor_plan_t* plan, void* stream)
{
    if (!numel || T == 0 || !grad || !workspace || !plan || !type_ok(grad_type)) return BAGUA_ERR_INVALID_ARG;
    if (param) {
        if (!m || !v || (state_bits != 8 && state_bits != 32)) return BAGUA_ERR_INVALID_ARG;
        if (param_type != BAGUA_F32 && param_type != BAGUA_BF16) return BAGUA_ERR_INVALID_ARG;
        if (param_type == BAGUA_BF16 && (copy || grad_type == BAGUA_F16)) return BAGUA_ERR_INVALID_ARG;
        if ((state_bits == 8) != (m_scale != nullptr) || (state_bits == 8) != (v_scale != nullptr)) return BAGUA_ERR_INVALID_ARG;
        if (copy && copy_type != BAGUA_BF16 && copy_type != BAGUA_F16) return BAGUA_ERR_INVALID_ARG;
    } else if (m || v || m_scale || v_scale || copy || decay || state_bits != 0) {
        return BAGUA_ERR_INVALID_ARG;
    }
    if (T > 0xfffffff0u) return BAGUA_ERR_UNSUPPORTED;
    size_t tiles = 0;
    for (size_t t = 0; t < T; ++t) {
        if (numel[t] / kTensorTile >= kMaxTiles || (tiles += tiles_of(numel[t])) > kMaxTiles) return BAGUA_ERR_UNSUPPORTED;
    }
    const size_t bytes = tensor_plan_bytes(T, tiles);
    if (workspace_bytes < bytes) return BAGUA_ERR_INVALID_ARG;
    if (!aligned16(workspace)) return BAGUA_ERR_ALIGNMENT;
    try {
        std::vector<unsigned char> host(bytes, 0);
        TensorEntry* entry = reinterpret_cast<TensorEntry*>(host.data() + kEntriesAt);
        uint32_t* tile_tensor = reinterpret_cast<uint32_t*>(entry + T);
        RangeList rl;
        rl.writes(workspace, bytes);
        uint32_t tile = 0;
        for (size_t t = 0; t < T; ++t) {
            const size_t n = numel[t];
            TensorEntry& d = entry[t];
            d.numel = n;
            d.first_tile = tile;
            d.index = static_cast<uint32_t>(t);
            d.decay = decay ? decay[t] : 1.0f;
            if (!(std::fabs(d.decay) < INFINITY)) return BAGUA_ERR_INVALID_ARG;
            for (size_t i = tiles_of(n); i > 0; --i) tile_tensor[tile++] = static_cast<uint32_t>(t);
            if (n == 0) continue;
            const size_t blocks = (n + kRow - 1) / kRow, state = state_bits / 8;
            if (!grad[t]) return BAGUA_ERR_INVALID_ARG;
            if (!aligned_to(grad[t], type_bytes(grad_type))) return BAGUA_ERR_ALIGNMENT;
            rl.reads(grad[t], n * type_bytes(grad_type));
            d.grad = reinterpret_cast<uintptr_t>(grad[t]);
            if (!param) continue;
            if (!param[t] || !m[t] || !v[t] || (m_scale && (!m_scale[t] || !v_scale[t])) || (copy && !copy[t])) return BAGUA_ERR_INVALID_ARG;
            if (!aligned_to(param[t], type_bytes(param_type)) || !aligned_to(m[t], state) || !aligned_to(v[t], state) ||
                (m_scale && (!aligned4(m_scale[t]) || !aligned4(v_scale[t]))) || (copy && !aligned2(copy[t])))
                return BAGUA_ERR_ALIGNMENT;
            rl.writes(param[t], n * type_bytes(param_type));
            rl.writes(m[t], n * state);
            rl.writes(v[t], n * state);
            d.param = reinterpret_cast<uintptr_t>(param[t]);
            d.m = reinterpret_cast<uintptr_t>(m[t]);
            d.v = reinterpret_cast<uintptr_t>(v[t]);
            if (m_scale) {
                rl.writes(m_scale[t], blocks * sizeof(float));
                rl.writes(v_scale[t], blocks * sizeof(float));
                d.m_scale = reinterpret_cast<uintptr_t>(m_scale[t]);
                d.v_scale = reinterpret_cast<uintptr_t>(v_scale[t]);
            }
            if (copy) {
                rl.writes(copy[t], n * type_bytes(copy_type));
                d.copy = reinterpret_cast<uintptr_t>(copy[t]);
            }
        }
        if (!rl.disjoint()) return BAGUA_ERR_INVALID_ARG;
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (hipMemcpyAsync(workspace, host.data(), bytes, hipMemcpyHostToDevice, s) != hipSuccess) return BAGUA_ERR_LAUNCH;
        if (hipStreamSynchronize(s) != hipSuccess) return BAGUA_ERR_LAUNCH;   // `host` dies at return
    } catch (const std::bad_alloc&) {
        return BAGUA_ERR_UNSUPPORTED;   // more tensors than the host has memory to list
    }
    *plan = bagua_tensor_plan_t{workspace, tiles, static_cast<uint32_t>(T), grad_type, param ? param_type : -1, copy ? copy_type : -1, state_bits};
    return BAGUA_OK;
}

static bool plan_ok(const bagua_tensor_plan_t* plan)
{
    return plan && plan->workspace && aligned16(plan->workspace) && plan->tensors != 0 && plan->tiles <= kMaxTiles && type_ok(plan->grad_type);
}

extern "C" int bagua_grad_norm(const bagua_tensor_plan_t* plan, double grad_scale, double max_norm, float* out, void* stream)
{
    if (!plan_ok(plan) || !out || !(std::fabs(grad_scale) < INFINITY) || !(max_norm >= 0.0)) return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(out)) return BAGUA_ERR_ALIGNMENT;
    const size_t groups = (plan->tiles + kNormWaves - 1) / kNormWaves;
    const dim3 grid(static_cast<unsigned>(std::min<size_t>(std::max<size_t>(groups, 1), kNormGroups))), block(kWave * kNormWaves);
    const TensorPlanView view = tensor_plan_view(plan);
    auto* kernel = plan->grad_type == BAGUA_F32 ? k_grad_norm<BAGUA_F32> : plan->grad_type == BAGUA_BF16 ? k_grad_norm<BAGUA_BF16> : k_grad_norm<BAGUA_F16>;
    launch_kernel(kernel, grid, block, 0, static_cast<hipStream_t>(stream), view, static_cast<uint32_t>(plan->tiles), grad_scale, max_norm, out);
    return launch_status();
}

namespace bagua {
typedef void (*AdamKernel)(const TensorEntry*, const uint32_t*, AdamArgs);

template <int G, int BITS>
AdamKernel pick_adamw(int param_type, int copy_type)
{
    if constexpr (G != BAGUA_F16)
        if (param_type == BAGUA_BF16) return k_adamw<G, BAGUA_BF16, -1, BITS>;
    return copy_type == BAGUA_BF16 ? k_adamw<G, BAGUA_F32, BAGUA_BF16, BITS>
           : copy_type == BAGUA_F16 ? k_adamw<G, BAGUA_F32, BAGUA_F16, BITS> : k_adamw<G, BAGUA_F32, -1, BITS>;
}
template <int BITS>
AdamKernel pick_adamw(int grad_type, int param_type, int copy_type)
{
    return grad_type == BAGUA_F32 ? pick_adamw<BAGUA_F32, BITS>(param_type, copy_type)
           : grad_type == BAGUA_BF16 ? pick_adamw<BAGUA_BF16, BITS>(param_type, copy_type) : pick_adamw<BAGUA_F16, BITS>(param_type, copy_type);
}
}  // namespace bagua

extern "C" int bagua_adamw_step(const bagua_tensor_plan_t* plan, uint64_t step, double lr, double beta1, double beta2, double eps,
                                double weight_decay, const float* clip, uint32_t seed, void* stream)
{
    if (!plan_ok(plan) || (plan->state_bits != 8 && plan->state_bits != 32) || step == 0) return BAGUA_ERR_INVALID_ARG;
    if (!(std::fabs(lr) < INFINITY) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0 && eps < INFINITY) ||
        !(std::fabs(weight_decay) < INFINITY))
        return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(clip)) return BAGUA_ERR_ALIGNMENT;
    if (plan->tiles == 0) return BAGUA_OK;
    const TensorPlanView view = tensor_plan_view(plan);
    const uint32_t rows = static_cast<uint32_t>(plan->tiles * kTileRows);
    const double t = static_cast<double>(step);
    const AdamArgs a{clip, static_cast<float>(beta1), static_cast<float>(1.0 - beta1), static_cast<float>(beta2), static_cast<float>(1.0 - beta2),
                     static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(beta2, t))), static_cast<float>(eps),
                     static_cast<float>(lr / (1.0 - std::pow(beta1, t))), static_cast<float>(lr * weight_decay), seed, rows};
    const AdamKernel kernel = plan->state_bits == 32 ? pick_adamw<32>(plan->grad_type, plan->param_type, plan->copy_type)
                                                     : pick_adamw<8>(plan->grad_type, plan->param_type, plan->copy_type);
    launch_kernel(kernel, dim3((rows + kRowWaves - 1) / kRowWaves), dim3(kWave * kRowWaves), 0, static_cast<hipStream_t>(stream), view.entry,
                  view.tile_tensor, a);
    return launch_status();
}
