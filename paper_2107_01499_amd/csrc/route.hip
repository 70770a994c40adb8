// Routing of tokens to experts and its backward pass (see bagua_hip.h).
//
// A row of logits lies in L lanes as in rows.hpp.  Which experts are chosen has to be what numbers of 64 bits give, though the scores are formed in
// 32: an element's key is its choice score, as an integer that is ordered as the numbers are, with the last bits replaced by how far its
// expert lies from the last one, so that a maximum of keys is the best score and of equal ones the lowest expert.  Where two neighbours among
// the chosen lie closer than the error of 32 bits (and are not the same logit with the same bias), the row is done again in 64 bits.
#include <cmath>

#include "lists.hpp"
#include "rows.hpp"

#pragma clang fp contract(off)

namespace bagua {

constexpr int kRouteWaves = 4;
constexpr uint32_t kRouteMostWaves = 65536;   // of a launch
constexpr int kMoreChoices = 4;               // rounds beyond the last choice that look for the end of a run of equal scores

enum { kLogits = 0, kMask, kIds, kWeights, kRouteLists };

struct RouteArgs {
    size_t ld, ids_ld, weights_ld;
    const float* bias;
    int experts, top_k, groups, each, top_groups, group_best, score, renormalise, id_bytes;
    int by_logit;              // the scores need not be formed: experts are chosen by their logits
    float scale;
    uint32_t index_mask;       // the bits of a key that tell the expert
    uint32_t per_k, per_each, per_groups;     // reciprocals, 0 for a divisor of 1
    uint32_t wave_words;       // LDS of a wave
    uint32_t part;             // lanes that look through a group together, a power of two
};

// Integers that are ordered as the numbers are; NaN above all, both zeros the same.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0xffffffffu : b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number(uint32_t o) { return __uint_as_float(o ^ (static_cast<int32_t>(o) < 0 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ uint64_t ordered(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);
    return x != x ? ~0ull : b ^ (static_cast<uint64_t>(static_cast<int64_t>(b) >> 63) | 1ull << 63);
}
__device__ __forceinline__ double number(uint64_t o) { return __builtin_bit_cast(double, o ^ (static_cast<int64_t>(o) < 0 ? 1ull << 63 : ~0ull)); }

struct OpMaxU { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); } };

// Lanes of a wave wait for what others of it have written to LDS.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ uint32_t quotient(uint32_t i, uint32_t reciprocal) { return reciprocal ? __umulhi(i, reciprocal) : i; }

__device__ __forceinline__ uint64_t wave_max(uint64_t v)
{
    for (int d = 32; d > 0; d /= 2) {
        const uint64_t o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}

// One row by the whole wave, in 64 bits; key: in LDS, one for every expert.  Leaves the choices as the fast way does: experts - id, and the logit.
template <int TYPE>
__device__ __forceinline__ void choose_in_64(const typename Elem<TYPE>::one* row, const RouteArgs& a, uint64_t* key, uint32_t* chosen, float* logit)
{
    const int lane = threadIdx.x & 63;
    double most = -INFINITY, sum = 0.0;
    if (!a.by_logit && a.score == BAGUA_SCORE_SOFTMAX) {
        float top = -INFINITY;
        for (int e = lane; e < a.experts; e += kWave) top = fmaxf(top, Elem<TYPE>::widen(row[e]));
        most = lanes_most<kWave>(top);
        if (most == -INFINITY) most = 0.0;                   // nothing but -infinity: all scores are 0
        for (int e = lane; e < a.experts; e += kWave) sum += exp(static_cast<double>(Elem<TYPE>::widen(row[e])) - most);
        sum = wave_sum(sum);
    }
    for (int e = lane; e < a.experts; e += kWave) {
        const double x = Elem<TYPE>::widen(row[e]);
        double c = x;
        if (!a.by_logit) {
            c = a.score == BAGUA_SCORE_SOFTMAX ? (sum == 0.0 ? 0.0 : exp(x - most) / sum) : 1.0 / (1.0 + exp(-x));
            if (a.bias) c += static_cast<double>(a.bias[e]);
        }
        key[e] = ordered(c);
    }
    wave_sync();
    if (a.groups > 1) {
        double good = 0.0;
        if (lane < a.groups) {
            uint64_t first = 0, second = 0;
            for (int i = 0; i < a.each; ++i) {
                const uint64_t v = key[lane * a.each + i];
                second = max(second, min(first, v));
                first = max(first, v);
            }
            good = a.group_best == 2 ? number(first) + number(second) : number(first);
        }
        const uint64_t mine = ordered(good);
        int better = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint64_t o = __shfl(mine, g);
            better += o > mine || (o == mine && g < lane);
        }
        const uint64_t allowed = __ballot(lane < a.groups && better < a.top_groups);
        for (int e = lane; e < a.experts; e += kWave)
            if (!(allowed >> quotient(static_cast<uint32_t>(e), a.per_each) & 1)) key[e] = 0;
        wave_sync();
    }
    for (int j = 0; j < a.top_k; ++j) {
        uint64_t best = 0;
        uint32_t at = 0xffffffffu;
        for (int e = lane; e < a.experts; e += kWave) {
            const uint64_t v = key[e];
            if (v > best) best = v, at = static_cast<uint32_t>(e);
        }
        const uint64_t of_all = wave_max(best);
        at = ~lanes_reduce<kWave>(best == of_all ? ~at : 0u, OpMaxU());    // the lowest of those that are as good
        if (lane == 0) {
            key[at] = 0;
            chosen[j] = static_cast<uint32_t>(a.experts) - at;
            logit[j] = Elem<TYPE>::widen(row[at]);
        }
        wave_sync();
    }
}

// EXACT: 16-bit logits are what experts are chosen by, and a key holds all of one.
template <int TYPE, int VEC, int L, int NV, bool EXACT>
__global__ void __launch_bounds__(kWave * kRouteWaves)
k_route(Lists<kRouteLists> ls, RouteArgs a, uint32_t tiles)
{
    typedef Row<TYPE, VEC, L, NV> R;
    typedef typename R::one one;
    constexpr int RW = R::kRows;
    extern __shared__ uint64_t lds_of_waves[];
    const int lane = threadIdx.x & 63, wave = wave_index(), row = lane / L, in_row = lane % L, experts = a.experts, top_k = a.top_k;
    const int slots = EXACT ? top_k : top_k + kMoreChoices;
    uint32_t* lds = reinterpret_cast<uint32_t*>(lds_of_waves) + static_cast<uint32_t>(wave) * a.wave_words;
    uint32_t* keys = lds + row * slots;                                          // the choices, and the runners-up
    float* logits = reinterpret_cast<float*>(lds + RW * slots) + row * slots;    // theirs; at last the weights
    uint32_t* more = lds + ((2 * RW * slots + 1) & ~1);                          // choice scores for the groups, or the keys of 64 bits
    const LaneLists<kRouteLists> table(ls);
    const uint32_t waves = gridDim.x * (blockDim.x / kWave), index_mask = a.index_mask;
    const bool softmax = a.score == BAGUA_SCORE_SOFTMAX, with_row = !EXACT ? !a.by_logit || (softmax && !a.renormalise) : softmax && !a.renormalise;
    float own[NV][VEC];
    R::owned(experts, own);

    for (uint32_t tile = blockIdx.x * (blockDim.x / kWave) + wave; tile < tiles; tile += waves) {
        const ListTile<kRouteLists> t(table, tile, RW);
        const uint32_t my_row = min(static_cast<uint32_t>(row), t.rows - 1);
        const one* x_row = t.template ptr<const one>(kLogits) + static_cast<size_t>(t.t0 + my_row) * a.ld;
        R raw;
        raw.load(x_row, experts, true);
        const bool counts = t.at[kMask] == 0 || t.template ptr<const uint8_t>(kMask)[t.t0 + my_row] != 0;
        float x[NV][VEC], top = -INFINITY, inverse = 1.0f, error = 0.0f;       // error: of a choice score, at most
        uint32_t key[NV][VEC];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[j][i] = Elem<TYPE>::widen(raw.q[j][i]);
        if (with_row) {
            float e[1][NV][VEC], most[1];
            most[0] = top = raw.largest(e[0]);
            if (softmax) {
                exponentials_of<R>(e, most, TYPE != BAGUA_F16);
                inverse = R::reciprocal_sum(own, e[0]);
                error = inverse * 0x1p-21f;
            } else {
                const float low = fminf(top, 0.0f);
                error = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * low)) * __builtin_fmaf(-low, 0x1p-23f, 0x1p-21f);
            }
            if (!EXACT && !a.by_logit) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        float c = softmax ? e[0][j][i] * inverse : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * x[j][i]));
                        if (a.bias) c = c + a.bias[R::at(j, experts) + i];
                        key[j][i] = ordered(c);
                    }
            }
        }
        if (EXACT || a.by_logit) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) key[j][i] = ordered(x[j][i]);
        }
        bool again = false;                                                     // the row needs 64 bits
        uint32_t allowed = 0xffffffffu;
        if (a.groups > 1) {
            uint32_t* score_of = more;
            float* good = reinterpret_cast<float*>(more + RW * experts);
            uint32_t* state = more + RW * experts + RW * a.groups;              // of every row: the groups that stay; whether that is not certain
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) score_of[row * experts + R::at(j, experts) + i] = key[j][i];
            if (in_row == 0) state[row] = 0, state[RW + row] = 0;
            float* errors = reinterpret_cast<float*>(state + 2 * RW);
            if (in_row == 0) errors[row] = error;
            wave_sync();
            const uint32_t pairs = static_cast<uint32_t>(RW * a.groups), at_once = kWave / a.part, sub = static_cast<uint32_t>(lane) & (a.part - 1);
            for (uint32_t p0 = 0; p0 < pairs; p0 += at_once) {
                const uint32_t pair = p0 + static_cast<uint32_t>(lane) / a.part, r = quotient(min(pair, pairs - 1), a.per_groups), g = min(pair, pairs - 1) - r * a.groups;
                uint32_t first = 0, second = 0;
                for (uint32_t i = sub; i < static_cast<uint32_t>(a.each); i += a.part) {
                    const uint32_t v = score_of[r * experts + g * a.each + i];
                    second = max(second, min(first, v));
                    first = max(first, v);
                }
                for (uint32_t d = 1; d < a.part; d *= 2) {
                    const uint32_t f = __shfl_xor(first, d), s = __shfl_xor(second, d);
                    second = max(min(first, f), max(second, s));
                    first = max(first, f);
                }
                if (pair < pairs && sub == 0) good[pair] = a.group_best == 2 ? number(first) + number(second) : number(first);
            }
            wave_sync();
            for (uint32_t pair = lane; pair < pairs; pair += kWave) {
                const uint32_t r = quotient(pair, a.per_groups), g = pair - r * a.groups;
                const float mine = good[pair];
                int before = 0, perhaps = 0;
                if (EXACT || a.by_logit) {
                    const uint32_t o = ordered(mine);
                    for (uint32_t h = 0; h < static_cast<uint32_t>(a.groups); ++h) {
                        const uint32_t other = ordered(good[r * a.groups + h]);
                        before += other > o || (other == o && h < g);
                    }
                    perhaps = before;
                } else {
                    for (uint32_t h = 0; h < static_cast<uint32_t>(a.groups); ++h) {
                        const float other = good[r * a.groups + h], apart = 4.0f * errors[r] + fmaxf(fabsf(mine), fabsf(other)) * 0x1p-21f;
                        before += h != g && other > mine + apart;
                        perhaps += h != g && !(other < mine - apart);
                    }
                }
                if (perhaps < a.top_groups) atomicOr(state + r, 1u << g);
                else if (before < a.top_groups) atomicOr(state + RW + r, 1u);
            }
            wave_sync();
            allowed = state[row];
            again = state[RW + row] != 0;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const uint32_t e = static_cast<uint32_t>(R::at(j, experts) + i);
                key[j][i] = (key[j][i] & ~index_mask) | (static_cast<uint32_t>(experts) - e);
                if (a.groups > 1) key[j][i] = allowed >> quotient(e, a.per_each) & 1u ? key[j][i] : 0u;
            }
        // Scores of two keys, the better one first, are too close to tell in 32 bits.
        auto close = [&](uint32_t better, uint32_t worse) {
            if (worse == 0) return false;                                       // there is none
            if (a.by_logit) return (better & ~index_mask) == (worse & ~index_mask);
            const float b = number(better & ~index_mask), w = number(worse & ~index_mask);
            return !(b - w > 2.0f * error + fmaxf(fabsf(b), fabsf(w)) * (static_cast<float>(index_mask) * 0x1p-22f + 0x1p-21f));
        };
        uint32_t last = 0;
        int taken = 0;
        auto take = [&] {
            uint32_t best = 0;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) best = max(best, key[j][i]);
            best = lanes_reduce<L>(best, OpMaxU());
            float its = 0.0f;
            bool here = false;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const bool is = key[j][i] == best;
                    key[j][i] = is ? 0u : key[j][i];
                    if (!EXACT) {
                        its = is ? x[j][i] : its;
                        here |= is;
                    }
                }
            if (in_row == 0) keys[taken] = best;
            if (!EXACT && here) logits[taken] = its;
            ++taken;
            return best;
        };
        for (int j = 0; j < top_k; ++j) last = take();
        if (!EXACT) {
            for (int j = 0; j < kMoreChoices; ++j) {
                const uint32_t next = take();
                if (!__any(close(last, next))) break;
            }
        }
        wave_sync();
        if (!EXACT) {
            auto same = [&](int j) {      // not only close: the same logit with the same bias, which the expert's place decides
                if (logits[j] != logits[j + 1]) return false;
                return !a.bias || a.bias[experts - (keys[j] & index_mask)] == a.bias[experts - (keys[j + 1] & index_mask)];
            };
            for (int j = in_row; j + 1 < top_k; j += L) again |= close(keys[j], keys[j + 1]) && !same(j);
            bool ends = false;
            for (int j = top_k - 1; j + 1 < taken; ++j) {
                if (ends) break;
                if (!close(keys[j], keys[j + 1])) ends = true;
                else if (!same(j)) break;
            }
            again = (again || !ends) && counts && static_cast<uint32_t>(row) < t.rows;
            const uint64_t rows_again = __ballot(again);
            for (uint64_t left = rows_again; left != 0;) {
                const int r = (__ffsll(static_cast<unsigned long long>(left)) - 1) / L;
                const uint64_t of_row = (L == 64 ? ~0ull : (1ull << (L & 63)) - 1) << (r * L & 63);
                left &= ~of_row;
                choose_in_64<TYPE>(t.template ptr<const one>(kLogits) + static_cast<size_t>(t.t0 + static_cast<uint32_t>(r)) * a.ld, a,
                                   reinterpret_cast<uint64_t*>(more), lds + r * slots, reinterpret_cast<float*>(lds + RW * slots) + r * slots);
            }
            wave_sync();
        }
        // The weights, formed of the chosen logits.
        auto logit = [&](int j) {      // (16-bit numbers as fp32 ones have zeros in a key's last bits, turned to ones below 0)
            const uint32_t o = keys[j] & ~index_mask;
            return EXACT ? number(static_cast<int32_t>(o) < 0 ? o : o | index_mask) : logits[j];
        };
        float most = -INFINITY;
        if (a.renormalise) {
            for (int j = in_row; j < top_k; j += L) most = fmaxf(most, logit(j));
            most = lanes_most<L>(most);
            if (!softmax) most = fminf(most, 0.0f);
        } else {
            most = softmax ? top : 0.0f;
        }
        if (most == -INFINITY) most = INFINITY;                                 // nothing but -infinity: weights of 0
        float sum = 0.0f;
        for (int j = in_row; j < top_k; j += L) {
            const float v = logit(j), s = expf((softmax || v <= 0.0f ? v : 0.0f) - most);
            float w = softmax ? s : s / (1.0f + expf(v <= 0.0f ? v : -v));
            if (v != v) w = v;
            sum += w;
            logits[j] = w;
        }
        float factor = a.scale;
        if (a.renormalise) {
            sum = lanes_reduce<L>(sum, OpAddF());
            factor = sum == 0.0f ? 0.0f : a.scale / sum;
            if (inverse != inverse) factor = inverse;
        } else if (softmax) {
            factor = inverse * a.scale;
        }
        for (int j = in_row; j < top_k; j += L) {
            const float w = logits[j];
            logits[j] = counts ? w * factor : 0.0f;
            keys[j] = counts ? static_cast<uint32_t>(experts) - (keys[j] & index_mask) : 0xffffffffu;
        }
        wave_sync();
        const uint32_t items = t.rows * static_cast<uint32_t>(top_k);
        float* weights = t.template ptr<float>(kWeights);
        for (uint32_t i = static_cast<uint32_t>(lane); i < items; i += kWave) {
            const uint32_t r = quotient(i, a.per_k), j = i - r * top_k;
            const size_t token = t.t0 + r;
            const int32_t id = static_cast<int32_t>(lds[r * slots + j]);
            if (a.id_bytes == 8) t.template ptr<int64_t>(kIds)[token * a.ids_ld + j] = id;
            else t.template ptr<int32_t>(kIds)[token * a.ids_ld + j] = id;
            weights[token * a.weights_ld + j] = reinterpret_cast<const float*>(lds)[RW * slots + r * slots + j];
        }
        wave_sync();
    }
}

// ---------------------------------------------------------------------------------------------- backward
enum { kGradLogits = 0, kGradIds, kGradWeights, kGradUp, kGradOut, kRouteGradLists };

struct RouteGradArgs {
    size_t ld, ids_ld, weights_ld, up_ld, out_ld;
    int experts, top_k, score, renormalise, id_bytes;
    float scale;
    uint32_t wave_words;
};

// A row's choices are spread over a row of fp32 numbers in LDS, which is zero before and after, and read from there as it is written to memory.
// FULL: softmax that was not renormalised, whose gradient reaches every logit; elsewhere the chosen ones alone.
template <int TYPE, int VEC, int L, int NV, bool FULL>
__global__ void __launch_bounds__(kWave * kRouteWaves)
k_route_grad(Lists<kRouteGradLists> ls, RouteGradArgs a, uint32_t tiles)
{
    typedef Row<TYPE, VEC, L, NV> R;
    typedef typename R::one one;
    constexpr int RW = R::kRows;
    extern __shared__ uint64_t lds_of_waves[];
    const int lane = threadIdx.x & 63, wave = wave_index(), row = lane / L, in_row = lane % L, experts = a.experts, top_k = a.top_k;
    float* spread = reinterpret_cast<float*>(lds_of_waves) + static_cast<uint32_t>(wave) * a.wave_words + row * experts;
    const LaneLists<kRouteGradLists> table(ls);
    const uint32_t waves = gridDim.x * (blockDim.x / kWave);
    float own[NV][VEC];
    R::owned(experts, own);
    for (int e = in_row; e < experts; e += L) spread[e] = 0.0f;
    wave_sync();
    for (uint32_t tile = blockIdx.x * (blockDim.x / kWave) + wave; tile < tiles; tile += waves) {
        const ListTile<kRouteGradLists> t(table, tile, RW);
        const bool there = static_cast<uint32_t>(row) < t.rows;
        const size_t token = t.t0 + min(static_cast<uint32_t>(row), t.rows - 1);
        const one* x_row = t.template ptr<const one>(kGradLogits) + token * a.ld;
        R raw;
        if (FULL) raw.load(x_row, experts, true);
        auto id = [&](int j) {
            const int64_t v = a.id_bytes == 8 ? t.template ptr<const int64_t>(kGradIds)[token * a.ids_ld + j]
                                              : static_cast<int64_t>(t.template ptr<const int32_t>(kGradIds)[token * a.ids_ld + j]);
            return static_cast<uint64_t>(v) < static_cast<uint64_t>(experts) ? static_cast<int>(v) : -1;
        };
        auto up = [&](int j) { return t.template ptr<const float>(kGradUp)[token * a.up_ld + j]; };
        const bool shares = !FULL && a.renormalise, softmax = FULL || a.score == BAGUA_SCORE_SOFTMAX;
        // a choice's part of the sum that the weights were divided by, and their mean gradient
        const float* weights = t.template ptr<const float>(kGradWeights);
        float most = -INFINITY, sum = 0.0f, mean = 0.0f;
        bool any = false;
        auto share = [&](int j, int e) {
            if (softmax) return weights[token * a.weights_ld + j] / a.scale;
            const float v = Elem<TYPE>::widen(x_row[e]);
            return expf((v <= 0.0f ? v : 0.0f) - most) / (1.0f + expf(v <= 0.0f ? v : -v));
        };
        if (shares && !softmax) {
            for (int j = in_row; j < top_k; j += L) {
                const int e = id(j);
                if (e >= 0) most = fmaxf(most, Elem<TYPE>::widen(x_row[e]));
            }
            most = fminf(lanes_most<L>(most), 0.0f);
            if (most == -INFINITY) most = INFINITY;
        }
        for (int j = in_row; j < top_k; j += L) {
            const int e = id(j);
            any |= e >= 0;
            if (shares && e >= 0) {
                const float r = share(j, e);
                sum += r;
                mean = __builtin_fmaf(r, up(j), mean);
            }
        }
        if (shares) {
            sum = softmax ? 1.0f : lanes_reduce<L>(sum, OpAddF());
            mean = lanes_reduce<L>(mean, OpAddF());
            mean = sum == 0.0f ? 0.0f : mean / sum;
        }
        // what a choice adds to its logit
        auto part = [&](int j, int e) {
            if (FULL) return up(j);
            if (shares) {
                const float r = sum == 0.0f ? 0.0f : share(j, e) / sum, d = a.scale * r * (up(j) - mean);
                if (softmax) return d;
                const float v = Elem<TYPE>::widen(x_row[e]), far = expf(v <= 0.0f ? v : -v);
                return d * ((v <= 0.0f ? 1.0f : far) / (1.0f + far));
            }
            const float v = Elem<TYPE>::widen(x_row[e]), far = expf(v <= 0.0f ? v : -v);
            return a.scale * up(j) * (far / ((1.0f + far) * (1.0f + far)));
        };
        // An expert that a row names twice gets both, one after the other in every call; the rows that have one are found by writing the
        // choices' places first.
        bool twice = false;
        for (int j = in_row; j < top_k && there; j += L) {
            const int e = id(j);
            if (e >= 0) reinterpret_cast<uint32_t*>(spread)[e] = static_cast<uint32_t>(j);
        }
        wave_sync();
        for (int j = in_row; j < top_k && there; j += L) {
            const int e = id(j);
            twice |= e >= 0 && reinterpret_cast<uint32_t*>(spread)[e] != static_cast<uint32_t>(j);
        }
        wave_sync();
        if (!__any(twice)) {
            for (int j = in_row; j < top_k && there; j += L) {
                const int e = id(j);
                if (e >= 0) spread[e] = part(j, e);
            }
        } else {
            for (int j = in_row; j < top_k && there; j += L) {
                const int e = id(j);
                if (e >= 0) spread[e] = 0.0f;
            }
            wave_sync();
            for (int j = 0; j < top_k; ++j) {
                const int e = there && j % L == in_row ? id(j) : -1;
                if (e >= 0) spread[e] += part(j, e);
                wave_sync();
            }
        }
        wave_sync();
        float e[1][NV][VEC], factor = 0.0f, shift = 0.0f, most_of[1];
        if (FULL) {
            float dot = 0.0f;
            most_of[0] = raw.largest(e[0]);
            exponentials_of<R>(e, most_of, TYPE != BAGUA_F16);
            const float inverse = R::reciprocal_sum(own, e[0]);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) dot = __builtin_fmaf(e[0][j][i], spread[R::at(j, experts) + i] * own[j][i], dot);
            shift = lanes_reduce<L>(dot, OpAddF()) * inverse;
            factor = a.scale * inverse;
            // a row without a choice (padding) has no gradient, whatever its logits are
            const uint64_t chosen = __ballot(any), of_row = (L == 64 ? ~0ull : (1ull << (L & 63)) - 1) << (row * L & 63);
            any = (chosen & of_row) != 0;
        }
        one* out = t.template ptr<one>(kGradOut) + token * a.out_ld;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            typename R::raw q;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float s = spread[R::at(j, experts) + i];
                q[i] = Elem<TYPE>::narrow(FULL ? (any ? e[0][j][i] * (factor * (s - shift)) : 0.0f) : s);
            }
            if (there) __builtin_nontemporal_store(q, reinterpret_cast<typename R::raw*>(out + R::at(j, experts)));
        }
        wave_sync();
        for (int j = in_row; j < top_k && there; j += L) {
            const int at = id(j);
            if (at >= 0) spread[at] = 0.0f;
        }
        wave_sync();
    }
}

inline uint32_t reciprocal_of(int d) { return d == 1 ? 0 : static_cast<uint32_t>((0x100000000ull + static_cast<uint64_t>(d) - 1) / static_cast<uint64_t>(d)); }

// Waves of a workgroup whose LDS fits, and the grid.
inline int route_waves(size_t wave_bytes)
{
    int waves = kRouteWaves;
    while (waves > 1 && waves * wave_bytes > 64 * 1024) waves /= 2;
    return waves;
}
inline dim3 route_grid(uint64_t tiles, int waves) { return dim3(static_cast<uint32_t>((std::min<uint64_t>(tiles, kRouteMostWaves) + waves - 1) / waves)); }

inline int route_check(int dtype, const size_t* tokens, int k, int experts, int score, int top_k, int id_bytes, double scale)
{
    if (!tokens || !type_ok(dtype) || k < 1 || k > BAGUA_MAX_WORKERS || experts < 1 || top_k < 1 || top_k > experts || (id_bytes != 4 && id_bytes != 8) ||
        (score != BAGUA_SCORE_SOFTMAX && score != BAGUA_SCORE_SIGMOID) || !(std::fabs(scale) < INFINITY))
        return BAGUA_ERR_INVALID_ARG;
    if (experts > BAGUA_MAX_EXPERTS || top_k > BAGUA_MAX_CHOICES) return BAGUA_ERR_UNSUPPORTED;
    for (int w = 0; w < k; ++w)
        if (tokens[w] > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    return BAGUA_OK;
}

}  // namespace bagua

using namespace bagua;

extern "C" int bagua_route(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts, const uint8_t* const* mask,
                           const float* bias, int score, int groups, int top_groups, int group_best, int top_k, int renormalise, double scale,
                           void* const* ids, int id_bytes, size_t ids_ld, float* const* weights, size_t weights_ld, void* stream)
{
    const int bad = route_check(dtype, tokens, k, experts, score, top_k, id_bytes, scale);
    if (bad) return bad;
    if (!logits || !ids || !weights || ld < static_cast<size_t>(experts) || ids_ld < static_cast<size_t>(top_k) || weights_ld < static_cast<size_t>(top_k) ||
        groups < 1 || experts % groups != 0 || top_groups < 1 || top_groups > groups || (group_best != 1 && group_best != 2) || group_best > experts / groups ||
        top_k > top_groups * (experts / groups))
        return BAGUA_ERR_INVALID_ARG;
    if (groups > BAGUA_MAX_EXPERT_GROUPS || ld > kMostStride || ids_ld > kMostStride || weights_ld > kMostStride) return BAGUA_ERR_UNSUPPORTED;
    if (top_groups == groups) groups = top_groups = group_best = 1;            // all groups stay
    Lists<kRouteLists> ls{};
    RangeCheck rc;
    const size_t e = static_cast<size_t>(experts), id_size = static_cast<size_t>(id_bytes), choices = static_cast<size_t>(top_k);
    for (int w = 0; w < k; ++w) {
        if (tokens[w] == 0) continue;
        if (!logits[w] || !ids[w] || !weights[w] || (mask && !mask[w])) return BAGUA_ERR_INVALID_ARG;
        if (!aligned_to(logits[w], type_bytes(dtype)) || !aligned_to(ids[w], id_size) || !aligned4(weights[w])) return BAGUA_ERR_ALIGNMENT;
        rc.reads(logits[w], rows_bytes(tokens[w], ld, e, type_bytes(dtype)));
        if (mask) rc.reads(mask[w], tokens[w]);
        rc.writes(ids[w], rows_bytes(tokens[w], ids_ld, choices, id_size));
        rc.writes(weights[w], rows_bytes(tokens[w], weights_ld, choices, sizeof(float)));
        ls.at[kLogits][w] = logits[w];
        ls.at[kMask][w] = mask ? mask[w] : nullptr;
        ls.at[kIds][w] = ids[w];
        ls.at[kWeights][w] = weights[w];
    }
    rc.reads(bias, e * sizeof(float));
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(bias)) return BAGUA_ERR_ALIGNMENT;
    RouteArgs a{};
    a.ld = ld, a.ids_ld = ids_ld, a.weights_ld = weights_ld, a.bias = bias;
    a.experts = experts, a.top_k = top_k, a.groups = groups, a.each = experts / groups, a.top_groups = top_groups, a.group_best = group_best;
    a.score = score, a.renormalise = renormalise != 0, a.id_bytes = id_bytes, a.scale = static_cast<float>(scale);
    a.by_logit = !bias && group_best == 1;                                     // the scores rise with the logits
    int bits = 1;
    while (1 << bits <= experts) ++bits;
    a.index_mask = (1u << bits) - 1;
    a.per_k = reciprocal_of(top_k), a.per_each = reciprocal_of(a.each), a.per_groups = reciprocal_of(groups);
    const bool exact = a.by_logit && dtype != BAGUA_F32;
    int status = BAGUA_OK;
    with_layout<false>(dtype, experts, [&](auto layout, auto type) {
        typedef decltype(layout) Lay;
        constexpr int TYPE = decltype(type)::value;
        constexpr uint32_t RW = kWave / Lay::L;
        const uint64_t tiles = tiles_of(ls, tokens, k, RW);
        if (tiles > kMaxGrid) {
            status = BAGUA_ERR_UNSUPPORTED;
            return;
        }
        if (tiles == 0) return;
        a.part = 1;
        while (a.part < 16 && 2 * a.part * RW * static_cast<uint32_t>(groups) <= kWave && 2 * a.part <= static_cast<uint32_t>(a.each)) a.part *= 2;
        const uint32_t chosen = (2 * RW * static_cast<uint32_t>(top_k + (exact ? 0 : kMoreChoices)) + 1) & ~1u;
        const uint32_t for_groups = groups > 1 ? RW * (static_cast<uint32_t>(experts) + static_cast<uint32_t>(groups) + 3) : 0, for_64 = exact ? 0 : 2 * static_cast<uint32_t>(experts);
        a.wave_words = (chosen + std::max(for_groups, for_64) + 1) & ~1u;
        const size_t wave_bytes = a.wave_words * sizeof(uint32_t);
        const int waves = route_waves(wave_bytes);
        const dim3 grid = route_grid(tiles, waves), block(static_cast<uint32_t>(kWave * waves));
        auto launch = [&](auto kernel) {
            launch_kernel(kernel, grid, block, wave_bytes * static_cast<size_t>(waves), static_cast<hipStream_t>(stream), ls, a, static_cast<uint32_t>(tiles));
        };
        if constexpr (TYPE != BAGUA_F32) {
            if (exact) launch(k_route<TYPE, Lay::VEC, Lay::L, Lay::NV, true>);
        }
        if (!exact) launch(k_route<TYPE, Lay::VEC, Lay::L, Lay::NV, false>);
        status = launch_status();
    });
    return status;
}

extern "C" int bagua_route_grad(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts, const void* const* ids, int id_bytes,
                                size_t ids_ld, int top_k, const float* const* weights, size_t weights_ld, const float* const* dweights, size_t dweights_ld,
                                int score, int renormalise, double scale, void* const* dlogits, size_t ld_out, void* stream)
{
    const int bad = route_check(dtype, tokens, k, experts, score, top_k, id_bytes, scale);
    if (bad) return bad;
    const bool of_weights = score == BAGUA_SCORE_SOFTMAX && renormalise;       // the weights tell all; elsewhere the logits do
    if (!ids || !dweights || !dlogits || ids_ld < static_cast<size_t>(top_k) || dweights_ld < static_cast<size_t>(top_k) || ld_out < static_cast<size_t>(experts))
        return BAGUA_ERR_INVALID_ARG;
    if (of_weights ? !weights || weights_ld < static_cast<size_t>(top_k) || scale == 0.0 : !logits || ld < static_cast<size_t>(experts)) return BAGUA_ERR_INVALID_ARG;
    if (ids_ld > kMostStride || dweights_ld > kMostStride || ld_out > kMostStride || (of_weights ? weights_ld : ld) > kMostStride) return BAGUA_ERR_UNSUPPORTED;
    Lists<kRouteGradLists> ls{};
    RangeCheck rc;
    const size_t e = static_cast<size_t>(experts), element = type_bytes(dtype), id_size = static_cast<size_t>(id_bytes), choices = static_cast<size_t>(top_k);
    for (int w = 0; w < k; ++w) {
        if (tokens[w] == 0) continue;
        if (!ids[w] || !dweights[w] || !dlogits[w] || !(of_weights ? weights[w] != nullptr : logits[w] != nullptr)) return BAGUA_ERR_INVALID_ARG;
        if (!aligned_to(ids[w], id_size) || !aligned4(dweights[w]) || !aligned_to(dlogits[w], element) ||
            !(of_weights ? aligned4(weights[w]) : aligned_to(logits[w], element)))
            return BAGUA_ERR_ALIGNMENT;
        rc.reads(ids[w], rows_bytes(tokens[w], ids_ld, choices, id_size));
        rc.reads(dweights[w], rows_bytes(tokens[w], dweights_ld, choices, sizeof(float)));
        if (of_weights) rc.reads(weights[w], rows_bytes(tokens[w], weights_ld, choices, sizeof(float)));
        else rc.reads(logits[w], rows_bytes(tokens[w], ld, e, element));
        rc.writes(dlogits[w], rows_bytes(tokens[w], ld_out, e, element));
        ls.at[kGradLogits][w] = of_weights ? nullptr : logits[w];
        ls.at[kGradIds][w] = ids[w];
        ls.at[kGradWeights][w] = of_weights ? weights[w] : nullptr;
        ls.at[kGradUp][w] = dweights[w];
        ls.at[kGradOut][w] = dlogits[w];
    }
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    RouteGradArgs a{};
    a.ld = ld, a.ids_ld = ids_ld, a.weights_ld = weights_ld, a.up_ld = dweights_ld, a.out_ld = ld_out;
    a.experts = experts, a.top_k = top_k, a.score = score, a.renormalise = renormalise != 0, a.id_bytes = id_bytes, a.scale = static_cast<float>(scale);
    int status = BAGUA_OK;
    with_layout<false>(dtype, experts, [&](auto layout, auto type) {
        typedef decltype(layout) Lay;
        constexpr int TYPE = decltype(type)::value;
        constexpr uint32_t RW = kWave / Lay::L;
        const uint64_t tiles = tiles_of(ls, tokens, k, RW);
        if (tiles > kMaxGrid) {
            status = BAGUA_ERR_UNSUPPORTED;
            return;
        }
        if (tiles == 0) return;
        a.wave_words = (RW * static_cast<uint32_t>(experts) + 1) & ~1u;
        const size_t wave_bytes = a.wave_words * sizeof(uint32_t);
        const int waves = route_waves(wave_bytes);
        const dim3 grid = route_grid(tiles, waves), block(static_cast<uint32_t>(kWave * waves));
        auto launch = [&](auto kernel) {
            launch_kernel(kernel, grid, block, wave_bytes * static_cast<size_t>(waves), static_cast<hipStream_t>(stream), ls, a, static_cast<uint32_t>(tiles));
        };
        if (score == BAGUA_SCORE_SOFTMAX && !renormalise) launch(k_route_grad<TYPE, Lay::VEC, Lay::L, Lay::NV, true>);
        else launch(k_route_grad<TYPE, Lay::VEC, Lay::L, Lay::NV, false>);
        status = launch_status();
    });
    return status;
}
