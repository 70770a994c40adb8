// C-ABI entry points of routing of tokens to experts and its backward pass (see bagua_hip.h).
#include <cmath>

#include "route.hpp"

namespace bagua {

inline uint32_t reciprocal_of(int d) { return d == 1 ? 0 : static_cast<uint32_t>((0x100000000ull + static_cast<uint64_t>(d) - 1) / static_cast<uint64_t>(d)); }

inline int route_check(int dtype, const size_t* tokens, int k, int experts, int score, int top_k, int id_bytes, double scale)
{
    if (!tokens || !type_ok(dtype) || k < 1 || k > BAGUA_MAX_WORKERS || experts < 1 || top_k < 1 || top_k > experts || (id_bytes != 4 && id_bytes != 8) ||
        (score != BAGUA_SCORE_SOFTMAX && score != BAGUA_SCORE_SIGMOID) || !(std::fabs(scale) < INFINITY))
        return BAGUA_ERR_INVALID_ARG;
    if (experts > BAGUA_MAX_EXPERTS || top_k > BAGUA_MAX_CHOICES || std::fabs(scale) > 0x1p64) return BAGUA_ERR_UNSUPPORTED;
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
    a.per_each = reciprocal_of(a.each), a.per_groups = reciprocal_of(groups);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == BAGUA_F32) return launch_route<BAGUA_F32>(ls, a, tokens, k, s);
    if (dtype == BAGUA_BF16) return launch_route<BAGUA_BF16>(ls, a, tokens, k, s);
    return launch_route<BAGUA_F16>(ls, a, tokens, k, s);
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
    if (of_weights && std::fabs(scale) < 0x1p-64) return BAGUA_ERR_UNSUPPORTED;      // (it is divided by)
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
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == BAGUA_F32) return launch_route_grad<BAGUA_F32>(ls, a, tokens, k, s);
    if (dtype == BAGUA_BF16) return launch_route_grad<BAGUA_BF16>(ls, a, tokens, k, s);
    return launch_route_grad<BAGUA_F16>(ls, a, tokens, k, s);
}
