// Arguments of the kernels of routing, and their launches for each element type.
#pragma once
#include "lists.hpp"

namespace bagua {

enum { kLogits = 0, kMask, kIds, kWeights, kRouteLists };

struct RouteArgs {
    size_t ld, ids_ld, weights_ld;
    const float* bias;
    int experts, top_k, groups, each, top_groups, group_best, score, renormalise, id_bytes;
    int by_logit;              // the scores need not be formed: experts are chosen by their logits
    float scale;
    uint32_t index_mask;       // the bits of a key that tell the expert
    uint32_t per_each, per_groups;     // reciprocals, 0 for a divisor of 1
    uint32_t wave_words;       // LDS of a wave
    uint32_t part;             // lanes that look through a group together, a power of two
};

enum { kGradLogits = 0, kGradIds, kGradWeights, kGradUp, kGradOut, kRouteGradLists };

struct RouteGradArgs {
    size_t ld, ids_ld, weights_ld, up_ld, out_ld;
    int experts, top_k, score, renormalise, id_bytes;
    float scale;
    uint32_t wave_words;
    int row_held;              // elements of a row in LDS: a multiple of a vector
};

template <int TYPE>
int launch_route(Lists<kRouteLists>& ls, RouteArgs a, const size_t* tokens, int k, hipStream_t stream);
template <int TYPE>
int launch_route_grad(Lists<kRouteGradLists>& ls, RouteGradArgs a, const size_t* tokens, int k, hipStream_t stream);

}  // namespace bagua
