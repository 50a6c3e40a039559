// Arguments of the kernels that choose experts and sum their outputs.
#pragma once

#include <stdint.h>

namespace tf {

struct RouteArgs {
    const void* logits;
    const float* bias;
    float* weights;
    int32_t* chosen;
    int64_t T, stride;
    int dtype, E, k, groups, top_groups;
    int lanes_per_group;     // a power of two, at most 64 / groups
    bool sigmoid, group_top2, renormalize;
    float scale;
};

struct CombineArgs {
    const uint16_t *Y, *add;
    const float* weights;
    const int32_t* places;
    uint16_t* out;
    int64_t T, S;
    int k, N;
};

}  // namespace tf
