// What the files of the losses over a vocabulary share.
#pragma once
#include "common.h"

namespace rev {

// What a call's kernels know of its rows.  list[i], i < *count: the rows that count, in order; place[r]: where row r is in it, or -1.
struct VocabRows {
    const int* labels;              // [M] or null
    const int* idx;                 // [M, K] teacher, or null (K = 0)
    const float* logits;
    const int *list, *place, *count;
    int M, V, K, bias;
    float inv_tau;
};

// The dense part of a row's dz at a logit z: c = {dloss_ce, lse, dloss tau, lse_tau}.
__device__ __forceinline__ float dense_dz(const float4& c, float z, float inv_tau) {
    float d = 0.f;
    if (c.x != 0.f) d = c.x * expf(z - c.y);
    if (c.z != 0.f) d += c.z * expf(z * inv_tau - c.w);
    return d;
}

}  // namespace rev
