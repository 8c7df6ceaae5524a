// What the files of the losses over a vocabulary share.
#pragma once
#include "common.h"

namespace rev {

// What follows from the number of rows that count; on the device.
struct VocabPlan {
    int count, rows;                // that many, and rounded up to whole tiles of 256
    int width;                      // of a piece of the vocabulary, a multiple of 256
    int splits, stages;             // ranges of a piece in dx, and stages of 64 in each but the last
};

// What a call's kernels know of its rows.  list[i], i < count: the rows that count, in order; place[r]: where row r is in it, or -1.
struct VocabRows {
    const int* labels;              // [M] or null
    const int* idx;                 // [M, K] teacher, or null (K = 0)
    const float* logits;
    const int *list, *place;
    const VocabPlan* plan;
    int M, V, K, bias;
    float inv_tau;
};

// The dense part of a row's dz at a logit z: c = {dloss_ce, lse, dloss tau, lse_tau}, {0, infinity} where the row has none.
__device__ __forceinline__ float dense_dz(const float4& c, float z, float inv_tau) {
    float d = 0.f;
    if (c.x != 0.f) d = c.x * expf(z - c.y);
    if (c.z != 0.f) d += c.z * expf(z * inv_tau - c.w);
    return d;
}

struct LabelDz { int label; float dz; };         // a row's label, and dz there

constexpr int LOSS_CE = 1, LOSS_KD = 2;
// The bf16 products (vocab_gemm.hip).
struct VocabGemm {
    const VocabPlan* plan;
    const bf16* x;                  // rows that count, [Mp, Dp], zeros behind them and beyond D
    const bf16* w;                  // [V, D]
    const bf16* wp;                 // the same with rows of Dp, zeros beyond D
    const bf16* bias;               // [V] or null
    float* stats;                   // forward: [half tiles][maximum, sum of exp(z - maximum), ...][Mp]; see vocab_logits_kernel
    const float4* coef;             // backward: of every row that counts (dense_dz)
    const LabelDz* label_dz;        // of every row that counts, where labels alone are named, or null
    bf16* dz;                       // [rows, width] of a piece
    float* acc;                     // dx, 65536 floats per tile and range
    int64_t Mp;
    int V, D, Dp, piece;            // piece: its number (backward)
    int losses;                     // whose exponentials without `dual`: LOSS_CE, LOSS_KD or both (tau = 1)
    float inv_tau;
};
int vocab_logits(hipStream_t s, const VocabGemm& p, bool grad, bool dual, int64_t blocks);
int vocab_dx(hipStream_t s, const VocabGemm& p, int64_t blocks);
int vocab_dx_rows(hipStream_t s, const VocabGemm& p, const int* place, int M, bf16* dX);
int vocab_dw(hipStream_t s, const VocabGemm& p, void* dparams, bool grad_bf16, bool db, int64_t blocks);

}  // namespace rev
