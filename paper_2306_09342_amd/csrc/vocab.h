// What the files of the losses over a vocabulary share.
#pragma once
#include "common.h"
#include "rowwise.h"

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

constexpr int LOSS_CE = 1, LOSS_KD = 2, HAS_LABEL = LOSS_CE, HAS_TEACHER = LOSS_KD;
__device__ __forceinline__ bool in_vocab(int v, int V) { return (unsigned)v < (unsigned)V; }
__device__ __forceinline__ bool teacher_counts(int idx, float logit, int V) { return in_vocab(idx, V) && !(logit == -INFINITY); }
// Entry 0 of a row is its label, entries 1 .. K its teacher's; -1: none.
__device__ __forceinline__ int entry_of(const VocabRows& v, int r, int e) {
    if (e == 0) {
        const int y = v.labels ? v.labels[r] : -1;
        return in_vocab(y, v.V) ? y : -1;
    }
    const int64_t at = (int64_t)r * v.K + e - 1;
    return teacher_counts(v.idx[at], v.logits[at], v.V) ? v.idx[at] : -1;
}
// z[e] = <W_n, x> + b_n for up to four entries n of row r from e0 on, by a wavefront: four rows of W are under way.
template <typename T>
__device__ __forceinline__ void named_logits(const VocabRows& v, const T* x, const T* params, int D, int r, int e0, float* z) {
    constexpr int E = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    int n[4];
    const T* w[4];
    float sum[4] = {};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        n[u] = e0 + u <= v.K ? entry_of(v, r, e0 + u) : -1;
        w[u] = params + (int64_t)max(n[u], 0) * D;
    }
    for (int d = lane * E; d < D; d += 64 * E) {
        f4 a[E / 4];
#pragma unroll
        for (int q = 0; q < E / 4; ++q) a[q] = load4(x + d + 4 * q);
        uint4 b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) b[u] = n[u] >= 0 ? *reinterpret_cast<const uint4*>(w[u] + d) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const T* f = reinterpret_cast<const T*>(&b[u]);
#pragma unroll
            for (int q = 0; q < E / 4; ++q) {
                const f4 c = load4(f + 4 * q);
                sum[u] = fmaf(a[q].x, c.x, sum[u]); sum[u] = fmaf(a[q].y, c.y, sum[u]);
                sum[u] = fmaf(a[q].z, c.z, sum[u]); sum[u] = fmaf(a[q].w, c.w, sum[u]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (e0 + u > v.K) break;
        float s = wave_sum(sum[u]);
        if (n[u] >= 0 && v.bias) s += to_f(params[(int64_t)v.V * D + n[u]]);
        if (lane == 0) z[e0 + u] = s;
    }
}

// The dense part of a row's dz at a logit z: c = {dloss_ce, lse, dloss tau, lse_tau}, {0, infinity} where the row has none (a cotangent of 0
// is not that: 0 exp(NaN) stays NaN).
__device__ __forceinline__ float dense_dz(const float4& c, float z, float inv_tau) {
    float d = 0.f;
    if (c.y != INFINITY) d = c.x * expf(z - c.y);
    if (c.w != INFINITY) d += c.z * expf(z * inv_tau - c.w);
    return d;
}

// The first entry of piece k of a vocabulary and how many it has.  A launch may be for a piece that the plan does not come to, up to 2^12
// pieces of 2^20 entries behind its end: n is 0 there, and v0 nothing.
struct Piece { int v0, n; };
__device__ __forceinline__ Piece piece_of(int k, int width, int V) {
    const int64_t v0 = (int64_t)k * width;
    return {(int)v0, v0 < V ? min(width, V - (int)v0) : 0};
}

// The products (vocab_gemm.hip).  bf16 operands are one part; a float32 one is the sum of three bf16 parts (split3).
struct VocabGemm {
    const VocabPlan* plan;
    const bf16* x;                  // rows that count, a part [Mp, Dp], zeros behind them and beyond D
    const bf16* w;                  // W with rows of ldw for dx: as given, or as wp
    const bf16* wp;                 // W with rows of Dp, zeros beyond D; a part [V, Dp]
    const void* bias;               // [V] or null, bf16, or float32 with three parts
    float* stats;                   // forward: [half tiles][maximum, sum of exp(z - maximum), ...][Mp]; see vocab_logits_kernel
    const float4* coef;             // backward: of every row that counts (dense_dz)
    const int* label;               // of every row that counts, where labels alone are named, or null
    bf16* dz;                       // a part [rows, width] of a piece
    float* acc;                     // dx, 65536 floats per tile and range
    int64_t Mp, dz_part;            // dz_part: elements from a part of dz to the next
    int V, D, Dp, ldw;
    int piece, span;                // piece: its number; span: its width in the forward pass, a multiple of 256
    int losses;                     // whose exponentials without `dual`: LOSS_CE, LOSS_KD or both (tau = 1)
    float inv_tau;
    float* dw_parts;                // dW and db of a range of rows, where the rows are cut into several: as dparams, dw_stride floats each
    int64_t dw_stride;
    int dw_splits;
    double work;                    // of a product over a piece, for the timing of kernel families
};
// x = p[0] + p[1] + p[2] to 2^-25 of |x|; an infinity (also of a value beyond the largest bf16, 3.39e38) or NaN is p[0] alone.
__device__ __forceinline__ void split3(float x, bf16 (&p)[3]) {
    p[0] = from_f<bf16>(x);
    const float r = x - to_f(p[0]);
    const float rest = fabsf(r) < INFINITY ? r : 0.f;
    p[1] = from_f<bf16>(rest);
    p[2] = from_f<bf16>(rest - to_f(p[1]));
}
// T: bf16 (one part) or float (three)
// mid: tiles of 128 instead of 256; blocks: most of the latter
template <typename T> int vocab_logits(hipStream_t s, const VocabGemm& p, bool grad, bool dual, bool mid, int64_t blocks);
template <typename T> int vocab_grads(hipStream_t s, const VocabGemm& p, int64_t dx_blocks, int64_t dw_blocks, void* dparams, bool grad_bf16, bool db);
int vocab_dw_sum(hipStream_t s, const VocabGemm& p, void* dparams, bool grad_bf16, int64_t n);
template <typename T> int vocab_dx_rows(hipStream_t s, const VocabGemm& p, const int* list, const int* place, int M, T* dX);

// Few rows (vocab_few.hip): the statistics of the logits of all rows and the logits that they name; or dz of the whole vocabulary in
// float32, of the rows that count, and the gradients from that.
template <typename T> struct FewRows {
    const VocabPlan* plan;          // null forward
    const T* x;                     // forward X; backward the rows that count, [rows_x, ldx], zeros behind them
    const T* w;                     // [V, D]
    const T* bias;                  // [V] or null
    VocabRows named;                // forward: whose logits go to
    float* zs;                      // [rows][K + 1]
    float* stats;                   // as VocabGemm::stats, of strips of 64 entries: row i at i stat_row, kinds stat_kind apart
    const float4* coef;
    const int* label;
    float* dz;                      // [rows_out, ldz], zeros behind the rows that count and the vocabulary
    bf16* tile_dz;                  // the same in bf16, for the products of tiles, in the plan's width; or null
    float* parts;                   // dx of ranges of the vocabulary, [places][rows][D]: the first of `places` ranges, those of the next turn added, ...
    int64_t stat_row, stat_kind, ldz;
    int V, D, ldx, losses, rows_x, rows, rows_out, blocks_m;    // rows: most that count
    int named_blocks;               // workgroups for the named logits, a multiple of 8
    int range, ranges, col_groups;  // entries per range, a multiple of 32
    int places, first;              // the first range of a turn
    float inv_tau;
};
template <typename T> int few_logits(hipStream_t s, FewRows<T> p, bool grad, bool dual);
template <typename T> int few_grads(hipStream_t s, FewRows<T> p, bool want_dx, void* dparams, bool grad_bf16, bool db);
template <typename T> int few_dx_rows(hipStream_t s, const FewRows<T>& p, const int* place, T* dX);
void few_ranges(int rows, int V, int D, int es, int* range, int* ranges, int* col_groups);

}  // namespace rev
