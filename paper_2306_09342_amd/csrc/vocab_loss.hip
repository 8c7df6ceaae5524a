// Losses over a vocabulary (softmax cross entropy, distillation from a teacher's top logits): entry points, workspace, and the
// kernels that go over rows.  The products with the vocabulary's weights go over it in pieces.
//
// Both losses have the gradient   dz = c0 exp(z - lse) + c1 exp(z / tau - lse_tau)   at every entry of the vocabulary, and
// something to be subtracted at the few entries that a row's label and teacher name.  The products compute the dense part only; the
// logits at the named entries are dot products of their own (gather_row: a row of W per entry), the losses are made of them, and in
// the backward pass the entries of dz that a teacher touches are written again, from float32, behind the dense part
// (sparse_dz_kernel), so that q - p is rounded once and not taken from a rounded q.  p - 1 at a label alone the products see to.
//
// Rows that do not count (no label, no teacher) are left out before anything is multiplied: the others are gathered to the
// front of a copy of X, in their order, with rows of zeros behind them.  Their number stays on the device.
#include "common.h"
#include "rowwise.h"
#include "vocab.h"
#include <algorithm>

namespace rev {

// What bounds a plan: floats of dz, tiles of 256 columns in dx, places for its ranges (0, 0, 0: there are no tiles); products of
// parts that make one; ranges of rows of dW, 0 if it is not wanted.
struct PlanLimits { int64_t dz; int tiles_d, slots, terms, dw; };
struct RowResults { float* p[4]; };

// Pieces of equal widths whose dz fits.  dx has few tiles: its contraction, the piece, is cut into ranges.  A tile or range costs about
// 10 stages besides its own (first loads, and writing and reading 256 KB), and a stage of dx 4/3 of one of dW, which goes along rows.  Alone,
// dx has the number of ranges that keeps the 256 CUs busiest; beside dW, whose tiles fill the CUs that it leaves, the smallest that
// lets its workgroups end before the whole does.  By one wavefront, a number of ranges per lane.
__device__ __forceinline__ void write_plan(int count, int V, const PlanLimits& lim, VocabPlan* __restrict__ plan, int lane) {
    VocabPlan p = {count, (count + 255) / 256 * 256, (V + 255) / 256 * 256, 1, 2};
    if (lim.dz != 0 && count != 0) {                               // (without rows: one piece of zeros for dW)
        const unsigned most = (unsigned)((lim.dz / 256) / (p.rows / 256) / 256 * 256), pieces = (V + most - 1) / most;
        p.width = (int)((V + pieces - 1) / pieces + 255) / 256 * 256;
        const int tiles = p.rows / 256 * lim.tiles_d, pairs = p.width / 128, s = lane + 1;
        const int stages = (pairs + s - 1) / s * 2, terms = lim.terms;
        unsigned cost = ~0u;                                       // in 768ths of a stage of dW
        if (s <= pairs && tiles * s <= lim.slots) {
            cost = (unsigned)((tiles * s + 255) / 256) * (terms * stages + 10) * 1024 + s;
            if (lim.dw) {
                const unsigned tile = terms * ((p.rows / 64 + lim.dw - 1) / lim.dw) + 10;
                const unsigned all = 4 * tiles * (terms * pairs * 2 + 10 * s) + 3 * (p.width / 256) * lim.tiles_d * lim.dw * tile;
                cost = max(cost, all + 384 * tile);                // half a tile of dW idle at the end
            }
        }
        unsigned best = cost;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) best = min(best, (unsigned)__shfl_xor((int)best, o, 64));
        const int who = __ffsll((unsigned long long)__ballot(cost == best)) - 1;
        p.splits = who + 1;
        p.stages = __shfl(stages, who, 64);
    }
    if (lane == 0) *plan = p;
}

// ---------------------------------------------------------------------------------
// which rows count
// ---------------------------------------------------------------------------------
// Whether a row has a label and whether it has a teacher, by a wavefront.
__device__ __forceinline__ int row_flags(const VocabRows& v, int r, int lane) {
    bool any = false;
    for (int k = lane; k < v.K; k += 64) any |= entry_of(v, r, k + 1) >= 0;
    return (__any(any) ? HAS_TEACHER : 0) | (entry_of(v, r, 0) >= 0 ? HAS_LABEL : 0);
}
__global__ __launch_bounds__(256) void row_flags_kernel(VocabRows v, uint8_t* __restrict__ flags) {
    const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= v.M) return;
    const int f = row_flags(v, r, lane);
    if (lane == 0) flags[r] = (uint8_t)f;
}

// list[i] = the i-th row that counts, place[r] = i or -1, zeros in the results of the others, and the plan.  16384 rows at a time, a
// wavefront 16 times 64 of them; all 16 workgroups count, and each writes for 1024 of the rows.  (One workgroup for all: 11 us for 16384
// rows in the place of 7.)
constexpr int SELECT_BLOCKS = 16;
__global__ __launch_bounds__(1024) void select_rows_kernel(const int* __restrict__ labels, const uint8_t* __restrict__ flags, int M, int V,
                                                           int* __restrict__ list, int* __restrict__ place, RowResults zero, PlanLimits lim,
                                                           VocabPlan* __restrict__ plan) {
    __shared__ unsigned long long masks[256];
    __shared__ int before[256], wsum[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int base = 0;
    for (int r0 = 0; r0 < M; r0 += 16384) {
        int y[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int r = r0 + k * 1024 + tid;
            y[k] = r < M ? flags ? flags[r] ? 0 : -1 : labels[r] : -1;
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const unsigned long long m = __ballot(in_vocab(y[k], V));
            if (lane == 0) masks[k * 16 + wave] = m;
        }
        __syncthreads();
        int n = 0, incl = 0;
        if (tid < 256) {
            n = incl = __popcll(masks[tid]);
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int t = __shfl_up(incl, o, 64);
                if (lane >= o) incl += t;
            }
            if (lane == 63) wsum[wave] = incl;
        }
        __syncthreads();
        if (tid < 256) before[tid] = base + incl - n + (wave > 0 ? wsum[0] : 0) + (wave > 1 ? wsum[1] : 0) + (wave > 2 ? wsum[2] : 0);
        base += wsum[0] + wsum[1] + wsum[2] + wsum[3];
        __syncthreads();
        const int k = blockIdx.x, r = r0 + k * 1024 + tid;
        if (r < M) {
            const unsigned long long m = masks[k * 16 + wave];
            const bool on = m >> lane & 1;
            const int i = before[k * 16 + wave] + __popcll(m & ((1ull << lane) - 1));
            place[r] = on ? i : -1;
            if (on) {
                list[i] = r;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (zero.p[q]) zero.p[q][r] = 0.f;
            }
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid < 64) write_plan(base, V, lim, plan, tid);
}

// Four float32 values as three bf16 parts each, `part` elements apart.
__device__ __forceinline__ void store_parts(uint4 u, bf16* out, int64_t part) {
    const unsigned x[4] = {u.x, u.y, u.z, u.w};
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    u16x4 q[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        bf16 p[3];
        split3(__uint_as_float(x[e]), p);
#pragma unroll
        for (int k = 0; k < 3; ++k) q[k][e] = *reinterpret_cast<const uint16_t*>(&p[k]);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<u16x4*>(out + k * part) = q[k];
}

// W as the products over its rows take it: padded with zeros to Dp columns, a multiple of 128, float32 in three parts.
template <typename T>
__global__ __launch_bounds__(256) void lay_out_kernel(const T* __restrict__ w, int V, int D, int Dp, bf16* __restrict__ out) {
    constexpr int E = 16 / sizeof(T);
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x, i = c / (Dp / E);
    if (i >= V) return;
    const int d = (int)(c - i * (Dp / E)) * E;
    uint4 u = make_uint4(0, 0, 0, 0);
    if (d < D) u = *reinterpret_cast<const uint4*>(w + i * D + d);
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint4*>(out + i * Dp + d) = u;
    else store_parts(u, out + i * Dp + d, (int64_t)V * Dp);
}

// ---------------------------------------------------------------------------------
// logits at the entries that a row names
// ---------------------------------------------------------------------------------
// Row i of Xc = row r of X, padded with zeros to Dp columns, all zeros beyond the last row that counts; zs[i][e] = <W_v, x> + b_v for its
// entries, a wavefront of the workgroup per entry at a time; in the backward pass also what the row's dense part is made of.  Without
// a teacher the products find dz at the label by themselves: the label goes with the row, and its logit is not wanted.  P: bf16 parts
// that the copy has, 0: its own type.
struct Cotangents { const float *lse, *lse_tau, *dce, *dkd; };
template <typename T> struct GatherArgs {
    const T* params; const T* X;
    int D, Dp;
    int64_t Mp;
    void* Xc;
    float* zs;
    Cotangents cot;
    float4* coef;
    int* label;
};
template <typename T, int P>
__device__ __forceinline__ void gather_row(const VocabRows& v, const GatherArgs<T>& g, int i, bool live, int r, int flags) {
    constexpr int E = 16 / sizeof(T);
    const T* x = g.X + (int64_t)r * g.D;
    for (int d = threadIdx.x * E; d < g.Dp; d += 256 * E) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (live && d < g.D) u = *reinterpret_cast<const uint4*>(x + d);
        if constexpr (P < 3) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(g.Xc) + (int64_t)i * g.Dp + d) = u;
        else store_parts(u, reinterpret_cast<bf16*>(g.Xc) + (int64_t)i * g.Dp + d, g.Mp * g.Dp);
    }
    if (!live) return;
    if (g.coef && threadIdx.x == 0) {
        float4 c = make_float4(0.f, INFINITY, 0.f, INFINITY);
        if (flags & HAS_LABEL) { c.x = g.cot.dce[r]; c.y = g.cot.lse[r]; }
        if (flags & HAS_TEACHER) { c.z = g.cot.dkd[r] / v.inv_tau; c.w = g.cot.lse_tau[r]; }
        g.coef[i] = c;
    }
    if (g.label) {
        if (threadIdx.x == 0) g.label[i] = entry_of(v, r, 0);
        return;
    }
    for (int e0 = (threadIdx.x >> 6) * 4 + (v.labels ? 0 : 1); e0 <= v.K; e0 += 16) named_logits(v, x, g.params, g.D, r, e0, g.zs + (int64_t)i * (v.K + 1));
}

// One workgroup per row of Xc.  Bound by reading the rows of W, scattered over all of it: 64 entries of 8192 rows of 1024, 1.07 GB,
// in 160 us.
template <typename T, int P>
__global__ __launch_bounds__(256) void gather_kernel(VocabRows v, GatherArgs<T> g, const uint8_t* __restrict__ flags) {
    const int i = blockIdx.x, count = v.plan->count;
    if (P > 0 && i >= v.plan->rows) return;                        // (the float32 products go over all rows)
    const int r = i < count ? v.list[i] : 0;
    gather_row<T, P>(v, g, i, i < count, r, flags ? flags[r] : HAS_LABEL);
}

// The same for up to SELECT_ROWS rows with up to SELECT_ENTRIES labels and teacher entries, without the launches before it: every
// workgroup goes over all of them and finds its own row.  The first one leaves what select_rows_kernel does.
constexpr int SELECT_ROWS = 1024, SELECT_ENTRIES = 8192;
template <typename T, int P>
__global__ __launch_bounds__(256) void select_gather_kernel(VocabRows v, GatherArgs<T> g, uint8_t* __restrict__ flags, int* __restrict__ list,
                                                            int* __restrict__ place, RowResults zero, PlanLimits lim, VocabPlan* __restrict__ plan) {
    __shared__ unsigned long long masks[SELECT_ROWS / 64];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = blockIdx.x;
    const bool first = blockIdx.x == 0;
    if (i >= v.M) {                                                // a row of zeros in any case
        gather_row<T, P>(v, g, i, false, 0, 0);
        return;
    }
    int f[SELECT_ROWS / 256];
#pragma unroll
    for (int q = 0; q < SELECT_ROWS / 256; ++q) {
        const int r = q * 256 + tid;
        f[q] = 0;
        if (r < v.M) {
            if (v.labels && in_vocab(v.labels[r], v.V)) f[q] = HAS_LABEL;
            for (int k = 0; k < v.K; ++k)
                if (teacher_counts(v.idx[(int64_t)r * v.K + k], v.logits[(int64_t)r * v.K + k], v.V)) f[q] |= HAS_TEACHER;
        }
        const unsigned long long m = __ballot(f[q] != 0);
        if (lane == 0) masks[q * 4 + wave] = m;
    }
    __syncthreads();
    int count = 0;
#pragma unroll
    for (int q = 0; q < SELECT_ROWS / 64; ++q) {
        const unsigned long long m = masks[q];
        const int before = count, mine = __popcll(m & ((1ull << lane) - 1));
        count += __popcll(m);
        const bool on = m >> lane & 1;
        if ((q & 3) == wave) {
            const int r = q * 64 + lane, rank = before + mine;
            if (on && rank == i) { found[0] = r; found[1] = f[q >> 2]; }
            if (first && r < v.M) {
                flags[r] = (uint8_t)f[q >> 2];
                place[r] = on ? rank : -1;
                if (on) {
                    list[rank] = r;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (zero.p[k]) zero.p[k][r] = 0.f;
                }
            }
        }
    }
    __syncthreads();
    if (first && wave == 0) write_plan(count, v.V, lim, plan, lane);
    const bool live = i < count;
    gather_row<T, P>(v, g, i, live, live ? found[0] : 0, live ? found[1] : 0);
}

// The teacher's probabilities of a row, entry e = 1 + lane + 64 q in p[q] (0: none), and log p_k = t_k - log_norm, t_k = (its logit - the
// largest) / tau: the difference first, since a lowest value has no room for a factor or a logarithm.
struct Teacher { float p[4], t[4], log_norm; };
__device__ __forceinline__ Teacher teacher_of(const VocabRows& v, int r, int lane) {
    Teacher a;
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int k = lane + 64 * q;
        a.t[q] = k < v.K && entry_of(v, r, k + 1) >= 0 ? v.logits[(int64_t)r * v.K + k] : -INFINITY;
        m = fmaxf(m, a.t[q]);
    }
    m = wave_max(m);
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (a.t[q] != -INFINITY) a.t[q] = (a.t[q] - m) * v.inv_tau;
        a.p[q] = expf(a.t[q]);
        s += a.p[q];
    }
    s = wave_sum(s);
    a.log_norm = logf(s);
#pragma unroll
    for (int q = 0; q < 4; ++q) a.p[q] = a.p[q] / s;
    return a;
}

// ---------------------------------------------------------------------------------
// losses
// ---------------------------------------------------------------------------------
// The divergence of a row from its teacher and its lse_tau, by a wavefront; top + log_s / inv_tau is the latter times tau.
__device__ __forceinline__ void teacher_loss(const VocabRows& v, int r, const float* z, float top, float log_s, int lane, float* kd, float* lse_tau) {
    const Teacher t = teacher_of(v, r, lane);
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (lane + 64 * q < v.K && t.p[q] != 0.f) sum += t.p[q] * ((t.t[q] - t.log_norm) - ((z[1 + lane + 64 * q] - top) * v.inv_tau - log_s));
    *kd = wave_sum(sum) / (v.inv_tau * v.inv_tau);
    *lse_tau = top * v.inv_tau + log_s;
}

// What a row's statistics come to, by a wavefront; z: its named logits.
__device__ __forceinline__ void row_losses(const VocabRows& v, int r, int flags, const float* z, float top, float log0, float log1, int lane,
                                           const RowResults& out) {
    float *loss_ce = out.p[0], *lse = out.p[1], *loss_kd = out.p[2], *lse_tau = out.p[3];
    const bool has = loss_ce && (flags & HAS_LABEL);
    float kd = 0.f, l1 = 0.f;
    if (loss_kd && (flags & HAS_TEACHER)) teacher_loss(v, r, z, top, log1, lane, &kd, &l1);
    if (lane == 0) {
        if (loss_ce) loss_ce[r] = has ? log0 + (top - z[0]) : 0.f;
        lse[r] = has ? top + log0 : 0.f;
        if (loss_kd) { loss_kd[r] = kd; lse_tau[r] = l1; }
    }
}

// The statistics of a row joined, and its losses, a workgroup per row: for few rows, those that do not count among them.  stats: see
// FewRows and losses_kernel.
template <int N>
__global__ __launch_bounds__(256) void few_losses_kernel(VocabRows v, const float* __restrict__ stats, int strips, int64_t stat_row, int64_t stat_kind,
                                                         const float* __restrict__ zs, RowResults out) {
    __shared__ float sh[3][4];
    const int r = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const float rate0 = N == 2 && !out.p[0] ? v.inv_tau : 1.f;
    const float* at = stats + r * stat_row;
    float m = -INFINITY, s0 = 0.f, s1 = 0.f;
    for (int p0 = threadIdx.x; p0 < strips; p0 += 1024) {
        float a[4][N];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int k = 0; k < N; ++k) a[u][k] = p0 + 256 * u < strips ? at[k * stat_kind + p0 + 256 * u] : k ? 0.f : -INFINITY;
        const float top = fmaxf(fmaxf(fmaxf(a[0][0], a[1][0]), fmaxf(a[2][0], a[3][0])), m);
        const float ref = top == -INFINITY ? 0.f : top;        // (sums are 0 or NaN there)
        s0 *= expf((m - ref) * rate0);
        if (N == 3) s1 *= expf((m - ref) * v.inv_tau);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            s0 += a[u][1] * expf((a[u][0] - ref) * rate0);
            if (N == 3) s1 += a[u][N - 1] * expf((a[u][0] - ref) * v.inv_tau);
        }
        m = top;
    }
    const float wm = wave_max(m), d = wm == -INFINITY ? 0.f : m - wm;
    s0 = wave_sum(s0 * expf(d * rate0));
    if (N == 3) s1 = wave_sum(s1 * expf(d * v.inv_tau));
    if (lane == 0) { sh[0][w] = wm; sh[1][w] = s0; sh[2][w] = s1; }
    __syncthreads();
    if (w) return;
    const float top = fmaxf(fmaxf(sh[0][0], sh[0][1]), fmaxf(sh[0][2], sh[0][3])), ref = top == -INFINITY ? 0.f : top;
    float t0 = 0.f, t1 = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        t0 += sh[1][k] * expf((sh[0][k] - ref) * rate0);
        if (N == 3) t1 += sh[2][k] * expf((sh[0][k] - ref) * v.inv_tau);
    }
    row_losses(v, r, row_flags(v, r, lane), zs + (int64_t)r * (v.K + 1), top, logf(t0), logf(N == 3 ? t1 : t0), lane, out);
}

// The same for 16 rows per workgroup.  stats: [strips][N][Mp] = maximum m of a strip, sums of exp(z - m) and exp((z - m) / tau), the
// second with N = 3 only, the first in its place if only the teacher's loss is wanted.  64 threads per row over the strips, then a
// wavefront per row.  Where the vocabulary comes in several pieces, `carry` is one more strip, of the pieces before, and what a piece
// that is not the last leaves in the place of losses.
constexpr int JOIN_ROWS = 16;
template <int N>
__global__ __launch_bounds__(1024) void losses_kernel(VocabRows v, const float* __restrict__ stats, int strips, int64_t Mp, const float* __restrict__ zs,
                                                      const uint8_t* __restrict__ flags, RowResults out, float* __restrict__ carry, bool first_piece,
                                                      bool last_piece) {
    __shared__ float sh[3][JOIN_ROWS][65];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = threadIdx.x & (JOIN_ROWS - 1), part = threadIdx.x / JOIN_ROWS;
    const int i0 = blockIdx.x * JOIN_ROWS, count = v.plan->count;
    if (i0 >= count) return;
    const float rate0 = N == 2 && !out.p[0] ? v.inv_tau : 1.f;
    float m = -INFINITY, s0 = 0.f, s1 = 0.f;
    if (i0 + row < count) {
        const float* at = stats + i0 + row;
        if (part == 0 && !first_piece) {
            m = carry[i0 + row];
            s0 = carry[Mp + i0 + row];
            if (N == 3) s1 = carry[2 * Mp + i0 + row];
        }
        for (int p0 = part; p0 < strips; p0 += 256) {
            float a[4][N];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int k = 0; k < N; ++k) a[u][k] = p0 + 64 * u < strips ? at[((int64_t)(p0 + 64 * u) * N + k) * Mp] : k ? 0.f : -INFINITY;
            const float top = fmaxf(fmaxf(fmaxf(a[0][0], a[1][0]), fmaxf(a[2][0], a[3][0])), m);
            const float ref = top == -INFINITY ? 0.f : top;        // (sums are 0 or NaN there)
            s0 *= expf((m - ref) * rate0);
            if (N == 3) s1 *= expf((m - ref) * v.inv_tau);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                s0 += a[u][1] * expf((a[u][0] - ref) * rate0);
                if (N == 3) s1 += a[u][N - 1] * expf((a[u][0] - ref) * v.inv_tau);
            }
            m = top;
        }
    }
    sh[0][row][part] = m; sh[1][row][part] = s0; sh[2][row][part] = s1;
    __syncthreads();
    const int i = i0 + w;
    if (i >= count) return;
    m = sh[0][w][lane];
    const float top = wave_max(m), d = top == -INFINITY ? 0.f : m - top;
    s0 = wave_sum(sh[1][w][lane] * expf(d * rate0));
    if (N == 3) s1 = wave_sum(sh[2][w][lane] * expf(d * v.inv_tau));
    if (!last_piece) {
        if (lane == 0) {
            carry[i] = top;
            carry[Mp + i] = s0;
            if (N == 3) carry[2 * Mp + i] = s1;
        }
        return;
    }
    const int r = v.list[i];
    row_losses(v, r, flags ? flags[r] : HAS_LABEL, zs + (int64_t)i * (v.K + 1), top, logf(s0), logf(N == 3 ? s1 : s0), lane, out);
}

// ---------------------------------------------------------------------------------
// gradient of the logits
// ---------------------------------------------------------------------------------
// dz at the entries of a piece that a row names, again.  One wavefront per row; an entry that is named several times is written by
// the first of them.  The piece: n entries from v0, or with n = 0 number v0 of the plan.
template <typename T, int P>
__global__ __launch_bounds__(256) void sparse_dz_kernel(VocabRows v, const float* __restrict__ zs, const float4* __restrict__ coef, int v0, int n,
                                                        T* __restrict__ dz, int64_t ld, int64_t part) {
    __shared__ int names[4][257];
    __shared__ float probs[4][257];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = blockIdx.x * 4 + w;
    const bool live = i < v.plan->count;
    if (n == 0) {
        ld = v.plan->width;
        const Piece of = piece_of(v0, (int)ld, v.V);
        v0 = of.v0;
        n = of.n;
        if (n == 0) return;
    }
    int mine[5];
    if (live) {
        const int r = v.list[i];
        const float4 c = coef[i];
#pragma unroll
        for (int q = 0; q < 5; ++q) {
            const int e = lane + 64 * q;
            mine[q] = e <= v.K ? entry_of(v, r, e) : -1;
            if (e <= v.K) names[w][e] = mine[q];
        }
        if (v.K > 0) {
            const Teacher t = teacher_of(v, r, lane);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (lane + 64 * q < v.K) probs[w][1 + lane + 64 * q] = c.z * t.p[q];
        }
        if (lane == 0) probs[w][0] = c.x;
    }
    __syncthreads();
    if (!live) return;
    const float4 c = coef[i];
#pragma unroll
    for (int q = 0; q < 5; ++q) {
        const int e = lane + 64 * q, name = mine[q];
        if (name < v0 || name >= v0 + n) continue;
        float less = 0.f;
        bool first = true;
        for (int k = 0; k <= v.K; ++k)
            if (names[w][k] == name) {
                if (k < e) first = false;
                less += probs[w][k];
            }
        if (!first) continue;
        const float d = dense_dz(c, zs[(int64_t)i * (v.K + 1) + e], v.inv_tau) - less;
        T* at = dz + (int64_t)i * ld + name - v0;
        if constexpr (P == 3) {
            bf16 q[3];
            split3(d, q);
            for (int k = 0; k < 3; ++k) at[k * part] = q[k];
        } else {
            *at = from_f<T>(d);
        }
    }
}

// ---------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------
static int vocab_check(const rev_vocab_cfg* c) {
    if (!c) { set_error("vocab cfg is null"); return REV_EINVAL; }
    if (c->rows <= 0 || c->d_model <= 0 || c->vocab <= 0) { set_error("vocab cfg: every size must be positive"); return REV_EINVAL; }
    if (c->mode != REV_MODE_FP32 && c->mode != REV_MODE_BF16) { set_error("vocab cfg: unknown mode"); return REV_EINVAL; }
    if (c->grad_mode != REV_MODE_FP32 && (c->grad_mode != REV_MODE_BF16 || c->mode != REV_MODE_BF16)) {
        set_error("vocab cfg: grad_mode must be REV_MODE_FP32, or REV_MODE_BF16 in bf16 mode"); return REV_EINVAL;
    }
    if (c->d_model % 8 != 0 || c->d_model > 8192) { set_error("vocab cfg: d_model must be a multiple of 8, at most 8192"); return REV_EINVAL; }
    if (c->rows > (1 << 20)) { set_error("vocab cfg: rows must be <= 2^20"); return REV_EINVAL; }
    if (c->vocab > (1 << 20)) { set_error("vocab cfg: vocab must be <= 2^20"); return REV_EINVAL; }
    if (c->bias != 0 && c->bias != 1) { set_error("vocab cfg: bias must be 0 or 1"); return REV_EINVAL; }
    if (c->top_k < 0 || c->top_k > 256) { set_error("vocab cfg: top_k must be between 0 and 256"); return REV_EINVAL; }
    if (!(c->temperature >= 1.f / 1024 && c->temperature <= 1024.f)) {
        set_error("vocab cfg: temperature must be between 1/1024 and 1024"); return REV_EINVAL;
    }
    return REV_OK;
}

// Where the kernels of few rows (vocab_few.hip) take the place of the products in tiles; blocks: of 64 rows and 64 entries.  us, tiles / few
// rows, D = 768 unless said.
// Forward, bf16: 64 rows, V = 50265: 35 / 26; 96: 33 / 36; V = 10007, 128 rows (314 blocks): 21 / 15; 256 (628): 22 / 19; 640, V = 5000 (790): 22 /
// 21; 300, V = 10007, D = 2048 (785): 35 / 38; 256, V = 15000 (940): 23 / 23; 1024, V = 5000, D = 256 (1264): 18 / 21.  float32: 128 rows, V = 50265: 182 /
// 119; 256, V = 10007: 79 / 66; 640, V = 5000: 75 / 69; 1024, V = 4000 (1008): 74 / 77; 200, V = 20000 (1252): 94 / 102.
static int64_t few_blocks(int64_t M, int64_t V) { return (M + 63) / 64 * ((V + 63) / 64); }
static bool few_forward(const rev_vocab_cfg& c) {
    return c.rows <= (c.mode == REV_MODE_BF16 ? 64 : 128) || few_blocks(c.rows, c.vocab) <= 800;
}
// Backward, where their time goes with the number of products (rows x D x V, in millions) and the tiles' does not.  bf16: 1 row, V = 50265 (39): 81 /
// 76; 64, V = 1000 (49): 28 / 25; 16, V = 10007 (123): 43 / 37; 64, V = 5000, D = 512 (164): 43 / 36; 64, V = 4000 (197): 39 / 37; 48, V = 6000 (221): 35 /
// 46; 8, V = 50265 (309): 81 / 80; 8, V = 50265, D = 1024 (412): 91 / 115; more than 64 rows: 128, V = 1000 (98): 28 / 33.  float32, whose tiles need W in
// parts first: 16, V = 1000 (12): 89 / 25; 64, V = 50265 (2470): 362 / 247; 64, V = 32000, D = 2048 (4194): 568 / 379; 128, V = 10007, D = 384 (492): 95 /
// 80; 640, V = 1000 (492): 137 / 110; 100, V = 10007, D = 512 (512): 103 / 106; 500, V = 5000, D = 256 (640): 108 / 116; 128, V = 10007 (984): 125 / 133.
static bool few_backward(const rev_vocab_cfg& c) {
    const int64_t products = (int64_t)c.rows * c.d_model * c.vocab;
    if (c.mode == REV_MODE_BF16) return c.rows <= 64 && products <= 170000000;
    return c.rows <= 64 || (c.rows <= 768 && products <= 500000000);
}
// dz alone by them, the gradients in tiles (bf16).  V = 1000, 128 rows: 35 / 29, 512: 45 / 39; V = 10007, 128 rows: 54 / 53.
static bool few_for_dz(const rev_vocab_cfg& c) { return c.mode == REV_MODE_BF16 && !few_backward(c) && few_blocks(c.rows, c.vocab) <= 160; }
// Tiles of 128 in the place of 256 for the logits, where the latter leave half of the CUs without one.  Forward, us, 256 / 128: 256 rows, V =
// 10007 (40 tiles of 256): 29 / 23; 512, D = 1280 (80): 41 / 35; 8192, V = 1000 (128): 44 / 37; 777, D = 256, V = 10007 (160): 24 / 25; 200, V =
// 50265 (197): 38 / 51.  float32: 512, D = 1280 (80): 152 / 133; 1024, V = 10007 (160): 110 / 144.
static bool mid_tiles_pay(int64_t M, int64_t V) { return (M + 255) / 256 * ((V + 255) / 256) <= 128; }

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// dz of a piece: 512 MB, or 256 entries of all rows if that is more.  Loss and gradients of 8192 x 1024 to 131072 entries with 128, 256, 512
// and 1024 MB: 8.31, 7.46, 7.34, 7.28 ms; 4096 x 768 to 50265 1.54, 1.50, 1.44, 1.45.  Fewer pieces have fuller rounds of tiles
// and fewer passes over dx; that 256 MB would stay in the memory-side cache does not make up for them.
constexpr int64_t VOCAB_DZ_BYTES = 512 << 20;
// the statistics of a piece in the forward pass, three per 128 entries of a row, or those of 256 entries if that is more
constexpr int64_t VOCAB_STATS_BYTES = 256 << 20;
// dW of ranges of rows, all together
constexpr int64_t VOCAB_DW_BYTES = 256 << 20;
// dx of few rows' ranges, all together; where there are more, they take turns at these places (a turn is thousands of workgroups then).
// Backward in ms, a place for each / turns: 64 float32 rows of 4096 to 131072 entries (537 MB) 2.63 / 2.69, 32 of 8192 to 262144 (1.1 GB) 5.99 / 6.04.
constexpr int64_t VOCAB_FEW_DX_BYTES = 256 << 20;
struct VocabLayout {
    int64_t plan, flags, place, list, coef, label, zs, stats, carry, xc, w, dz, acc, dzf, parts_dx, dw_parts, total;
    int64_t Mp, ldz;                 // ldz: of dz in float32
    bool few_f, few_b, few_dz, mid;  // few rows: forward, backward, dz alone; tiles of 128
    int parts;                       // bf16 parts of an operand of the products of tiles
    int Dp, strips, pieces;          // strips of a piece forward; pieces: most that a plan may have backward
    int span;                        // width of a piece forward (tiles of 256)
    int range, ranges, col_groups;   // few_ranges
    int places;                      // of ranges of dx
    int dw_splits;
    int64_t dw_stride;
    PlanLimits lim;
};
static VocabLayout vocab_layout(const rev_vocab_cfg& c) {
    VocabLayout L = {};
    const int64_t M = c.rows, D = c.d_model, V = c.vocab;
    L.few_f = few_forward(c);
    L.few_b = few_backward(c);
    L.parts = c.mode == REV_MODE_BF16 ? 1 : 3;
    const int es = L.parts == 1 ? 2 : 4;
    L.few_dz = few_for_dz(c);
    L.Dp = (int)up(D, 128);
    L.Mp = up(M, 256);
    L.mid = mid_tiles_pay(M, V);
    const bool large = !L.few_f && !L.mid;
    L.span = (int)(large ? std::min(std::max(VOCAB_STATS_BYTES * 128 / 12 / L.Mp / 256 * 256, (int64_t)256), up(V, 256)) : up(V, 256));
    L.strips = (int)(L.few_f ? (V + 63) / 64 : L.mid ? (V + 127) / 128 * 2 : L.span / 128);
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t o = at; at += up(bytes, 256); return o; };
    L.plan = take(sizeof(VocabPlan));
    L.flags = take(M);
    L.place = take(4 * M);
    L.list = take(4 * M);
    L.coef = take(16 * L.Mp);
    L.label = take(4 * L.Mp);
    L.zs = take(4 * M * (c.top_k + 1));
    L.stats = take(12 * (L.few_f ? M : L.Mp) * L.strips);
    if (large) L.carry = take(12 * L.Mp);
    // the rows' copy: their own type, or parts of it, in the place of the larger
    L.xc = take(L.Mp * L.Dp * (L.parts == 1 ? 2 : 6));
    if (!L.few_f || !L.few_b) L.w = L.Dp != D || L.parts > 1 ? take(2 * L.parts * V * L.Dp) : 0;
    if (!L.few_b) {
        const int64_t all = L.Mp * up(V, 256);
        L.lim.dz = L.few_dz ? all : std::min(std::max(VOCAB_DZ_BYTES / 2 / L.parts / 256 * 256, L.Mp * 256), all);
        L.lim.tiles_d = (int)((D + 255) / 256);
        L.lim.terms = L.parts == 1 ? 1 : 6;
        // places for the ranges of dx: two rounds of tiles, but no more than there can be (write_plan: at most 64, and pairs of stages)
        const int64_t tiles_x = L.Mp / 256 * L.lim.tiles_d;
        L.lim.slots = (int)std::max(tiles_x, std::min<int64_t>(512, tiles_x * std::min<int64_t>(64, up(V, 256) / 128)));
        const int64_t least = L.lim.dz / L.Mp / 256 * 256;
        L.pieces = (int)((V + least - 1) / least);
        L.dz = take(2 * L.parts * L.lim.dz);
        L.acc = take((int64_t)L.lim.slots * 65536 * 4);
        // dW has as many tiles as the narrowest piece: where these leave CUs without one, ranges of at least 8 stages (6 times 4)
        L.dw_stride = up(V * D + V, 4);
        const int64_t tiles_w = std::min(std::max<int64_t>(least, 256), up(V, 256)) / 256 * L.lim.tiles_d;
        L.dw_splits = (int)std::max<int64_t>(1, std::min({256 / tiles_w, L.Mp / 64 / (L.parts == 1 ? 8 : 4), VOCAB_DW_BYTES / 4 / L.dw_stride}));
        if (L.dw_splits > 1) L.dw_parts = take(4 * L.dw_splits * L.dw_stride);
    } else {
        L.ldz = up(V, 4);
        few_ranges(c.rows, c.vocab, c.d_model, es, &L.range, &L.ranges, &L.col_groups);
        L.dzf = take(4 * M * L.ldz);
        L.places = (int)std::min<int64_t>(L.ranges, VOCAB_FEW_DX_BYTES / 4 / (M * D));
        L.parts_dx = take(4 * (int64_t)L.places * M * D);
    }
    L.total = at;
    return L;
}

#define RC(expr) do { int _rc = (expr); if (_rc != REV_OK) return _rc; } while (0)
#define LAUNCH(kern, grid, block, ...) do { hipLaunchKernelGGL(kern, grid, block, 0, s, __VA_ARGS__); REV_HIP(hipGetLastError()); } while (0)
static dim3 blocks_of(int64_t n, int per) { return dim3((unsigned)((n + per - 1) / per)); }

template <typename T>
struct VocabRunner {
    static constexpr int kParts = sizeof(T) == 2 ? 1 : 3;
    rev_vocab_cfg c;
    VocabLayout L;
    char* ws;
    const T* params;
    hipStream_t s;
    VocabRows v;
    int M, D, V;

    VocabRunner(const rev_vocab_cfg& cfg, const void* p, void* w, hipStream_t st, const int* labels, const int* idx, const float* logits)
        : c(cfg), L(vocab_layout(cfg)), ws((char*)w), params((const T*)p), s(st) {
        M = c.rows; D = c.d_model; V = c.vocab;
        v = {labels, idx, logits, at<int>(L.list), at<int>(L.place), at<VocabPlan>(L.plan), M, V, idx ? c.top_k : 0, c.bias,
             idx ? 1.f / c.temperature : 1.f};
    }
    template <typename U> U* at(int64_t off) const { return static_cast<U*>(static_cast<void*>(ws + off)); }
    const uint8_t* flags() const { return v.idx ? at<uint8_t>(L.flags) : nullptr; }
    const T* bias() const { return c.bias ? params + (int64_t)V * D : nullptr; }
    int losses() const { return (v.labels ? LOSS_CE : 0) | (v.idx ? LOSS_KD : 0); }
    bool dual() const { return losses() == (LOSS_CE | LOSS_KD) && c.temperature != 1.f; }

    // the rows that count, their logits at named entries, and in the backward pass (cot.lse) what their dense parts are made of
    template <int P> int prepare(const void* X, const RowResults& zero, const Cotangents& cot, bool dw = false) {
        PlanLimits lim = L.lim;
        lim.dw = dw ? L.dw_splits : 0;
        ProfScope ps(K_CONVERT, s, (double)M * D * 2 * sizeof(T));
        const GatherArgs<T> g = {params, (const T*)X, D, L.Dp, L.Mp, at<void>(L.xc), at<float>(L.zs), cot, cot.lse ? at<float4>(L.coef) : nullptr,
                                 cot.lse && !v.idx ? at<int>(L.label) : nullptr};
        const dim3 rows((unsigned)L.Mp), block(256);
        if (M <= SELECT_ROWS && (int64_t)M * (v.K + 1) <= SELECT_ENTRIES) {
            LAUNCH((select_gather_kernel<T, P>), rows, block, v, g, at<uint8_t>(L.flags), at<int>(L.list), at<int>(L.place), zero, lim, at<VocabPlan>(L.plan));
            return REV_OK;
        }
        if (v.idx) LAUNCH(row_flags_kernel, blocks_of(M, 4), dim3(256), v, at<uint8_t>(L.flags));
        LAUNCH(select_rows_kernel, dim3(SELECT_BLOCKS), dim3(1024), v.labels, flags(), M, V, at<int>(L.list), at<int>(L.place), zero, lim, at<VocabPlan>(L.plan));
        LAUNCH((gather_kernel<T, P>), rows, block, v, g, flags());
        return REV_OK;
    }
    int join(const RowResults& out, int piece = 0, int pieces = 1) {
        ProfScope ps(K_REDUCE, s, 12.0 * M * L.strips);
        const int64_t kind = L.strips;
        const int strips = L.few_f || L.mid ? L.strips : (int)((std::min<int64_t>(L.span, V - (int64_t)piece * L.span) + 255) / 256 * 2);
        float* carry = at<float>(L.carry);
        if (L.few_f && dual()) LAUNCH(few_losses_kernel<3>, dim3(M), dim3(256), v, at<float>(L.stats), strips, 3 * kind, kind, at<float>(L.zs), out);
        else if (L.few_f) LAUNCH(few_losses_kernel<2>, dim3(M), dim3(256), v, at<float>(L.stats), strips, 3 * kind, kind, at<float>(L.zs), out);
        else if (dual()) LAUNCH(losses_kernel<3>, blocks_of(M, JOIN_ROWS), dim3(1024), v, at<float>(L.stats), strips, L.Mp, at<float>(L.zs), flags(), out, carry,
                                piece == 0, piece + 1 == pieces);
        else LAUNCH(losses_kernel<2>, blocks_of(M, JOIN_ROWS), dim3(1024), v, at<float>(L.stats), strips, L.Mp, at<float>(L.zs), flags(), out, carry, piece == 0,
                    piece + 1 == pieces);
        return REV_OK;
    }
    template <typename U, int P> int sparse_dz(int v0, int n, U* dz, int64_t ld, int64_t part) {
        ProfScope ps(K_CONVERT, s, 4.0 * M * (v.K + 1));
        LAUNCH((sparse_dz_kernel<U, P>), blocks_of(M, 4), dim3(256), v, at<float>(L.zs), at<float4>(L.coef), v0, n, dz, ld, part);
        return REV_OK;
    }
    FewRows<T> few_args() {
        FewRows<T> f = {};
        f.plan = v.plan; f.x = at<T>(L.xc); f.w = params; f.bias = bias(); f.stats = at<float>(L.stats); f.coef = at<float4>(L.coef);
        f.label = v.idx ? nullptr : at<int>(L.label); f.dz = at<float>(L.dzf); f.parts = at<float>(L.parts_dx);
        f.stat_kind = L.strips; f.stat_row = 3 * f.stat_kind; f.ldz = L.ldz;
        f.V = V; f.D = D; f.ldx = L.Dp; f.losses = losses(); f.rows_x = (int)L.Mp; f.rows = f.rows_out = M;
        f.range = L.range; f.ranges = L.ranges; f.places = L.places; f.col_groups = L.col_groups; f.inv_tau = v.inv_tau;
        return f;
    }

    // ---- products of bf16 parts ----
    int gemm_args(VocabGemm* g) {
        *g = {};
        g->plan = v.plan; g->x = at<bf16>(L.xc); g->bias = bias(); g->label = v.idx ? nullptr : at<int>(L.label);
        g->stats = at<float>(L.stats); g->coef = at<float4>(L.coef); g->dz = at<bf16>(L.dz); g->acc = at<float>(L.acc);
        g->Mp = L.Mp; g->dz_part = L.lim.dz; g->V = V; g->D = D; g->Dp = L.Dp; g->losses = losses(); g->inv_tau = v.inv_tau;
        g->w = g->wp = (const bf16*)params;
        g->ldw = D;
        if (L.Dp != D || kParts > 1) {
            ProfScope ps(K_CONVERT, s, (sizeof(T) + 2.0 * kParts) * V * L.Dp);
            LAUNCH(lay_out_kernel<T>, blocks_of((int64_t)V * L.Dp * sizeof(T) / 16, 256), dim3(256), params, V, D, L.Dp, at<bf16>(L.w));
            g->wp = at<bf16>(L.w);
            if (kParts > 1) { g->w = g->wp; g->ldw = L.Dp; }
        }
        return REV_OK;
    }
    int forward_parts(const RowResults& out) {
        VocabGemm g;
        RC(gemm_args(&g));
        const int pieces = (V + L.span - 1) / L.span;
        g.span = L.span;
        for (int k = 0; k < pieces; ++k) {
            g.piece = k;
            g.work = 2.0 * M * D * std::min<int64_t>(L.span, V - (int64_t)k * L.span);
            RC(vocab_logits<T>(s, g, false, dual(), L.mid, L.Mp / 256 * (L.span / 256)));
            RC(join(out, k, pieces));
        }
        return REV_OK;
    }
    int backward_parts(T* dX, void* dparams) {
        VocabGemm g;
        RC(gemm_args(&g));
        FewRows<T> f = few_args();
        f.tile_dz = at<bf16>(L.dz);
        g.dw_parts = at<float>(L.dw_parts); g.dw_stride = L.dw_stride; g.dw_splits = L.dw_splits;
        g.work = 2.0 * M * D * V / L.pieces;                       // (how many of them there are is known to the device)
        f.rows_out = (int)up(M, 128);                              // dW goes over whole 128 rows
        for (int k = 0; k < L.pieces; ++k) {
            // tiles of 256 entries that piece k may have: there is a piece k only if a piece is at most a k+1-th of the vocabulary
            const int64_t tiles_v = ((V + k) / (k + 1) + 255) / 256;
            g.piece = k;
            if (L.few_dz) RC(few_logits<T>(s, f, true, false));
            else RC(vocab_logits<T>(s, g, true, dual(), L.mid, std::min(L.Mp / 256 * tiles_v, std::max(L.lim.dz / 65536, tiles_v))));
            if (v.idx) RC((sparse_dz<bf16, kParts>(k, 0, at<bf16>(L.dz), 0, L.lim.dz)));
            RC(vocab_grads<T>(s, g, dX ? up(L.lim.slots, 8) : 0, dparams ? tiles_v * (L.lim.tiles_d + (c.bias ? 1 : 0)) * L.dw_splits : 0, dparams,
                              c.grad_mode == REV_MODE_BF16, c.bias));
        }
        if (dparams && L.dw_splits > 1) RC(vocab_dw_sum(s, g, dparams, c.grad_mode == REV_MODE_BF16, (int64_t)V * D + (c.bias ? V : 0)));
        return dX ? vocab_dx_rows<T>(s, g, v.list, v.place, M, dX) : REV_OK;
    }

    // ---- few rows ----
    int backward_few(T* dX, void* dparams) {
        const FewRows<T> f = few_args();
        RC(few_logits<T>(s, f, true, false));
        if (v.idx) RC((sparse_dz<float, 0>(0, V, f.dz, f.ldz, 0)));
        RC(few_grads<T>(s, f, dX != nullptr, dparams, c.grad_mode == REV_MODE_BF16, c.bias));
        return dX ? few_dx_rows<T>(s, f, v.place, dX) : REV_OK;
    }

    int forward(const void* X, const RowResults& out) {
        if (!L.few_f) {
            RC(prepare<kParts>(X, out, Cotangents{}));
            return forward_parts(out);
        }
        FewRows<T> f = few_args();
        f.plan = nullptr; f.x = (const T*)X; f.ldx = D; f.rows_x = M; f.named = v; f.zs = at<float>(L.zs);
        RC(few_logits<T>(s, f, false, dual()));
        return join(out);
    }
    int backward(const void* X, const Cotangents& cot, void* dX, void* dparams) {
        if (!L.few_b) {
            RC(prepare<kParts>(X, RowResults{}, cot, dparams != nullptr));
            return backward_parts((T*)dX, dparams);
        }
        RC(prepare<0>(X, RowResults{}, cot));
        return backward_few((T*)dX, dparams);
    }
};

}  // namespace rev

using namespace rev;

extern "C" {

int rev_vocab_check_cfg(const rev_vocab_cfg* cfg) { return vocab_check(cfg); }

int64_t rev_vocab_param_count(const rev_vocab_cfg* cfg) {
    if (vocab_check(cfg) != REV_OK) return REV_EINVAL;
    return (int64_t)cfg->vocab * cfg->d_model + (cfg->bias ? cfg->vocab : 0);
}

int64_t rev_vocab_workspace_bytes(const rev_vocab_cfg* cfg) {
    if (vocab_check(cfg) != REV_OK) return REV_EINVAL;
    return vocab_layout(*cfg).total;
}

// `wide` buffers are read and written 16 bytes at a time
static int vocab_common(const rev_vocab_cfg* cfg, const void* params, const void* X, uintptr_t wide, uintptr_t narrow, const void* ws, int64_t ws_bytes) {
    RC(vocab_check(cfg));
    if (!params || !X) { set_error("a required pointer is null"); return REV_EINVAL; }
    if ((((uintptr_t)params | (uintptr_t)X | wide) & 15) != 0) { set_error("params, X, dX and dparams must be 16-byte aligned"); return REV_EINVAL; }
    if ((narrow & 3) != 0) { set_error("every buffer must be 4-byte aligned"); return REV_EINVAL; }
    if (!ws) { set_error("workspace is null"); return REV_EINVAL; }
    if (((uintptr_t)ws & 255) != 0) { set_error("workspace must be 256-byte aligned"); return REV_EINVAL; }
    const int64_t need = vocab_layout(*cfg).total;
    if (ws_bytes < need) {
        set_error("workspace too small: need " + std::to_string(need) + " bytes, got " + std::to_string(ws_bytes));
        return REV_EWORKSPACE;
    }
    return REV_OK;
}
static int vocab_forward(const rev_vocab_cfg* cfg, const void* params, const void* X, const int* labels, const int* idx, const float* logits,
                         float* loss_ce, float* loss_kd, float* lse, void* ws, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    const RowResults out = {{loss_ce, lse, loss_kd, idx ? lse + cfg->rows : nullptr}};
    if (cfg->mode == REV_MODE_BF16) return VocabRunner<bf16>(*cfg, params, ws, s, labels, idx, logits).forward(X, out);
    return VocabRunner<float>(*cfg, params, ws, s, labels, idx, logits).forward(X, out);
}
static int vocab_backward(const rev_vocab_cfg* cfg, const void* params, const void* X, const int* labels, const int* idx, const float* logits,
                          const float* lse, const float* dce, const float* dkd, void* dX, void* dparams, void* ws, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    const Cotangents cot = {lse, lse + cfg->rows, dce, dkd};
    if (cfg->mode == REV_MODE_BF16) return VocabRunner<bf16>(*cfg, params, ws, s, labels, idx, logits).backward(X, cot, dX, dparams);
    return VocabRunner<float>(*cfg, params, ws, s, labels, idx, logits).backward(X, cot, dX, dparams);
}

int rev_xent_forward(const rev_vocab_cfg* cfg, const void* params, const void* X, const int32_t* labels, float* loss, float* lse,
                     void* workspace, int64_t workspace_bytes, void* stream) {
    RC(vocab_common(cfg, params, X, 0, (uintptr_t)labels | (uintptr_t)loss | (uintptr_t)lse, workspace, workspace_bytes));
    if (!labels || !loss || !lse) { set_error("a required pointer is null"); return REV_EINVAL; }
    return vocab_forward(cfg, params, X, labels, nullptr, nullptr, loss, nullptr, lse, workspace, stream);
}

int rev_xent_backward(const rev_vocab_cfg* cfg, const void* params, const void* X, const int32_t* labels, const float* lse, const float* dloss,
                      void* dX, void* dparams, void* workspace, int64_t workspace_bytes, void* stream) {
    RC(vocab_common(cfg, params, X, (uintptr_t)dX | (uintptr_t)dparams, (uintptr_t)labels | (uintptr_t)lse | (uintptr_t)dloss, workspace,
                    workspace_bytes));
    if (!labels || !lse || !dloss) { set_error("a required pointer is null"); return REV_EINVAL; }
    if (!dX && !dparams) { set_error("dX and dparams are both null"); return REV_EINVAL; }
    return vocab_backward(cfg, params, X, labels, nullptr, nullptr, lse, dloss, nullptr, dX, dparams, workspace, stream);
}

int rev_distill_forward(const rev_vocab_cfg* cfg, const void* params, const void* X, const int32_t* labels, const int32_t* teacher_idx,
                        const float* teacher_logits, float* loss_ce, float* loss_kd, float* lse, void* workspace, int64_t workspace_bytes,
                        void* stream) {
    RC(vocab_common(cfg, params, X, 0, (uintptr_t)labels | (uintptr_t)teacher_idx | (uintptr_t)teacher_logits | (uintptr_t)loss_ce | (uintptr_t)loss_kd |
                    (uintptr_t)lse, workspace, workspace_bytes));
    if (cfg->top_k < 1) { set_error("distillation needs top_k >= 1"); return REV_EINVAL; }
    if (!teacher_idx || !teacher_logits || !loss_kd || !lse) { set_error("a required pointer is null"); return REV_EINVAL; }
    if (!labels != !loss_ce) { set_error("labels and loss_ce go together"); return REV_EINVAL; }
    return vocab_forward(cfg, params, X, labels, teacher_idx, teacher_logits, loss_ce, loss_kd, lse, workspace, stream);
}

int rev_distill_backward(const rev_vocab_cfg* cfg, const void* params, const void* X, const int32_t* labels, const int32_t* teacher_idx,
                         const float* teacher_logits, const float* lse, const float* dloss_ce, const float* dloss_kd, void* dX, void* dparams,
                         void* workspace, int64_t workspace_bytes, void* stream) {
    RC(vocab_common(cfg, params, X, (uintptr_t)dX | (uintptr_t)dparams, (uintptr_t)labels | (uintptr_t)teacher_idx | (uintptr_t)teacher_logits |
                    (uintptr_t)lse | (uintptr_t)dloss_ce | (uintptr_t)dloss_kd, workspace, workspace_bytes));
    if (cfg->top_k < 1) { set_error("distillation needs top_k >= 1"); return REV_EINVAL; }
    if (!teacher_idx || !teacher_logits || !lse || !dloss_kd) { set_error("a required pointer is null"); return REV_EINVAL; }
    if (!labels != !dloss_ce) { set_error("labels and dloss_ce go together"); return REV_EINVAL; }
    if (!dX && !dparams) { set_error("dX and dparams are both null"); return REV_EINVAL; }
    return vocab_backward(cfg, params, X, labels, teacher_idx, teacher_logits, lse, dloss_ce, dloss_kd, dX, dparams, workspace, stream);
}

}  // extern "C"
