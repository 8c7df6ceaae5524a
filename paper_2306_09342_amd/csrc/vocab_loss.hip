// Losses over a vocabulary (softmax cross entropy, distillation from a teacher's top logits): entry points, workspace, and the
// kernels that go over rows.  The products with the vocabulary's weights go over it in pieces.
//
// Both losses have the gradient   dz = c0 exp(z - lse) + c1 exp(z / tau - lse_tau)   at every entry of the vocabulary, and
// something to be subtracted at the few entries that a row's label and teacher name.  The products compute the dense part only; the
// logits at the named entries are dot products of their own (sparse_logits_kernel: a row of W per entry), the losses
// are made of them, and in the backward pass the entries of dz that they touch are written again, from float32, behind the
// dense part (sparse_dz_kernel), so that p - 1 and q - p are rounded once and not taken from a rounded p.
//
// Rows that do not count (no label, no teacher) are left out before anything is multiplied: the others are gathered to the
// front of a copy of X, in their order, with rows of zeros behind them.  Their number stays on the device.
#include "common.h"
#include "rowwise.h"
#include "vocab.h"
#include <algorithm>

namespace rev {

// What bounds a plan: floats of dz, tiles of 256 columns in dx, places for its ranges (0, 0, 0: the float32 products, which have none).
struct PlanLimits { int64_t dz; int tiles_d, slots; };
struct RowResults { float* p[4]; };

// Pieces of equal widths whose dz fits.  dx has few tiles: its contraction, the piece, is cut into the number of ranges that keeps the
// 256 CUs busiest; a range costs about 10 stages besides its own (first loads, and writing and reading 256 KB).  By one wavefront,
// a number of ranges per lane.
__device__ __forceinline__ void write_plan(int count, int V, const PlanLimits& lim, VocabPlan* __restrict__ plan, int lane) {
    VocabPlan p = {count, (count + 255) / 256 * 256, (V + 255) / 256 * 256, 1, 2};
    if (lim.dz != 0 && count != 0) {                               // (without rows: one piece of zeros for dW)
        const unsigned most = (unsigned)((lim.dz / 256) / (p.rows / 256) / 256 * 256), pieces = (V + most - 1) / most;
        p.width = (int)((V + pieces - 1) / pieces + 255) / 256 * 256;
        const int tiles = p.rows / 256 * lim.tiles_d, pairs = p.width / 128, s = lane + 1;
        const int stages = (pairs + s - 1) / s * 2;
        unsigned cost = s <= pairs && tiles * s <= lim.slots ? (unsigned)((tiles * s + 255) / 256) * (stages + 10) : ~0u;
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
constexpr int HAS_LABEL = LOSS_CE, HAS_TEACHER = LOSS_KD;
__device__ __forceinline__ bool in_vocab(int v, int V) { return (unsigned)v < (unsigned)V; }
__device__ __forceinline__ bool teacher_counts(int idx, float logit, int V) { return in_vocab(idx, V) && !(logit == -INFINITY); }

// One wavefront per row: whether it has a label and whether it has a teacher.
__global__ __launch_bounds__(256) void row_flags_kernel(const int* __restrict__ labels, const int* __restrict__ idx,
                                                        const float* __restrict__ logits, int M, int V, int K, uint8_t* __restrict__ flags) {
    const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= M) return;
    bool any = false;
    for (int k = lane; k < K; k += 64) any |= teacher_counts(idx[(int64_t)r * K + k], logits[(int64_t)r * K + k], V);
    const bool taught = __any(any);
    if (lane == 0) flags[r] = (labels && in_vocab(labels[r], V) ? HAS_LABEL : 0) | (taught ? HAS_TEACHER : 0);
}

// One workgroup: list[i] = the i-th row that counts, place[r] = i or -1, zeros in the results of the others, and the plan.  Each
// thread takes 16 rows at a time.
__global__ __launch_bounds__(1024) void select_rows_kernel(const int* __restrict__ labels, const uint8_t* __restrict__ flags, int M, int V,
                                                           int* __restrict__ list, int* __restrict__ place, RowResults zero, PlanLimits lim,
                                                           VocabPlan* __restrict__ plan) {
    __shared__ int wsum[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int base = 0;
    for (int r0 = 0; r0 < M; r0 += 16384) {
        const int first = r0 + tid * 16;
        unsigned mask = 0;
        int y[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) y[k] = first + k < M ? flags ? flags[first + k] ? 0 : -1 : labels[first + k] : -1;
#pragma unroll
        for (int k = 0; k < 16; ++k) mask |= in_vocab(y[k], V) ? 1u << k : 0u;
        int incl = __popc(mask);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int t = __shfl_up(incl, o, 64);
            if (lane >= o) incl += t;
        }
        if (lane == 63) wsum[wave] = incl;
        __syncthreads();
        int before = base, total = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) before += wsum[w];
            total += wsum[w];
        }
        int i = before + incl - __popc(mask);
        for (int k = 0; k < 16; ++k) {
            const int r = first + k;
            if (r >= M) break;
            const bool on = mask >> k & 1;
            place[r] = on ? i : -1;
            if (on) {
                list[i++] = r;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (zero.p[q]) zero.p[q][r] = 0.f;
            }
        }
        base += total;
        __syncthreads();
    }
    if (tid < 64) write_plan(base, V, lim, plan, tid);
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
// Entry 0 of a row is its label, entries 1 .. K its teacher's; -1: none.
__device__ __forceinline__ int entry_of(const VocabRows& v, int r, int e) {
    if (e == 0) {
        const int y = v.labels ? v.labels[r] : -1;
        return in_vocab(y, v.V) ? y : -1;
    }
    const int64_t at = (int64_t)r * v.K + e - 1;
    return teacher_counts(v.idx[at], v.logits[at], v.V) ? v.idx[at] : -1;
}

// Row i of Xc = X[list[i]], padded with zeros to Dp columns and to whole tiles of rows, and zs[i][e] = <W_v, x> + b_v for its entries: one
// workgroup per row, one wavefront per entry at a time.  Bound by reading the rows of W, scattered over all of it: 64 entries of 8192
// rows of 1024, 1.07 GB, in 160 us.  In the backward pass also what the row's dense part is made of, and dz at its label, which
// without a teacher is all that is named.
struct Cotangents { const float *lse, *lse_tau, *dce, *dkd; };
// P: parts that the copy of X has, 0: its own type, over all rows.
template <typename T, int P>
__global__ __launch_bounds__(256) void gather_kernel(VocabRows v, const T* __restrict__ params, const T* __restrict__ X, int D, int Dp, int64_t Mp,
                                                     void* __restrict__ Xc, float* __restrict__ zs, const uint8_t* __restrict__ flags, Cotangents cot,
                                                     float4* __restrict__ coef, LabelDz* __restrict__ label_dz) {
    constexpr int E = 16 / sizeof(T);
    const int i = blockIdx.x, count = v.plan->count;
    if (P > 0 && i >= v.plan->rows) return;
    const int r = i < count ? v.list[i] : 0;
    const T* x = X + (int64_t)r * D;
    for (int d = threadIdx.x * E; d < Dp; d += 256 * E) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (i < count && d < D) u = *reinterpret_cast<const uint4*>(x + d);
        if constexpr (P < 3) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(Xc) + (int64_t)i * Dp + d) = u;
        else store_parts(u, reinterpret_cast<bf16*>(Xc) + (int64_t)i * Dp + d, Mp * Dp);
    }
    if (i >= count) return;
    float4 c = make_float4(0.f, INFINITY, 0.f, INFINITY);
    if (coef) {
        const int f = flags ? flags[r] : HAS_LABEL;
        if (f & HAS_LABEL) { c.x = cot.dce[r]; c.y = cot.lse[r]; }
        if (f & HAS_TEACHER) { c.z = cot.dkd[r] / v.inv_tau; c.w = cot.lse_tau[r]; }
        if (threadIdx.x == 0) coef[i] = c;
    }
    const int lane = threadIdx.x & 63;
    for (int e = threadIdx.x >> 6; e <= v.K; e += 4) {
        const int n = entry_of(v, r, e);
        float s = 0.f;
        if (n >= 0) {
            const T* w = params + (int64_t)n * D;
            for (int d = lane * E; d < D; d += 64 * E) {
#pragma unroll
                for (int q = 0; q < E; q += 4) {
                    const f4 a = load4(x + d + q), b = load4(w + d + q);
                    s = fmaf(a.x, b.x, s); s = fmaf(a.y, b.y, s); s = fmaf(a.z, b.z, s); s = fmaf(a.w, b.w, s);
                }
            }
        }
        s = wave_sum(s);
        if (n >= 0 && v.bias) s += to_f(params[(int64_t)v.V * D + n]);
        if (lane == 0) zs[(int64_t)i * (v.K + 1) + e] = s;
        if (e == 0 && lane == 0 && label_dz) label_dz[i] = {n, dense_dz(c, s, v.inv_tau) - c.x};
    }
}

// The teacher's probabilities of a row, entry e = 1 + lane + 64 q in p[q] (0: none), and log p_k = t_k / tau - log_norm.
struct Teacher { float p[4], t[4], log_norm; };
__device__ __forceinline__ Teacher teacher_of(const VocabRows& v, int r, int lane) {
    Teacher a;
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int k = lane + 64 * q;
        a.t[q] = k < v.K && entry_of(v, r, k + 1) >= 0 ? v.logits[(int64_t)r * v.K + k] * v.inv_tau : -INFINITY;
        m = fmaxf(m, a.t[q]);
    }
    m = wave_max(m);
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        a.p[q] = a.t[q] == -INFINITY ? 0.f : expf(a.t[q] - m);
        s += a.p[q];
    }
    s = wave_sum(s);
    a.log_norm = m + logf(s);
#pragma unroll
    for (int q = 0; q < 4; ++q) a.p[q] = a.p[q] / s;
    return a;
}

// ---------------------------------------------------------------------------------
// losses
// ---------------------------------------------------------------------------------
// The statistics of 64 rows that count joined, and their losses.  stats: [strips][N][Mp] = maximum m of a strip, sums of
// exp(z - m) and exp((z - m) / tau), the second with N = 3 only, the first in its place if only the teacher's loss is wanted.  A lane
// per row and 16 wavefronts over the strips; then a wavefront per row over the teacher's entries.
template <int N>
__global__ __launch_bounds__(1024) void losses_kernel(VocabRows v, const float* __restrict__ stats, int strips, int64_t Mp, const float* __restrict__ zs,
                                                      const uint8_t* __restrict__ flags, RowResults out) {
    __shared__ float sh[3][16][64];
    __shared__ float row[3][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i0 = blockIdx.x * 64, count = v.plan->count;
    float *loss_ce = out.p[0], *lse = out.p[1], *loss_kd = out.p[2], *lse_tau = out.p[3];
    if (i0 >= count) return;
    const float rate0 = N == 2 && !loss_ce ? v.inv_tau : 1.f;
    float m = -INFINITY, s0 = 0.f, s1 = 0.f;
    const float* at = stats + i0 + lane;
    if (i0 + lane < count)
        for (int p0 = w; p0 < strips; p0 += 64) {
            float a[4][N];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int k = 0; k < N; ++k) a[u][k] = p0 + 16 * u < strips ? at[((int64_t)(p0 + 16 * u) * N + k) * Mp] : k ? 0.f : -INFINITY;
            const float top = fmaxf(fmaxf(fmaxf(a[0][0], a[1][0]), fmaxf(a[2][0], a[3][0])), m);
            if (top == -INFINITY) continue;
            s0 *= expf((m - top) * rate0);
            if (N == 3) s1 *= expf((m - top) * v.inv_tau);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                s0 += a[u][1] * expf((a[u][0] - top) * rate0);
                if (N == 3) s1 += a[u][N - 1] * expf((a[u][0] - top) * v.inv_tau);
            }
            m = top;
        }
    sh[0][w][lane] = m; sh[1][w][lane] = s0; sh[2][w][lane] = s1;
    __syncthreads();
    if (w == 0) {
        float top = -INFINITY, t0 = 0.f, t1 = 0.f;
        for (int k = 0; k < 16; ++k) top = fmaxf(top, sh[0][k][lane]);
        for (int k = 0; k < 16; ++k) {
            const float d = sh[0][k][lane] - top;
            t0 += sh[1][k][lane] * expf(d * rate0);
            if (N == 3) t1 += sh[2][k][lane] * expf(d * v.inv_tau);
        }
        row[0][lane] = top; row[1][lane] = logf(t0); row[2][lane] = logf(N == 3 ? t1 : t0);
    }
    __syncthreads();
    if (w == 0 && i0 + lane < count) {
        const int i = i0 + lane, r = v.list[i];
        const bool has = loss_ce && (!flags || flags[r] & HAS_LABEL);
        if (loss_ce) loss_ce[r] = has ? row[1][lane] + (row[0][lane] - zs[(int64_t)i * (v.K + 1)]) : 0.f;
        lse[r] = has ? row[0][lane] + row[1][lane] : 0.f;
    }
    if (!loss_kd) return;
    for (int k = w; k < 64 && i0 + k < count; k += 16) {
        const int i = i0 + k, r = v.list[i];
        const float top = row[0][k], log_s = row[2][k];
        float kd = 0.f, l = 0.f;
        if (flags[r] & HAS_TEACHER) {
            const float* z = zs + (int64_t)i * (v.K + 1);
            const Teacher t = teacher_of(v, r, lane);
            l = top * v.inv_tau + log_s;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (t.p[q] != 0.f) kd += t.p[q] * ((t.t[q] - t.log_norm) - ((z[1 + lane + 64 * q] - top) * v.inv_tau - log_s));
            kd = wave_sum(kd) / (v.inv_tau * v.inv_tau);
        }
        if (lane == 0) { loss_kd[r] = kd; lse_tau[r] = l; }
    }
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
        v0 *= (int)ld;
        n = min((int)ld, v.V - v0);
        if (n <= 0) return;
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
// float32: a piece of the vocabulary with its logits in memory
// ---------------------------------------------------------------------------------
// One workgroup per row: maximum and sums of a piece (n entries, pitch ld).
__global__ __launch_bounds__(256) void piece_stats_kernel(const float* __restrict__ z, int64_t ld, int n, const float* __restrict__ bias,
                                                          const VocabPlan* __restrict__ plan, float inv_tau, int64_t Mp, float* __restrict__ stats) {
    __shared__ float sh[3][4];
    const int i = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (i >= plan->count) return;
    const float* row = z + (int64_t)i * ld;
    float m = -INFINITY;
    for (int c = threadIdx.x; c < n; c += 256) m = fmaxf(m, row[c] + (bias ? bias[c] : 0.f));
    m = wave_max(m);
    if (lane == 0) sh[0][w] = m;
    __syncthreads();
    m = fmaxf(fmaxf(sh[0][0], sh[0][1]), fmaxf(sh[0][2], sh[0][3]));
    const float ref = m == -INFINITY ? 0.f : m;
    float s0 = 0.f, s1 = 0.f;
    for (int c = threadIdx.x; c < n; c += 256) {
        const float d = row[c] + (bias ? bias[c] : 0.f) - ref;
        s0 += expf(d);
        s1 += expf(d * inv_tau);
    }
    s0 = wave_sum(s0);
    s1 = wave_sum(s1);
    if (lane == 0) { sh[1][w] = s0; sh[2][w] = s1; }
    __syncthreads();
    if (threadIdx.x == 0) {
        stats[i] = m;
        stats[Mp + i] = (sh[1][0] + sh[1][1]) + (sh[1][2] + sh[1][3]);
        stats[2 * Mp + i] = (sh[2][0] + sh[2][1]) + (sh[2][2] + sh[2][3]);
    }
}

// The dense part of dz in the place of the logits, zeros in the columns behind the piece and the rows behind the last one that counts.
__global__ __launch_bounds__(256) void piece_dz_kernel(float* z, int64_t ld, int n, const float* __restrict__ bias, const VocabPlan* __restrict__ plan,
                                                       const float4* __restrict__ coef, float inv_tau) {
    const int across = (int)((ld + 255) / 256), i = blockIdx.x / across, c = (blockIdx.x - i * across) * 256 + threadIdx.x;
    if (c >= ld) return;
    float d = 0.f;
    if (i < plan->count && c < n) d = dense_dz(coef[i], z[(int64_t)i * ld + c] + (bias ? bias[c] : 0.f), inv_tau);
    z[(int64_t)i * ld + c] = d;
}

// Column sums of a piece of dz: 64 columns per workgroup, 16 wavefronts over the rows.
__global__ __launch_bounds__(1024) void piece_colsum_kernel(const float* __restrict__ dz, int64_t ld, int n, const VocabPlan* __restrict__ plan,
                                                            float* __restrict__ out) {
    __shared__ float sh[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, count = plan->count;
    float s = 0.f;
    if (c < n)
        for (int i = w; i < count; i += 16) s += dz[(int64_t)i * ld + c];
    sh[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < n) {
        for (int k = 1; k < 16; ++k) s += sh[k][lane];
        out[c] = s;
    }
}

__global__ __launch_bounds__(256) void add_kernel(const float* __restrict__ more, int64_t n, float* __restrict__ acc) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c < n) acc[c] += more[c];
}
__global__ __launch_bounds__(256) void copy_kernel(const float* __restrict__ src, int valid, int total, float* __restrict__ dst) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < total) dst[c] = c < valid ? src[c] : 0.f;
}

// dX[r] from the sums of its place, zeros for a row that does not count.
__global__ __launch_bounds__(256) void dx_rows_kernel(const float* __restrict__ acc, const int* __restrict__ place, int M, int D, float* __restrict__ dX) {
    const int per = D / 4;
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= (int64_t)M * per) return;
    const int64_t r = c / per;
    const int d = (int)(c - r * per) * 4, i = place[r];
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if (i >= 0) v = load4(acc + (int64_t)i * D + d);
    store4(dX + r * D + d, v);
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

// float32: by parts from PARTS_ROWS rows on
constexpr int PARTS_ROWS = 128;
static bool takes_parts(const rev_vocab_cfg& c) { return c.rows > PARTS_ROWS; }

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// dz of a piece: 256 MB, what the memory-side cache holds, or 256 entries of all rows if that is more
constexpr int64_t VOCAB_DZ_BYTES = 256 << 20;
struct VocabLayout {
    int64_t plan, flags, place, list, coef, label_dz, zs, stats, xc, w, dz, acc, more, total;
    int64_t Mp;
    int parts;                       // bf16 parts of an operand of the products; 0: float32 products (gemm_f32.hip)
    int Dp, strips, pieces;          // parts: most pieces that a plan may have
    int Vc, rest;                    // float32: width of a piece, entries left over behind whole multiples of 4 (the last piece)
    PlanLimits lim;
};
static VocabLayout vocab_layout(const rev_vocab_cfg& c) {
    VocabLayout L = {};
    L.parts = c.mode == REV_MODE_BF16 ? 1 : takes_parts(c) ? 3 : 0;
    const int64_t M = c.rows, D = c.d_model, V = c.vocab;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t o = at; at += up(bytes, 256); return o; };
    L.plan = take(sizeof(VocabPlan));
    L.flags = take(M);
    L.place = take(4 * M);
    L.list = take(4 * M);
    L.label_dz = take(8 * M);
    L.zs = take(4 * M * (c.top_k + 1));
    if (L.parts) {
        L.Mp = up(M, 256);
        L.Dp = (int)up(D, 128);
        L.lim.dz = std::min(std::max(VOCAB_DZ_BYTES / 2 / L.parts / 256 * 256, L.Mp * 256), L.Mp * up(V, 256));
        L.lim.tiles_d = (int)((D + 255) / 256);
        L.lim.slots = (int)std::max<int64_t>(L.Mp / 256 * L.lim.tiles_d, 512);
        const int64_t least = L.lim.dz / L.Mp / 256 * 256;
        L.pieces = (int)((V + least - 1) / least);
        L.strips = (int)((V + 255) / 256) * 2;
        L.coef = take(16 * M);
        L.stats = take(12 * L.Mp * L.strips);
        L.xc = take(2 * L.parts * L.Mp * L.Dp);
        L.w = L.Dp != D || L.parts > 1 ? take(2 * L.parts * V * L.Dp) : 0;
        L.dz = take(2 * L.parts * L.lim.dz);
        L.acc = take((int64_t)L.lim.slots * 65536 * 4);
    } else {
        L.Mp = up(M, 64);
        L.Dp = c.d_model;
        const int64_t whole = V / 4 * 4;
        L.Vc = (int)std::min(std::max(VOCAB_DZ_BYTES / 4 / L.Mp / 256 * 256, (int64_t)256), std::max<int64_t>(whole, 4));
        L.rest = (int)(V - whole);
        L.pieces = L.strips = (int)((whole + L.Vc - 1) / L.Vc) + (L.rest ? 1 : 0);
        L.coef = take(16 * M);
        L.stats = take(12 * L.Mp * L.strips);
        L.xc = take(4 * L.Mp * D);
        L.w = take(4 * 4 * D);
        L.dz = take(4 * L.Mp * L.Vc);
        L.acc = take(4 * L.Mp * D);
        L.more = take(4 * std::max<int64_t>(4, L.pieces > 1 ? L.Mp : 0) * D);
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
    int prepare(const void* X, const RowResults& zero, const Cotangents& cot) {
        ProfScope ps(K_CONVERT, s, (double)M * D * 2 * sizeof(T));
        if (v.idx) LAUNCH(row_flags_kernel, blocks_of(M, 4), dim3(256), v.labels, v.idx, v.logits, M, V, v.K, at<uint8_t>(L.flags));
        LAUNCH(select_rows_kernel, dim3(1), dim3(1024), v.labels, flags(), M, V, at<int>(L.list), at<int>(L.place), zero, L.lim, at<VocabPlan>(L.plan));
        float4* coef = cot.lse ? at<float4>(L.coef) : nullptr;
        LabelDz* label_dz = cot.lse && !v.idx ? at<LabelDz>(L.label_dz) : nullptr;
        const dim3 grid((unsigned)L.Mp), block(256);
        if (L.parts)
            LAUNCH((gather_kernel<T, kParts>), grid, block, v, params, (const T*)X, D, L.Dp, L.Mp, at<void>(L.xc), at<float>(L.zs), flags(), cot, coef, label_dz);
        else
            LAUNCH((gather_kernel<T, 0>), grid, block, v, params, (const T*)X, D, L.Dp, L.Mp, at<void>(L.xc), at<float>(L.zs), flags(), cot, coef, label_dz);
        return REV_OK;
    }
    int join(const RowResults& out, bool three) {
        ProfScope ps(K_REDUCE, s, 12.0 * L.Mp * L.strips);
        if (three) LAUNCH(losses_kernel<3>, blocks_of(M, 64), dim3(1024), v, at<float>(L.stats), L.strips, L.Mp, at<float>(L.zs), flags(), out);
        else LAUNCH(losses_kernel<2>, blocks_of(M, 64), dim3(1024), v, at<float>(L.stats), L.strips, L.Mp, at<float>(L.zs), flags(), out);
        return REV_OK;
    }

    // ---- products of bf16 parts ----
    int gemm_args(VocabGemm* g) {
        *g = {};
        g->plan = v.plan; g->x = at<bf16>(L.xc); g->bias = bias(); g->label_dz = v.idx ? nullptr : at<LabelDz>(L.label_dz);
        g->stats = at<float>(L.stats); g->coef = at<float4>(L.coef); g->dz = at<bf16>(L.dz); g->acc = at<float>(L.acc);
        g->Mp = L.Mp; g->dz_part = L.lim.dz; g->V = V; g->D = D; g->Dp = L.Dp; g->losses = losses(); g->inv_tau = v.inv_tau;
        g->w = g->wp = (const bf16*)params;
        g->ldw = D;
        if (L.w) {
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
        RC(vocab_logits<T>(s, g, false, dual(), L.Mp / 256 * ((V + 255) / 256)));
        return join(out, dual());
    }
    int backward_parts(T* dX, void* dparams) {
        VocabGemm g;
        RC(gemm_args(&g));
        for (int k = 0; k < L.pieces; ++k) {
            // tiles of 256 entries that piece k may have: there is a piece k only if a piece is at most a k+1-th of the vocabulary
            const int64_t tiles_v = ((V + k) / (k + 1) + 255) / 256;
            g.piece = k;
            RC(vocab_logits<T>(s, g, true, dual(), std::min(L.Mp / 256 * tiles_v, std::max(L.lim.dz / 65536, tiles_v))));
            if (v.idx) LAUNCH((sparse_dz_kernel<bf16, kParts>), blocks_of(M, 4), dim3(256), v, at<float>(L.zs), at<float4>(L.coef), k, 0, at<bf16>(L.dz),
                              (int64_t)0, L.lim.dz);
            if (dX) RC(vocab_dx<T>(s, g, L.lim.slots));
            if (dparams) RC(vocab_dw<T>(s, g, dparams, c.grad_mode == REV_MODE_BF16, c.bias, tiles_v * (L.lim.tiles_d + (c.bias ? 1 : 0))));
        }
        return dX ? vocab_dx_rows<T>(s, g, v.place, M, dX) : REV_OK;
    }

    // ---- float32 products ----
    struct Piece { int v0, n, width; const float* w; };              // first entry, entries, width (a multiple of 4), its rows of W
    int piece(int k, Piece* p) {
        const bool last = L.rest && k == L.pieces - 1;
        p->v0 = last ? V - L.rest : k * L.Vc;
        p->n = last ? L.rest : std::min(L.Vc, V / 4 * 4 - p->v0);
        p->width = last ? 4 : p->n;
        p->w = (const float*)params + (int64_t)p->v0 * D;
        if (last) {
            LAUNCH(copy_kernel, blocks_of(4 * D, 256), dim3(256), p->w, L.rest * D, 4 * D, at<float>(L.w));
            p->w = at<float>(L.w);
        }
        Epi e = {}; e.kind = EPI_PLAIN_F32; e.outf = at<float>(L.dz); e.ldo = p->width; e.solo = true;
        return gemm_nt_f32(s, at<float>(L.xc), D, p->w, D, (int)L.Mp, p->width, D, e);
    }
    int forward_f32(const RowResults& out) {
        for (int k = 0; k < L.pieces; ++k) {
            Piece p;
            RC(piece(k, &p));
            LAUNCH(piece_stats_kernel, dim3(M), dim3(256), at<float>(L.dz), (int64_t)p.width, p.n, bias() ? (const float*)bias() + p.v0 : nullptr, v.plan, v.inv_tau,
                   L.Mp, at<float>(L.stats) + (int64_t)k * 3 * L.Mp);
        }
        return join(out, true);
    }
    int backward_f32(float* dX, float* dparams) {
        float *dz = at<float>(L.dz), *acc = at<float>(L.acc), *more = at<float>(L.more);
        for (int k = 0; k < L.pieces; ++k) {
            Piece p;
            RC(piece(k, &p));
            LAUNCH(piece_dz_kernel, dim3((unsigned)((p.width + 255) / 256 * L.Mp)), dim3(256), dz, (int64_t)p.width, p.n, bias() ? (const float*)bias() + p.v0 : nullptr,
                   v.plan, at<float4>(L.coef), v.inv_tau);
            LAUNCH((sparse_dz_kernel<float, 1>), blocks_of(M, 4), dim3(256), v, at<float>(L.zs), at<float4>(L.coef), p.v0, p.n, dz, (int64_t)p.width, (int64_t)0);
            if (dX) {
                Epi e = {}; e.kind = EPI_PLAIN_F32; e.outf = k ? more : acc; e.ldo = D; e.solo = true;
                RC(gemm_nn_f32(s, dz, p.width, p.w, D, (int)L.Mp, D, p.width, e));
                if (k) LAUNCH(add_kernel, blocks_of(L.Mp * D, 256), dim3(256), more, L.Mp * D, acc);
            }
            if (dparams) {
                float* dw = dparams + (int64_t)p.v0 * D;
                const WgradF32Item it = {dz, p.width, at<float>(L.xc), D, p.width, D, p.width == p.n ? dw : more, nullptr};
                RC(gemm_wgrad_f32_group(s, &it, 1, (int)L.Mp));
                if (p.width != p.n) LAUNCH(copy_kernel, blocks_of(p.n * D, 256), dim3(256), more, p.n * D, p.n * D, dw);
                if (c.bias) LAUNCH(piece_colsum_kernel, blocks_of(p.n, 64), dim3(1024), dz, (int64_t)p.width, p.n, v.plan, dparams + (int64_t)V * D + p.v0);
            }
        }
        if (dX) LAUNCH(dx_rows_kernel, blocks_of((int64_t)M * D / 4, 256), dim3(256), acc, v.place, M, D, dX);
        return REV_OK;
    }

    int forward(const void* X, const RowResults& out) {
        RC(prepare(X, out, Cotangents{}));
        if (L.parts) return forward_parts(out);
        if constexpr (kParts == 3) return forward_f32(out);
        return REV_OK;
    }
    int backward(const void* X, const Cotangents& cot, void* dX, void* dparams) {
        RC(prepare(X, RowResults{}, cot));
        if (L.parts) return backward_parts((T*)dX, dparams);
        if constexpr (kParts == 3) return backward_f32((float*)dX, (float*)dparams);
        return REV_OK;
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
