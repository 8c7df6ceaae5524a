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

// ---------------------------------------------------------------------------------
// which rows count
// ---------------------------------------------------------------------------------
constexpr int HAS_LABEL = 1, HAS_TEACHER = 2;
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

// One workgroup: list[i] = the i-th row that counts, place[r] = i or -1, *count.  Each thread takes 16 rows at a time.
__global__ __launch_bounds__(1024) void select_rows_kernel(const int* __restrict__ labels, const uint8_t* __restrict__ flags, int M, int V,
                                                           int* __restrict__ list, int* __restrict__ place, int* __restrict__ count) {
    __shared__ int wsum[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int base = 0;
    for (int r0 = 0; r0 < M; r0 += 16384) {
        const int first = r0 + tid * 16;
        unsigned mask = 0;
        for (int k = 0; k < 16; ++k) {
            const int r = first + k;
            if (r < M && (flags ? flags[r] != 0 : in_vocab(labels[r], V))) mask |= 1u << k;
        }
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
            if (on) list[i++] = r;
        }
        base += total;
        __syncthreads();
    }
    if (tid == 0) *count = base;
}

// Xc[i] = X[list[i]], padded with zeros to Dp columns and to all of Mp rows.  Chunks of 16 bytes, one per thread.
template <typename T>
__global__ __launch_bounds__(256) void gather_rows_kernel(const T* __restrict__ X, const int* __restrict__ list, const int* __restrict__ count,
                                                          int D, int Dp, int64_t chunks, T* __restrict__ Xc) {
    constexpr int E = 16 / sizeof(T);
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= chunks) return;
    const int per = Dp / E;
    const int64_t i = c / per;
    const int d = (int)(c - i * per) * E;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (i < *count && d < D) v = *reinterpret_cast<const uint4*>(X + (int64_t)list[i] * D + d);
    *reinterpret_cast<uint4*>(Xc + i * Dp + d) = v;
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

// zs[i][e] = <W_v, x> + b_v.  One workgroup per row, one wavefront per entry at a time.  Bound by reading the rows of W,
// scattered over all of it.
template <typename T>
__global__ __launch_bounds__(256) void sparse_logits_kernel(VocabRows v, const T* __restrict__ params, const T* __restrict__ Xc, int D, int Dp,
                                                            float* __restrict__ zs) {
    constexpr int E = 16 / sizeof(T);
    const int i = blockIdx.x;
    if (i >= *v.count) return;
    const int lane = threadIdx.x & 63, r = v.list[i];
    const T* x = Xc + (int64_t)i * Dp;
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
        if (lane == 0) zs[(int64_t)i * (v.K + 1) + e] = n >= 0 && v.bias ? s + to_f(params[(int64_t)v.V * D + n]) : s;
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
// One wavefront per row of X: the statistics of its pieces joined, the losses, and zeros for what a row has not.
// stats: [pieces][3][Mp] = maximum, sum of exp(z - maximum), sum of exp((z - maximum) / tau).
__global__ __launch_bounds__(256) void losses_kernel(VocabRows v, const float* __restrict__ stats, int pieces, int64_t Mp,
                                                     const float* __restrict__ zs, float* __restrict__ loss_ce, float* __restrict__ loss_kd,
                                                     float* __restrict__ lse, float* __restrict__ lse_tau) {
    const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= v.M) return;
    const int i = v.place[r];
    float ce = 0.f, kd = 0.f, l0 = 0.f, l1 = 0.f;
    if (i >= 0) {
        float m = -INFINITY;
        for (int p = lane; p < pieces; p += 64) m = fmaxf(m, stats[(int64_t)p * 3 * Mp + i]);
        m = wave_max(m);
        float s0 = 0.f, s1 = 0.f;
        for (int p = lane; p < pieces; p += 64) {
            const float* q = stats + (int64_t)p * 3 * Mp + i;
            const float d = q[0] - m;
            s0 += q[Mp] * expf(d);
            if (loss_kd) s1 += q[2 * Mp] * expf(d * v.inv_tau);
        }
        s0 = wave_sum(s0);
        s1 = wave_sum(s1);
        const float* z = zs + (int64_t)i * (v.K + 1);
        const bool has = entry_of(v, r, 0) >= 0;
        if (has) {
            l0 = m + logf(s0);
            ce = logf(s0) + (m - z[0]);
        }
        if (loss_kd) {
            const Teacher t = teacher_of(v, r, lane);
            if (t.log_norm != -INFINITY) {
                l1 = m * v.inv_tau + logf(s1);
                float sum = 0.f;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (t.p[q] != 0.f) sum += t.p[q] * ((t.t[q] - t.log_norm) - ((z[1 + lane + 64 * q] - m) * v.inv_tau - logf(s1)));
                kd = wave_sum(sum) / (v.inv_tau * v.inv_tau);
            }
        }
    }
    if (lane == 0) {
        if (loss_ce) loss_ce[r] = ce;
        lse[r] = l0;
        if (loss_kd) { loss_kd[r] = kd; lse_tau[r] = l1; }
    }
}

// ---------------------------------------------------------------------------------
// gradient of the logits
// ---------------------------------------------------------------------------------
// coef[i] = {dloss_ce or 0, lse, dloss tau or 0, lse_tau}: what a row's dense part is made of.
__global__ __launch_bounds__(256) void coef_kernel(VocabRows v, const uint8_t* __restrict__ flags, const float* __restrict__ lse,
                                                   const float* __restrict__ lse_tau, const float* __restrict__ dce,
                                                   const float* __restrict__ dkd, float4* __restrict__ coef) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= *v.count) return;
    const int r = v.list[i], f = flags ? flags[r] : HAS_LABEL;
    float4 c = make_float4(0.f, 0.f, 0.f, 0.f);
    if (f & HAS_LABEL) { c.x = dce[r]; c.y = lse[r]; }
    if (f & HAS_TEACHER) { c.z = dkd[r] / v.inv_tau; c.w = lse_tau[r]; }
    coef[i] = c;
}

// dz at the entries v0 .. v0 + n - 1 that a row names, again.  One wavefront per row; an entry that is named several times is written by
// the first of them.
template <typename T>
__global__ __launch_bounds__(256) void sparse_dz_kernel(VocabRows v, const float* __restrict__ zs, const float4* __restrict__ coef, int v0, int n,
                                                        T* __restrict__ dz, int64_t ld) {
    __shared__ int names[4][257];
    __shared__ float probs[4][257];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = blockIdx.x * 4 + w;
    const bool live = i < *v.count;
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
        if (first) dz[(int64_t)i * ld + name - v0] = from_f<T>(dense_dz(c, zs[(int64_t)i * (v.K + 1) + e], v.inv_tau) - less);
    }
}

// dX[r] from the sums of its place, zeros for a row that does not count.
template <typename T>
__global__ __launch_bounds__(256) void scatter_dx_kernel(const float* __restrict__ acc, const int* __restrict__ place, int M, int D,
                                                         T* __restrict__ dX) {
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
// a piece of the vocabulary with its logits in float32
// ---------------------------------------------------------------------------------
// One workgroup per row: maximum and sums of a piece (n entries, pitch ld).
template <typename T>
__global__ __launch_bounds__(256) void piece_stats_kernel(const float* __restrict__ z, int64_t ld, int n, const T* __restrict__ bias,
                                                          const int* __restrict__ count, float inv_tau, int64_t Mp, float* __restrict__ stats) {
    __shared__ float sh[3][4];
    const int i = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (i >= *count) return;
    const float* row = z + (int64_t)i * ld;
    float m = -INFINITY;
    for (int c = threadIdx.x; c < n; c += 256) m = fmaxf(m, row[c] + (bias ? to_f(bias[c]) : 0.f));
    m = wave_max(m);
    if (lane == 0) sh[0][w] = m;
    __syncthreads();
    m = fmaxf(fmaxf(sh[0][0], sh[0][1]), fmaxf(sh[0][2], sh[0][3]));
    const float ref = m == -INFINITY ? 0.f : m;
    float s0 = 0.f, s1 = 0.f;
    for (int c = threadIdx.x; c < n; c += 256) {
        const float d = row[c] + (bias ? to_f(bias[c]) : 0.f) - ref;
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

// The dense part of dz, zeros in the columns behind the piece and the rows behind the last one that counts.
template <typename T>
__global__ __launch_bounds__(256) void piece_dz_kernel(const float* z, int64_t ld, int n, const T* __restrict__ bias,
                                                       const int* __restrict__ count, const float4* __restrict__ coef, float inv_tau, int64_t ldz,
                                                       T* dz) {
    const int across = (int)((ld + 255) / 256), i = blockIdx.x / across, c = (blockIdx.x - i * across) * 256 + threadIdx.x;
    if (c >= ld) return;
    float d = 0.f;
    if (i < *count && c < n) d = dense_dz(coef[i], z[(int64_t)i * ld + c] + (bias ? to_f(bias[c]) : 0.f), inv_tau);
    dz[(int64_t)i * ldz + c] = from_f<T>(d);
}

// Column sums of a piece of dz, one thread per column.
template <typename T>
__global__ __launch_bounds__(256) void piece_colsum_kernel(const T* __restrict__ dz, int64_t ld, int n, const int* __restrict__ count,
                                                           void* out, int64_t at, bool out_bf16) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    float s = 0.f;
    for (int i = 0; i < *count; ++i) s += to_f(dz[(int64_t)i * ld + c]);
    if (out_bf16) reinterpret_cast<bf16*>(out)[at + c] = from_f<bf16>(s);
    else reinterpret_cast<float*>(out)[at + c] = s;
}

__global__ __launch_bounds__(256) void add_kernel(const float* __restrict__ more, int64_t n, float* __restrict__ acc) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c < n) acc[c] += more[c];
}
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(const T* __restrict__ src, int64_t valid, int64_t total, T* __restrict__ dst) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c < total) dst[c] = c < valid ? src[c] : from_f<T>(0.f);
}
__global__ __launch_bounds__(256) void store_grad_kernel(const float* __restrict__ src, int64_t n, void* out, int64_t at, bool out_bf16) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    if (out_bf16) reinterpret_cast<bf16*>(out)[at + c] = from_f<bf16>(src[c]);
    else reinterpret_cast<float*>(out)[at + c] = src[c];
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

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
struct VocabLayout {
    int64_t flags, place, list, count, coef, zs, stats, xc, w, z, dz, acc, dw, wg, total;
    int64_t Mp, wg_elems;
    int Dp, Vc, rest, pieces;        // width of a piece, what is left over behind whole multiples of 8, pieces in all
};
static VocabLayout vocab_layout(const rev_vocab_cfg& c) {
    VocabLayout L = {};
    const int64_t M = c.rows, D = c.d_model, V = c.vocab, es = c.mode == REV_MODE_BF16 ? 2 : 4;
    L.Mp = up(M, 64);
    L.Dp = c.d_model;
    const int64_t whole = V / 8 * 8;
    L.Vc = (int)std::min<int64_t>(std::max<int64_t>((int64_t)(256 << 20) / 4 / L.Mp / 256 * 256, 1024), up(std::max<int64_t>(whole, 8), 8));
    L.rest = (int)(V - whole);
    L.pieces = (int)((whole + L.Vc - 1) / L.Vc) + (L.rest ? 1 : 0);
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t o = at; at += up(bytes, 256); return o; };
    L.count = take(4);
    L.flags = take(M);
    L.place = take(4 * M);
    L.list = take(4 * M);
    L.coef = take(16 * L.Mp);
    L.zs = take(4 * M * (c.top_k + 1));
    L.stats = take(12 * L.Mp * L.pieces);
    L.xc = take(es * L.Mp * L.Dp);
    L.w = take(es * 8 * D);
    L.z = take(4 * L.Mp * L.Vc);
    L.dz = take(es * L.Mp * L.Vc);
    L.acc = take(4 * L.Mp * D);
    L.dw = take(4 * std::max<int64_t>(L.Vc, L.Mp) * D);
    if (es == 2) {
        const int K = c.d_model, widths[3] = {L.Vc, whole % L.Vc ? (int)(whole % L.Vc) : L.Vc, 8};
        for (int n : widths) L.wg_elems = std::max(L.wg_elems, wgrad_scratch_elems((int)L.Mp, &n, &K, 1));
    }
    L.wg = take(4 * L.wg_elems);
    L.total = at;
    return L;
}

#define RC(expr) do { int _rc = (expr); if (_rc != REV_OK) return _rc; } while (0)
static dim3 blocks_of(int64_t n, int per) { return dim3((unsigned)((n + per - 1) / per)); }

template <typename T>
struct VocabRunner {
    static constexpr bool kBf16 = sizeof(T) == 2;
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
        v = {labels, idx, logits, at<int>(L.list), at<int>(L.place), at<int>(L.count), M, V, idx ? c.top_k : 0, c.bias,
             idx ? 1.f / c.temperature : 1.f};
    }
    template <typename U> U* at(int64_t off) const { return reinterpret_cast<U*>(ws + off); }
    const uint8_t* flags() const { return v.idx ? at<uint8_t>(L.flags) : nullptr; }
    const T* bias() const { return c.bias ? params + (int64_t)V * D : nullptr; }

    int prepare(const void* X) {
        ProfScope ps(K_CONVERT, s, (double)M * D * 2 * sizeof(T));
        if (v.idx) {
            hipLaunchKernelGGL(row_flags_kernel, blocks_of(M, 4), dim3(256), 0, s, v.labels, v.idx, v.logits, M, V, v.K, at<uint8_t>(L.flags));
            REV_HIP(hipGetLastError());
        }
        hipLaunchKernelGGL(select_rows_kernel, dim3(1), dim3(1024), 0, s, v.labels, flags(), M, V, at<int>(L.list), at<int>(L.place),
                           at<int>(L.count));
        REV_HIP(hipGetLastError());
        const int64_t chunks = L.Mp * L.Dp * sizeof(T) / 16;
        hipLaunchKernelGGL(gather_rows_kernel<T>, blocks_of(chunks, 256), dim3(256), 0, s, (const T*)X, at<int>(L.list), at<int>(L.count), D, L.Dp,
                           chunks, at<T>(L.xc));
        REV_HIP(hipGetLastError());
        hipLaunchKernelGGL(sparse_logits_kernel<T>, dim3(M), dim3(256), 0, s, v, params, at<T>(L.xc), D, L.Dp, at<float>(L.zs));
        REV_HIP(hipGetLastError());
        return REV_OK;
    }
    // piece k: first entry, entries, width (a multiple of 8), its rows of W
    struct Piece { int v0, n, width; const T* w; };
    int piece(int k, Piece* p) {
        const bool last = L.rest && k == L.pieces - 1;
        p->v0 = last ? V - L.rest : k * L.Vc;
        p->n = last ? L.rest : std::min(L.Vc, V / 8 * 8 - p->v0);
        p->width = last ? 8 : p->n;
        p->w = params + (int64_t)p->v0 * D;
        if (last) {
            hipLaunchKernelGGL(copy_rows_kernel<T>, blocks_of(8 * D, 256), dim3(256), 0, s, p->w, (int64_t)L.rest * D, (int64_t)8 * D, at<T>(L.w));
            REV_HIP(hipGetLastError());
            p->w = at<T>(L.w);
        }
        return REV_OK;
    }
    int logits(const Piece& p) {
        Epi e = {}; e.kind = EPI_PLAIN_F32; e.outf = at<float>(L.z); e.ldo = p.width; e.solo = true;
        if constexpr (kBf16) return gemm_nt_bf16(s, at<T>(L.xc), L.Dp, p.w, D, (int)L.Mp, p.width, D, e);
        else return gemm_nt_f32(s, at<T>(L.xc), L.Dp, p.w, D, (int)L.Mp, p.width, D, e);
    }

    int forward(const void* X, float* loss_ce, float* loss_kd, float* lse) {
        RC(prepare(X));
        for (int k = 0; k < L.pieces; ++k) {
            Piece p;
            RC(piece(k, &p));
            RC(logits(p));
            hipLaunchKernelGGL(piece_stats_kernel<T>, dim3(M), dim3(256), 0, s, at<float>(L.z), (int64_t)p.width, p.n, bias() ? bias() + p.v0 : nullptr,
                               at<int>(L.count), v.inv_tau, L.Mp, at<float>(L.stats) + (int64_t)k * 3 * L.Mp);
            REV_HIP(hipGetLastError());
        }
        ProfScope ps(K_REDUCE, s, 12.0 * L.Mp * L.pieces);
        hipLaunchKernelGGL(losses_kernel, blocks_of(M, 4), dim3(256), 0, s, v, at<float>(L.stats), L.pieces, L.Mp, at<float>(L.zs), loss_ce, loss_kd,
                           lse, lse + M);
        REV_HIP(hipGetLastError());
        return REV_OK;
    }

    int backward(const void* X, const float* lse, const float* dce, const float* dkd, void* dX, void* dparams) {
        RC(prepare(X));
        hipLaunchKernelGGL(coef_kernel, blocks_of(M, 256), dim3(256), 0, s, v, flags(), lse, lse + M, dce, dkd, at<float4>(L.coef));
        REV_HIP(hipGetLastError());
        const bool gb = c.grad_mode == REV_MODE_BF16;
        for (int k = 0; k < L.pieces; ++k) {
            Piece p;
            RC(piece(k, &p));
            RC(logits(p));
            T* dz = at<T>(L.dz);
            hipLaunchKernelGGL(piece_dz_kernel<T>, dim3((unsigned)((p.width + 255) / 256 * L.Mp)), dim3(256), 0, s, at<float>(L.z), (int64_t)p.width, p.n,
                               bias() ? bias() + p.v0 : nullptr, at<int>(L.count), at<float4>(L.coef), v.inv_tau, (int64_t)p.width, dz);
            REV_HIP(hipGetLastError());
            hipLaunchKernelGGL(sparse_dz_kernel<T>, blocks_of(M, 4), dim3(256), 0, s, v, at<float>(L.zs), at<float4>(L.coef), p.v0, p.n, dz,
                               (int64_t)p.width);
            REV_HIP(hipGetLastError());
            if (dX) {
                Epi e = {}; e.kind = EPI_PLAIN_F32; e.outf = at<float>(k ? L.dw : L.acc); e.ldo = D; e.solo = true;
                if constexpr (kBf16) RC(gemm_nn_bf16(s, dz, p.width, p.w, D, (int)L.Mp, D, p.width, e));
                else RC(gemm_nn_f32(s, dz, p.width, p.w, D, (int)L.Mp, D, p.width, e));
                if (k) {
                    hipLaunchKernelGGL(add_kernel, blocks_of(L.Mp * D, 256), dim3(256), 0, s, at<float>(L.dw), L.Mp * D, at<float>(L.acc));
                    REV_HIP(hipGetLastError());
                }
            }
            if (dparams) {
                float* dw = at<float>(L.dw);
                if constexpr (kBf16) {
                    const WgradItem it = {dz, p.width, at<T>(L.xc), L.Dp, p.width, D, dw, nullptr};
                    RedSeg segs[RED_MAX_SEGS];
                    int nseg = 0;
                    RC(gemm_wgrad_bf16_group(s, &it, 1, (int)L.Mp, at<float>(L.wg), L.wg_elems, segs, &nseg));
                    RC(reduce_multi(s, segs, nseg));
                } else {
                    const WgradF32Item it = {dz, p.width, at<T>(L.xc), L.Dp, p.width, D, dw, nullptr};
                    RC(gemm_wgrad_f32_group(s, &it, 1, (int)L.Mp));
                }
                hipLaunchKernelGGL(store_grad_kernel, blocks_of((int64_t)p.n * D, 256), dim3(256), 0, s, dw, (int64_t)p.n * D, dparams,
                                   (int64_t)p.v0 * D, gb);
                REV_HIP(hipGetLastError());
                if (c.bias) {
                    hipLaunchKernelGGL(piece_colsum_kernel<T>, blocks_of(p.n, 256), dim3(256), 0, s, dz, (int64_t)p.width, p.n, at<int>(L.count), dparams,
                                       (int64_t)V * D + p.v0, gb);
                    REV_HIP(hipGetLastError());
                }
            }
        }
        if (dX) {
            hipLaunchKernelGGL(scatter_dx_kernel<T>, blocks_of((int64_t)M * D / 4, 256), dim3(256), 0, s, at<float>(L.acc), at<int>(L.place), M, D, (T*)dX);
            REV_HIP(hipGetLastError());
        }
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
    if (cfg->mode == REV_MODE_BF16) return VocabRunner<bf16>(*cfg, params, ws, s, labels, idx, logits).forward(X, loss_ce, loss_kd, lse);
    return VocabRunner<float>(*cfg, params, ws, s, labels, idx, logits).forward(X, loss_ce, loss_kd, lse);
}
static int vocab_backward(const rev_vocab_cfg* cfg, const void* params, const void* X, const int* labels, const int* idx, const float* logits,
                          const float* lse, const float* dce, const float* dkd, void* dX, void* dparams, void* ws, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    if (cfg->mode == REV_MODE_BF16) return VocabRunner<bf16>(*cfg, params, ws, s, labels, idx, logits).backward(X, lse, dce, dkd, dX, dparams);
    return VocabRunner<float>(*cfg, params, ws, s, labels, idx, logits).backward(X, lse, dce, dkd, dX, dparams);
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
