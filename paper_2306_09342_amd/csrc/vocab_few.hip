// Logits of few rows: what vocab_gemm.hip's tiles would leave empty.
//
// A workgroup takes 32 MB rows and 64 entries; its four wavefronts share the contraction, 64 bytes of every row in turn, out of a
// ring in LDS that only the wavefront uses (direct-to-LDS loads, waited for with its own counter, no barrier).  Two workgroups per
// CU: the loads of one run beside the other's end.  The four partial tiles meet in LDS, a few entries of a row per thread,
// which the softmax statistics or dz are made of.  (Both operands read straight into registers instead: every lane of such a load is
// in another row, and the address unit took 12 us for 64 rows and 1000 entries of 768, 31 for one row and 50265.)
//
// Forward the rows are taken from X as they lie, those that do not count too (their results are not kept): nothing has to be selected first,
// and the logits that the rows name are dot products in workgroups ahead of the others.  (Selected, copied and their named logits
// taken by a launch of its own: 26 us for one row and 41 for 16 rows with 8 named entries each, in the place of 20 and 29.)
//
// What bounds it: reading W.  One row of 768, 50265 entries, bf16 (77 MB): 19 us, 4.1 TB/s; 16 rows of 1024 (103 MB): 22 us.
#include "mfma.h"
#include "vocab.h"
#include <algorithm>

namespace rev {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// 16 bytes of a row of each operand: 8 bf16 or 4 float32 of the contraction
template <typename T> __device__ __forceinline__ f32x16_t few_product(u32x4_t a, u32x4_t b, f32x16_t c) {
    if constexpr (sizeof(T) == 2) {
        return mfma32(as_bf16x8(a), as_bf16x8(b), c);
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) c = mfma_f32(__uint_as_float(a[s]), __uint_as_float(b[s]), c);
        return c;
    }
}

template <int MB> struct FewCfg {
    static constexpr int ROWS = 32 * MB, PITCH = 68, STAGES = MB == 1 ? 3 : 2, LOADS = 2 * MB + 4, STAGE = LOADS * 1024;
    static constexpr int RING = 4 * STAGES * STAGE, RED = 4 * ROWS * PITCH * 4, LDS = RING > RED ? RING : RED;
};

template <typename T, bool GRAD, bool DUAL, int MB>
__global__ __launch_bounds__(256, 2) void few_logits_kernel(FewRows<T> p) {
    using C = FewCfg<MB>;
    constexpr int NB = 2, ROWS = C::ROWS, PITCH = C::PITCH, NS = C::STAGES, LOADS = C::LOADS, TPR = 256 / ROWS, EPT = 64 / TPR;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    float* red = reinterpret_cast<float*>(smem);
    const int lane = threadIdx.x & 63, g = lane >> 5, fr = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (!GRAD && (int)blockIdx.x < p.named_blocks) {               // four named entries of a row per wavefront
        const int from = p.named.labels ? 0 : 1, per = (p.named.K + 4 - from) >> 2, item = blockIdx.x * 4 + wave, r = item / per;
        if (r < p.rows) named_logits(p.named, p.x + (int64_t)r * p.ldx, p.w, p.D, r, from + (item - r * per) * 4, p.zs + (int64_t)r * (p.named.K + 1));
        return;
    }
    const int ahead = GRAD ? 0 : p.named_blocks, tile = xcd_remap(blockIdx.x - ahead, gridDim.x - ahead), nt = tile / p.blocks_m, m0 = (tile - nt * p.blocks_m) * ROWS, n0 = nt * 64;
    const int count = GRAD ? p.plan->count : p.rows;

    f32x16_t acc[NB][MB];
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[j][i][v] = 0.f;
    if (m0 < count && n0 < p.V) {
        // a load takes 16 rows of four 16-byte units, unit u of row r at position u ^ ((r >> 1) & 3); rows beyond the last read it again,
        // units beyond the row zeros
        const int units = p.D * (int)sizeof(T) / 16, lr = lane >> 2, unit = (lane & 3) ^ ((lr >> 1) & 3);
        const char* src[LOADS];
#pragma unroll
        for (int t = 0; t < 2 * MB; ++t) src[t] = reinterpret_cast<const char*>(p.x + (int64_t)min(m0 + 16 * t + lr, p.rows_x - 1) * p.ldx) + unit * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t) src[2 * MB + t] = reinterpret_cast<const char*>(p.w + (int64_t)min(n0 + 16 * t + lr, p.V - 1) * p.D) + unit * 16;
        unsigned char* ring = smem + wave * NS * C::STAGE;
        const unsigned lds0 = (unsigned)(uintptr_t)LDS_PTR(unsigned char, ring);
        const char* zero = reinterpret_cast<const char*>(g_zero_chunk);
        auto issue = [&](int c, int stage) {
            const bool in = c * 4 + unit < units;
#pragma unroll
            for (int t = 0; t < LOADS; ++t) dma16_ptr(in ? src[t] + c * 64 : zero, lds0 + stage * C::STAGE + t * 1024);
        };
        const int chunks = (units + 3) / 4, mine = wave < chunks ? (chunks - wave + 3) / 4 : 0;
#pragma unroll
        for (int k = 0; k < NS; ++k)
            if (k < mine) issue(wave + 4 * k, k);
        int st = 0;
        for (int k = 0; k < mine; ++k) {
            if (k + NS <= mine) wait_vm<(NS - 1) * LOADS>();       // this stage's loads are the oldest
            else wait_vm<0>();
            const unsigned char* at = ring + st * C::STAGE;
            u32x4_t xf[2][MB], wf[2][NB];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int pos = fr * 64 + (((2 * q + g) ^ ((fr >> 1) & 3)) << 4);
#pragma unroll
                for (int i = 0; i < MB; ++i) xf[q][i] = *reinterpret_cast<const u32x4_t*>(at + i * 2048 + pos);
#pragma unroll
                for (int j = 0; j < NB; ++j) wf[q][j] = *reinterpret_cast<const u32x4_t*>(at + (MB + j) * 2048 + pos);
            }
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int i = 0; i < MB; ++i) acc[j][i] = few_product<T>(wf[q][j], xf[q][i], acc[j][i]);
            wait_lds();                                            // the stage has been read: it may be refilled
            if (k + NS < mine) issue(wave + 4 * (k + NS), st);
            st = st + 1 == NS ? 0 : st + 1;
        }
    }
    __syncthreads();                                               // the partial tiles take the rings' place
    float* part = red + wave * ROWS * PITCH;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4_t*>(part + (32 * i + fr) * PITCH + 32 * j + 8 * q + 4 * g) =
                    f32x4_t{acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
    __syncthreads();
    const int row = threadIdx.x / TPR, sub = threadIdx.x % TPR, i = m0 + row, c0 = n0 + sub * EPT;
    float z[EPT];
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
        f32x4_t s = *reinterpret_cast<const f32x4_t*>(red + row * PITCH + sub * EPT + e);
#pragma unroll
        for (int k = 1; k < 4; ++k) s += *reinterpret_cast<const f32x4_t*>(red + (k * ROWS + row) * PITCH + sub * EPT + e);
#pragma unroll
        for (int k = 0; k < 4; ++k) z[e + k] = s[k];
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
        if (c0 + e >= p.V) z[e] = -INFINITY;
        else if (p.bias) z[e] += to_f(p.bias[c0 + e]);
    }
    if constexpr (!GRAD) {
        float m = z[0];
#pragma unroll
        for (int e = 1; e < EPT; ++e) m = fmaxf(m, z[e]);
#pragma unroll
        for (int o = 1; o < TPR; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        const float ref = m == -INFINITY ? 0.f : m, rate0 = !DUAL && p.losses == LOSS_KD ? p.inv_tau : 1.f;
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            s0 += expf((z[e] - ref) * rate0);
            if (DUAL) s1 += expf((z[e] - ref) * p.inv_tau);
        }
#pragma unroll
        for (int o = 1; o < TPR; o <<= 1) {
            s0 += __shfl_xor(s0, o, 64);
            if (DUAL) s1 += __shfl_xor(s1, o, 64);
        }
        if (sub == 0 && i < count) {
            float* out = p.stats + i * p.stat_row + nt;
            out[0] = m;
            out[p.stat_kind] = s0;
            if (DUAL) out[2 * p.stat_kind] = s1;
        }
    } else {
        float4 c = make_float4(0.f, INFINITY, 0.f, INFINITY);
        int y = -1;
        if (i < count) {
            c = p.coef[i];
            if (p.label) y = p.label[i];
        }
        const int64_t ldz = p.tile_dz ? p.plan->width : p.ldz;
        float d[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            d[e] = i < count && c0 + e < p.V ? dense_dz(c, z[e], p.inv_tau) : 0.f;
            if (c0 + e == y) d[e] -= c.x;
        }
#pragma unroll
        for (int e = 0; e < EPT; e += 4) {
            if (c0 + e >= ldz || i >= p.rows_out) continue;
            const int64_t at = i * ldz + c0 + e;
            if (sizeof(T) == 2 && p.tile_dz) {
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<bf16x4*>(p.tile_dz + at) = bf16x4{(__bf16)d[e], (__bf16)d[e + 1], (__bf16)d[e + 2], (__bf16)d[e + 3]};
            } else {
                *reinterpret_cast<f32x4_t*>(p.dz + at) = f32x4_t{d[e], d[e + 1], d[e + 2], d[e + 3]};
            }
        }
    }
}

// The gradients of a range of the vocabulary and a group of columns from dz in float32, on the float32 matrix cores, so that dz is not
// rounded again:  dW[v, d] = sum over i of dz[i, v] x[i, d]  of the range's entries, and dx[i, d] = sum over the range of dz[i, v]
// W[v, d], to be added to the other ranges'.  The workgroup keeps the range's dz in LDS, where both products find their first
// operand; the second, rows of W and x, is read from memory as it lies, 128 bytes of two rows at a time (bf16: as pairs of columns,
// the two products of a pair one after the other).
//
// What bounds it: the float32 matrix cores and the LDS reads of their operands; with one row reading W and writing dW.  768 to 50265
// entries, float32: one row 67 us (4.6 TB/s of W and dW), 32 rows 87 us.
//
// ADD: a turn behind the first one, whose dx is added to what is there (a kernel of its own: the loads cost the others registers).
template <typename T, typename TG, int MB, bool ADD>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 3) void few_grads_kernel(FewRows<T> p, int want_dx, TG* dparams, int db, int apart) {
    constexpr int CS = 4 / sizeof(T), COLS = 32 * CS;              // columns per lane and word; of a block
    extern __shared__ __attribute__((aligned(16))) float dzs[];    // [rows up to whole 32][range + 1], 256 more for db
    const int lane = threadIdx.x & 63, g = lane >> 5, fr = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int count = __builtin_amdgcn_readfirstlane(p.plan->count);
    int block = blockIdx.x;
    if (apart) {                                                   // dW in the first half of the workgroups, dx in the second
        const int half = gridDim.x >> 1;
        if (block < half) want_dx = 0;
        else { block -= half; dparams = nullptr; }
    }
    const int r = block / p.col_groups, cg = block - r * p.col_groups, P = p.range + 1;
    const int v0 = (p.first + r) * p.range, nv = min(p.range, p.V - v0), rows32 = (count + 31) & ~31;
    // four entries of a row per thread and load, eight of these in flight (dz has whole quads, zeros behind the vocabulary)
    const int per = p.range >> 2, quads = rows32 * per;
    for (int k0 = threadIdx.x; k0 < quads; k0 += 2048) {
        f32x4_t u[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int k = k0 + 256 * q, i = k / per, c = (k - i * per) * 4;
            u[q] = i < count && v0 + c < p.ldz ? *reinterpret_cast<const f32x4_t*>(p.dz + i * p.ldz + v0 + c) : f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int k = k0 + 256 * q, i = k / per, c = (k - i * per) * 4;
            if (k < quads) {
#pragma unroll
                for (int e = 0; e < 4; ++e) dzs[i * P + c + e] = u[q][e];
            }
        }
    }
    __syncthreads();
    if (db && dparams && cg == 0) {                                // every eighth row per 32 threads, 32 entries at a time
        float (*sums)[32] = reinterpret_cast<float (*)[32]>(dzs + rows32 * P);
        const int c = threadIdx.x & 31, part = threadIdx.x >> 5;
        for (int vb = 0; vb < nv; vb += 32) {
            float s = 0.f;
#pragma unroll 4
            for (int i = part; i < rows32; i += 8) s += dzs[i * P + vb + c];
            sums[part][c] = s;
            __syncthreads();
            if (part == 0 && vb + c < nv) {
#pragma unroll
                for (int k = 1; k < 8; ++k) s += sums[k][c];
                dparams[(int64_t)p.V * p.D + v0 + vb + c] = from_f<TG>(s);
            }
            __syncthreads();
        }
    }
    const int blocks = (p.D + COLS - 1) / COLS;
    auto columns = [&](unsigned u, float (&f)[CS]) {
        if constexpr (CS == 1) f[0] = __uint_as_float(u);
        else { f[0] = __uint_as_float(u << 16); f[1] = __uint_as_float(u & 0xFFFF0000u); }
    };
    // (what differs between the lanes in 32 bits)
    auto word = [&](const T* at, unsigned offset) { return *reinterpret_cast<const unsigned*>(reinterpret_cast<const char*>(at) + offset); };
    auto clear = [&](f32x16_t& c) {
#pragma unroll
        for (int v = 0; v < 16; ++v) c[v] = 0.f;
    };
    if (const int b = cg * 4 + wave; b < blocks) {
        const int d = b * COLS + CS * fr, dc = min(d, p.D - CS);   // columns beyond D read the last ones again (never stored)
        const T* w = p.w + (int64_t)v0 * p.D;
        // up to 32 rows of x stay in registers
        constexpr int KEPT = MB == 1 ? 16 : 1;
        unsigned kept[KEPT];
        if (MB == 1 && dparams) {
#pragma unroll
            for (int s = 0; s < KEPT; ++s) kept[s] = 2 * s < count ? word(p.x, (unsigned)((2 * s + g) * p.ldx + dc) * sizeof(T)) : 0u;
        }
        for (int vb = 0; vb < nv && dparams; vb += 32) {
            f32x16_t acc[CS];
#pragma unroll
            for (int q = 0; q < CS; ++q) clear(acc[q]);
            if constexpr (MB == 1) {
                auto add = [&](int s, unsigned u) {
                    const float a = dzs[(2 * s + g) * P + vb + fr];    // (rows up to whole 32 are there)
                    float f[CS];
                    columns(u, f);
#pragma unroll
                    for (int q = 0; q < CS; ++q) acc[q] = mfma_f32(a, f[q], acc[q]);
                };
#pragma unroll
                for (int s = 0; s < KEPT; ++s)
                    if (2 * s < count) add(s, kept[s]);
            } else {
                // 32 rows at a time, as many as there are of dz; the next ones asked for first
                unsigned even[16], odd[16];
                auto load = [&](unsigned (&to)[16], int i0) {
                    const T* at = p.x + (int64_t)min(i0, p.rows_x - 32) * p.ldx;
#pragma unroll
                    for (int s = 0; s < 16; ++s) to[s] = word(at + 2 * s * p.ldx, (unsigned)(g * p.ldx + dc) * sizeof(T));
                    __builtin_amdgcn_sched_barrier(0);             // (the compiler moves them behind the products)
                };
                auto add = [&](unsigned (&u)[16], int i0) {
                    int at = (i0 + g) * P + vb + fr;
                    asm volatile("" : "+v"(at));                   // (no sixteen addresses kept over the loop)
#pragma unroll
                    for (int s = 0; s < 16; ++s) {
                        const float a = dzs[at + 2 * s * P];
                        float f[CS];
                        columns(u[s], f);
#pragma unroll
                        for (int q = 0; q < CS; ++q) acc[q] = mfma_f32(a, f[q], acc[q]);
                    }
                };
                load(even, 0);
                for (int i0 = 0; i0 < count; i0 += 64) {
                    load(odd, i0 + 32);
                    add(even, i0);
                    if (i0 + 32 >= count) break;
                    load(even, i0 + 64);
                    add(odd, i0 + 32);
                }
            }
            if (d < p.D) {
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int n = vb + 8 * (v >> 2) + 4 * g + (v & 3);
                    if (n >= nv) continue;
                    TG* out = dparams + (int64_t)(v0 + n) * p.D + d;
                    if constexpr (CS == 1) {
                        *out = from_f<TG>(acc[0][v]);
                    } else if constexpr (sizeof(TG) == 2) {
                        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
                        *reinterpret_cast<bf16x2_t*>(out) = bf16x2_t{(__bf16)acc[0][v], (__bf16)acc[1][v]};
                    } else {
                        *reinterpret_cast<float2*>(out) = make_float2(acc[0][v], acc[1][v]);
                    }
                }
            }
        }
        if (!want_dx || rows32 == 0) return;
        constexpr int DB = CS == 2 ? 1 : MB;                       // blocks of 32 rows at a time
        unsigned even[16], odd[16];                                // 32 entries; the next 32, of the range or for the next rows, asked for first
        f32x16_t acc[DB][CS];
        int m0 = 0, vb = 0;
        const unsigned both = (unsigned)(g * p.D + dc) * (unsigned)sizeof(T);
        auto load = [&](unsigned (&to)[16], int v) {
#pragma unroll
            for (int s = 0; s < 16; ++s)                           // rows beyond the range, where dz is 0, read its last one again
                to[s] = word(w + (int64_t)min(v + 2 * s, nv - 1) * p.D, v + 2 * s + 1 < nv ? both : (unsigned)dc * (unsigned)sizeof(T));
            __builtin_amdgcn_sched_barrier(0);
        };
        auto step = [&](unsigned (&u)[16], unsigned (&next)[16]) {
            load(next, vb + 32 < nv ? vb + 32 : 0);
            if (vb == 0) {
#pragma unroll
                for (int m = 0; m < DB; ++m)
#pragma unroll
                    for (int q = 0; q < CS; ++q) clear(acc[m][q]);
            }
            const float* a[DB];                                    // blocks beyond the last repeat it (not stored)
#pragma unroll
            for (int m = 0; m < DB; ++m) a[m] = dzs + (min(m0 + m * 32, rows32 - 32) + fr) * P + vb + g;
#pragma unroll
            for (int s = 0; s < 16; ++s) {
                float f[CS];
                columns(u[s], f);
#pragma unroll
                for (int m = 0; m < DB; ++m) {
                    const float z = a[m][2 * s];
#pragma unroll
                    for (int q = 0; q < CS; ++q) acc[m][q] = mfma_f32(z, f[q], acc[m][q]);
                }
            }
            vb += 32;
            if (vb < nv) return;
            if (d < p.D) {
#pragma unroll
                for (int m = 0; m < DB; ++m)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int i = m0 + m * 32 + 8 * (v >> 2) + 4 * g + (v & 3);
                        if (i >= count) continue;
                        float* out = p.parts + ((int64_t)r * p.rows + i) * p.D + d;
                        if constexpr (ADD) {
#pragma unroll
                            for (int q = 0; q < CS; ++q) acc[m][q][v] += out[q];
                        }
                        if constexpr (CS == 1) *out = acc[m][0][v];
                        else *reinterpret_cast<float2*>(out) = make_float2(acc[m][0][v], acc[m][1][v]);
                    }
            }
            vb = 0;
            m0 += 32 * DB;
        };
        load(even, 0);
        for (;;) {
            step(even, odd);
            if (m0 >= rows32) break;
            step(odd, even);
            if (m0 >= rows32) break;
        }
    }
}

// dX[r], 64 columns per workgroup: a sixteenth of the ranges' places per group of 16 lanes, added in order; zeros for a row that does not count.
template <typename T>
__global__ __launch_bounds__(256) void few_dx_rows_kernel(FewRows<T> p, const int* __restrict__ place, T* __restrict__ dX) {
    __shared__ f32x4_t sh[16][16];
    const int r = blockIdx.x, i = place[r], q = threadIdx.x & 15, k = threadIdx.x >> 4, d = blockIdx.y * 64 + q * 4;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if (i >= 0 && d < p.D) {
        const int per = (p.places + 15) >> 4, last = min(p.places, (k + 1) * per);
        const float* at = p.parts + (int64_t)i * p.D + d;
        const int64_t step = (int64_t)p.rows * p.D;
        for (int n = k * per; n < last; n += 8) {
            f32x4_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = n + u < last ? *reinterpret_cast<const f32x4_t*>(at + (n + u) * step) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < 8; ++u) s += v[u];
        }
    }
    sh[k][q] = s;
    __syncthreads();
    if (k || d >= p.D) return;
#pragma unroll
    for (int n = 1; n < 16; ++n) s += sh[n][q];
    T* out = dX + (int64_t)r * p.D + d;
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4_t*>(out) = s;
    } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4*>(out) = bf16x4{(__bf16)s[0], (__bf16)s[1], (__bf16)s[2], (__bf16)s[3]};
    }
}

// Ranges of the vocabulary and groups of columns: about 320 ranges, of at most 256 entries (of fewer where their dz would not leave LDS
// for two workgroups) and, from 5120 entries on, of no fewer than 64, each by as many workgroups as it has groups of four column blocks.  32 rows
// of 768 to 50265 entries, loss and gradients backward in us by entries per range and groups, bf16 / float32: 224, 2: 126 / 149; 224, 3: 121 / 143; 128,
// 3: 118 / 157; 64, 3: 129 / 178.  10007 entries in ranges of 32 / 64: 16 bf16 rows of 768 36 / 32, 128 float32 rows of 384 77 / 69.
// Several groups to a workgroup, 1024 of these / one each: 4 float32 rows of 1544 to 51456 entries 324 / 268, 32 of 728 to 129805 376 / 348, a bf16
// row of 2048 to 32000 104 / 107.
void few_ranges(int rows, int V, int D, int es, int* range, int* ranges, int* col_groups) {
    const int blocks32 = (V + 31) / 32, rows32 = (rows + 31) / 32 * 32;
    int per = blocks32 > 160 ? std::max(2, (blocks32 + 319) / 320) : 1;
    while (per > 1 && (per > 8 || rows32 * (per * 32 + 1) * 4 > 72 * 1024)) --per;
    *range = per * 32;
    *ranges = (blocks32 + per - 1) / per;
    *col_groups = ((D * es + 127) / 128 + 3) / 4;                  // of four blocks of columns
}

template <typename T> int few_logits(hipStream_t s, FewRows<T> p, bool grad, bool dual) {
    ProfScope ps(K_VOCAB, s, 2.0 * p.rows * p.V * p.D);
    // 32 rows per workgroup instead of 64 as long as all of them run at once: the matrix cores of a CU then have half as much to do
    const int tiles = grad && p.tile_dz ? (p.V + 255) / 256 * 4 : (p.V + 63) / 64, covered = grad ? p.rows_out : p.rows;
    const bool one = p.rows <= 32 || (int64_t)((p.rows + 31) / 32) * tiles <= 512;
    p.blocks_m = (covered + (one ? 31 : 63)) / (one ? 32 : 64);
    p.named_blocks = grad ? 0 : (int)(((int64_t)p.rows * ((p.named.K + (p.named.labels ? 4 : 3)) >> 2) + 31) / 32 * 8);
    const dim3 grid((unsigned)(p.named_blocks + p.blocks_m * tiles)), block(256);
#define FEW1(G, U, MB) do {                                                                                          \
        static LdsLimit lim;                                                                                         \
        if (int rc = lim.ensure(reinterpret_cast<const void*>(few_logits_kernel<T, G, U, MB>), FewCfg<MB>::LDS)) return rc; \
        hipLaunchKernelGGL((few_logits_kernel<T, G, U, MB>), grid, block, FewCfg<MB>::LDS, s, p);                    \
    } while (0)
#define FEW(G, U) do { if (one) FEW1(G, U, 1); else FEW1(G, U, 2); } while (0)
    if (grad) FEW(true, false);
    else if (dual) FEW(false, true);
    else FEW(false, false);
#undef FEW
#undef FEW1
    REV_HIP(hipGetLastError());
    return REV_OK;
}
template <typename T> int few_grads(hipStream_t s, FewRows<T> p, bool want_dx, void* dparams, bool grad_bf16, bool db) {
    ProfScope ps(K_VOCAB, s, 2.0 * p.rows * p.V * p.D * (want_dx + (dparams != nullptr)));
    const int rows32 = (p.rows + 31) / 32 * 32, lds = rows32 * (p.range + 1) * 4 + 1024;
    // Few workgroups wait for memory most of the time: dW and dx in workgroups of their own.  Gradients in us, together / apart: float32, 128 rows,
    // D = 384, V = 1000 (96 workgroups): 34 / 29; 512, 768, 1000 (192): 80 / 71; 333, 200, 5003 (314): 88 / 85; 64, 768, 10007 (939): 80 / 82;
    // bf16, 8, 768, 10007 (939): 35 / 37.
    const int blocks = p.ranges * p.col_groups, apart = want_dx && dparams && blocks <= 384 && p.places == p.ranges;
    // Turns in float32 only: bf16 calls whose ranges would not all have a place go through tiles (few_backward: at most 21 MB of dx).
    const int turn = want_dx ? p.places : p.ranges;
    constexpr bool turns = sizeof(T) == 4;
#define GRADS1(TG, MB, ADD) do {                                                                                       \
        static LdsLimit lim;                                                                                           \
        if (int rc = lim.ensure(reinterpret_cast<const void*>(few_grads_kernel<T, TG, MB, ADD>), 160 * 1024)) return rc; \
        const dim3 grid((unsigned)((std::min(turn, p.ranges - p.first) * p.col_groups) << apart));                     \
        hipLaunchKernelGGL((few_grads_kernel<T, TG, MB, ADD>), grid, dim3(256), lds, s, p, (int)want_dx, (TG*)dparams, (int)db, apart); \
        REV_HIP(hipGetLastError());                                                                                    \
    } while (0)
#define GRADS(TG, MB) do {                                                                                             \
        p.first = 0;                                                                                                   \
        GRADS1(TG, MB, false);                                                                                         \
        for (p.first = turn; turns && p.first < p.ranges; p.first += turn) GRADS1(TG, MB, turns);                      \
        return REV_OK;                                                                                                 \
    } while (0)
    if constexpr (sizeof(T) == 2)
        if (grad_bf16) { if (rows32 == 32) GRADS(bf16, 1); else GRADS(bf16, 2); }
    if (rows32 == 32) GRADS(float, 1);
    GRADS(float, 2);
#undef GRADS
#undef GRADS1
}
template <typename T> int few_dx_rows(hipStream_t s, const FewRows<T>& p, const int* place, T* dX) {
    ProfScope ps(K_REDUCE, s, 4.0 * p.places * p.rows * p.D);
    hipLaunchKernelGGL(few_dx_rows_kernel<T>, dim3(p.rows, (p.D + 63) / 64), dim3(256), 0, s, p, place, dX);
    REV_HIP(hipGetLastError());
    return REV_OK;
}
#define BOTH(T)                                                                       \
    template int few_logits<T>(hipStream_t, FewRows<T>, bool, bool);                  \
    template int few_grads<T>(hipStream_t, FewRows<T>, bool, void*, bool, bool);      \
    template int few_dx_rows<T>(hipStream_t, const FewRows<T>&, const int*, T*);
BOTH(bf16)
BOTH(float)
#undef BOTH

}  // namespace rev
