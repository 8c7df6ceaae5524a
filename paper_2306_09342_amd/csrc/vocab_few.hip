// Logits of few rows: what vocab_gemm.hip's tiles would leave empty.
//
// A workgroup takes 32 MB rows and 64 entries; its four wavefronts share the contraction, 64 bytes of every row in turn, out of a
// ring in LDS that only the wavefront uses (direct-to-LDS loads, waited for with its own counter, no barrier).  Two workgroups per
// CU: the loads of one run beside the other's end.  The four partial tiles meet in LDS, a few entries of a row per thread,
// which the softmax statistics or dz are made of.  (Both operands read straight into registers instead: every lane of such a load is
// in another row, and the address unit took 12 us for 64 rows and 1000 entries of 768, 31 for one row and 50265.)
//
// What bounds it: reading W.
#include "mfma.h"
#include "vocab.h"

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
    const VocabPlan pl = *p.plan;
    const int lane = threadIdx.x & 63, g = lane >> 5, fr = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = xcd_remap(blockIdx.x, gridDim.x), nt = tile / p.blocks_m, m0 = (tile - nt * p.blocks_m) * ROWS, n0 = nt * 64;
    if (!GRAD && m0 >= pl.count) return;
    const int count = pl.count;

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
        for (int t = 0; t < 2 * MB; ++t) src[t] = reinterpret_cast<const char*>(p.x + (int64_t)min(m0 + 16 * t + lr, p.rows_x - 1) * p.Dp) + unit * 16;
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
        LabelDz y = {-1, 0.f};
        if (i < count) {
            c = p.coef[i];
            if (p.label_dz) y = p.label_dz[i];
        }
        const int64_t ldz = p.ldz ? p.ldz : pl.width;
        T* out = p.dz + i * ldz + c0;
        float d[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            d[e] = i < count && c0 + e < p.V ? dense_dz(c, z[e], p.inv_tau) : 0.f;
            if (c0 + e == y.label) d[e] = y.dz;
        }
#pragma unroll
        for (int e = 0; e < EPT; e += 4)
            if (c0 + e < ldz && i < p.rows_out) {
                if constexpr (sizeof(T) == 4) {
                    *reinterpret_cast<f32x4_t*>(out + e) = f32x4_t{d[e], d[e + 1], d[e + 2], d[e + 3]};
                } else {
                    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<bf16x4*>(out + e) = bf16x4{(__bf16)d[e], (__bf16)d[e + 1], (__bf16)d[e + 2], (__bf16)d[e + 3]};
                }
            }
    }
}

template <typename T> int few_logits(hipStream_t s, FewRows<T> p, bool grad, bool dual, int rows, int64_t width) {
    ProfScope ps(K_VOCAB, s, 2.0 * rows * p.V * p.D);
    // 32 rows per workgroup instead of 64 as long as all of them run at once: the matrix cores of a CU then have half as much to do
    const bool one = rows <= 32 || (int64_t)((rows + 31) / 32) * ((width + 63) / 64) <= 512;
    const int covered = grad ? p.rows_out : rows;
    p.blocks_m = (covered + (one ? 31 : 63)) / (one ? 32 : 64);
    const dim3 grid((unsigned)(p.blocks_m * ((width + 63) / 64))), block(256);
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
template int few_logits<bf16>(hipStream_t, FewRows<bf16>, bool, bool, int, int64_t);
template int few_logits<float>(hipStream_t, FewRows<float>, bool, bool, int, int64_t);

}  // namespace rev
