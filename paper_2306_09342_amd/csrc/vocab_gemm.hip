// The products of the losses over a vocabulary in bf16, 256x256 tiles:
//   logits   z[i, v] = <x_i, W_v> + b_v       x [rows, Dp] and W [V, D] along the contraction; never stored:
//              forward    a row's maximum and sum of exponentials over half a tile's entries leave the kernel,
//              backward   dz of a piece of the vocabulary does, in bf16 (float32: in three parts);
//   dx       dx[i, d] = sum over v of dz[i, v] W[v, d], the vocabulary cut into ranges where there are few tiles;
//   dw       dW[v, d] = sum over i of dz[i, v] x[i, d], the rows cut into ranges where there are few tiles.
//
// dz is rounded to bf16 once, from float32, whatever the type of dparams: as an operand it meets W and X, which have as many bits.  Against exact
// results dX and dW are then off by 0.0023 of their norm; with float32 products, rounded at the end, by 0.0017.  Two parts of dz would be twice
// the stages of dx and dw: 8192 rows of 1024 to 131072 entries 3.3 ms more, on 7.1.
//
// One workgroup of 8 wavefronts per CU, 128 x 64 of the tile per wavefront.  A stage is 64 of the contraction; it travels as four
// parts of 16 KB (two halves of each operand) through two stages of LDS.  A part is requested again, for the stage after
// next, as soon as everybody has read it, so seven phases of products pass between a request and its use.  A stage is four phases of
// one quadrant each; the two wavefronts of a SIMD are half a phase apart, so that one multiplies while the other reads.
//
// float32 operands come as three bf16 parts each (split3), and the products whose parts' indices add to at most 2 are summed, the small
// ones first: six times the stages of bf16 operands, and 2^-23 of |x||w| left out.  The float32 matrix cores take sixteen times the cycles
// of the bf16 ones.
//
// The number of rows, and what follows from it (tiles, width of a piece, ranges), is read from the device (VocabPlan): a workgroup
// that finds no tile ends at once.
#include "mfma.h"
#include "vocab.h"
#include <algorithm>
#include <type_traits>

namespace rev {

constexpr int VG_PART = 16384, VG_LDS = 8 * VG_PART, VG_SIDE = 2048;
template <int V> using vg_int = std::integral_constant<int, V>;
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// The part of each operand that a stage takes, and the stage within it: six products of parts in turn, `stages` of each.
template <int P> struct Parts {
    int stages;
    __device__ __forceinline__ int term(int kt) const {
        if (P == 1) return 0;
        return (kt >= stages) + (kt >= 2 * stages) + (kt >= 3 * stages) + (kt >= 4 * stages) + (kt >= 5 * stages);
    }
    __device__ __forceinline__ int a(int t) const { return P == 1 ? 0 : (0x118 >> (2 * t)) & 3; }    // 0 2 1 0 1 0
    __device__ __forceinline__ int b(int t) const { return P == 1 ? 0 : (0x052 >> (2 * t)) & 3; }    // 2 0 1 1 0 0
    __device__ __forceinline__ int within(int kt, int t) const { return P == 1 ? kt : kt - t * stages; }
    __device__ __forceinline__ int total() const { return P == 1 ? stages : 6 * stages; }
};
struct TileLane {
    int lane, wave, wm, wn, g, fr;
    __device__ __forceinline__ TileLane() {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wm = wave & 1; wn = wave >> 1; g = lane >> 5; fr = lane & 31;
    }
    // A wavefront-wide load of an operand that lies along the contraction takes 8 rows of 8 chunks, of one that lies across it 4 rows
    // of 16 chunks: the row and the byte within it that this lane takes.
    __device__ __forceinline__ int row_along() const { return wave * 8 + (lane >> 3); }
    __device__ __forceinline__ int byte_along() const { return ((lane & 7) ^ ((row_along() >> 1) & 7)) << 4; }
    __device__ __forceinline__ int row_across() const { return wave * 4 + (lane >> 4); }
    __device__ __forceinline__ int byte_across() const { return ((lane & 15) ^ (4 * (row_across() & 3))) << 4; }
};

// acc[h][j][i] += the products of B half h (32-entry block i of this wavefront's 64) and A half j over nst stages, an even number,
// at least two.  Accumulator register v of lane (g, fr) is B entry h 128 + wm 64 + i 32 + 8 (v / 4) + 4 g + v % 4, A entry
// j 128 + wn 32 + fr.  AKM / BKM: the operand lies across the contraction.  issue_x(half, stage, address in LDS) requests a part.
// request_stages has asked for the first two stages; what the wavefront has asked of memory since then is only waited for longer.
// In LDS: B0 B1 of stage 0, B0 B1 of stage 1, then the same of A.
template <class IssueA, class IssueB>
__device__ __forceinline__ void request_stages(unsigned char* smem, const TileLane& t, const IssueA& issue_a, const IssueB& issue_b) {
    const unsigned lds_w = (unsigned)(uintptr_t)LDS_PTR(unsigned char, smem) + t.wave * 1024;
    using H0 = vg_int<0>; using H1 = vg_int<1>;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const unsigned b = lds_w + kt * (2 * VG_PART), a = b + 4 * VG_PART;
        issue_b(H0{}, kt, b); issue_a(H0{}, kt, a); issue_a(H1{}, kt, a + VG_PART); issue_b(H1{}, kt, b + VG_PART);
    }
}
template <bool AKM, bool BKM, class IssueA, class IssueB>
__device__ __forceinline__ void tile_products(unsigned char* smem, const TileLane& t, const IssueA& issue_a, const IssueB& issue_b, int nst,
                                              f32x16_t (&acc)[2][2][2]) {
    const unsigned lds0 = (unsigned)(uintptr_t)LDS_PTR(unsigned char, smem), lds_w = lds0 + t.wave * 1024;
    const int grp = t.wave >> 2;
    auto request_b = [&](auto half, int kt) { issue_b(half, kt, lds_w + (kt & 1) * (2 * VG_PART) + decltype(half)::value * VG_PART); };
    auto request_a = [&](auto half, int kt) { issue_a(half, kt, lds_w + 4 * VG_PART + (kt & 1) * (2 * VG_PART) + decltype(half)::value * VG_PART); };
    using H0 = vg_int<0>; using H1 = vg_int<1>;

    unsigned a_addr[4], b_addr[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        const int koff = ((2 * kk + t.g) ^ ((t.fr >> 1) & 7)) << 4;
        a_addr[kk] = lds0 + 4 * VG_PART + (t.wn * 32 + t.fr) * 128 + koff;
        b_addr[kk] = lds0 + (t.wm * 64 + t.fr) * 128 + koff;
    }
    {
        const int jj = t.lane & 15, qq = t.lane >> 4, r = (qq >> 1) * 8 + (jj >> 2), c = (qq & 1) * 16 + 4 * (jj & 3);
        auto at = [&](int col) { return lds0 + r * 256 + (((col >> 3) ^ (4 * (r & 3))) << 4) + (col & 7) * 2; };
        if (AKM) a_addr[0] = at(t.wn * 32 + c) + 4 * VG_PART;
        if (BKM) {
            b_addr[0] = at(t.wm * 64 + c);
            b_addr[1] = at(t.wm * 64 + 32 + c);
        }
    }
    u32x4_t b0[4][2], b1[4][2], a0[4], a1[4];
    auto read_tr = [&](unsigned addr, auto off_tag) {
        constexpr int off = decltype(off_tag)::value;
        return join64(lds_read_tr16_b64(addr, off), lds_read_tr16_b64(addr, off + 1024));
    };
    auto read_b = [&](u32x4_t (&f)[4][2], auto half_tag, auto par_tag) {
        constexpr int off = decltype(half_tag)::value * VG_PART + decltype(par_tag)::value * (2 * VG_PART);
        if constexpr (BKM) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f[0][i] = read_tr(b_addr[i], vg_int<off>{});
                f[1][i] = read_tr(b_addr[i], vg_int<off + 4096>{});
                f[2][i] = read_tr(b_addr[i], vg_int<off + 8192>{});
                f[3][i] = read_tr(b_addr[i], vg_int<off + 12288>{});
            }
        } else {
            f[0][0] = lds_read_b128(b_addr[0], off); f[0][1] = lds_read_b128(b_addr[0], off + 4096);
            f[1][0] = lds_read_b128(b_addr[1], off); f[1][1] = lds_read_b128(b_addr[1], off + 4096);
            f[2][0] = lds_read_b128(b_addr[2], off); f[2][1] = lds_read_b128(b_addr[2], off + 4096);
            f[3][0] = lds_read_b128(b_addr[3], off); f[3][1] = lds_read_b128(b_addr[3], off + 4096);
        }
    };
    auto read_a = [&](u32x4_t (&f)[4], auto half_tag, auto par_tag) {
        constexpr int off = decltype(half_tag)::value * VG_PART + decltype(par_tag)::value * (2 * VG_PART);
        if constexpr (AKM) {
            f[0] = read_tr(a_addr[0], vg_int<off>{});
            f[1] = read_tr(a_addr[0], vg_int<off + 4096>{});
            f[2] = read_tr(a_addr[0], vg_int<off + 8192>{});
            f[3] = read_tr(a_addr[0], vg_int<off + 12288>{});
        } else {
            f[0] = lds_read_b128(a_addr[0], off);
            f[1] = lds_read_b128(a_addr[1], off);
            f[2] = lds_read_b128(a_addr[2], off);
            f[3] = lds_read_b128(a_addr[3], off);
        }
    };
    auto pin_b = [&](u32x4_t (&f)[4][2]) {
        asm volatile("" : "+v"(f[0][0]), "+v"(f[0][1]), "+v"(f[1][0]), "+v"(f[1][1]), "+v"(f[2][0]), "+v"(f[2][1]), "+v"(f[3][0]), "+v"(f[3][1]));
    };
    auto pin_a = [&](u32x4_t (&f)[4]) { asm volatile("" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3])); };
    auto barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](u32x4_t (&fb)[4][2], u32x4_t (&fa)[4], f32x16_t (&c)[2]) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i) c[i] = mfma32(as_bf16x8(fb[kk][i]), as_bf16x8(fa[kk]), c[i]);
        __builtin_amdgcn_s_setprio(0);
    };
    // kind 0 requests as it goes; kind 1 is the last stage but one, kind 2 the last.  8 loads of a stage per wavefront, 2 per part.
    auto stage = [&](auto par_tag, auto kind_tag, int kt) {
        constexpr int par = decltype(par_tag)::value, kind = decltype(kind_tag)::value;
        using SP = vg_int<par>; using NP = vg_int<1 - par>;
        read_a(a0, H0{}, SP{});
        if (kind == 0) request_b(H0{}, kt + 2);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kind == 0 ? 12 : kind == 1 ? 10 : 2) : "memory");
        pin_a(a0);
        barrier();
        products(b0, a0, acc[0][0]);
        barrier();

        read_a(a1, H1{}, SP{});
        if (kind == 0) request_a(H0{}, kt + 2);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kind == 0 ? 12 : kind == 1 ? 8 : 0) : "memory");
        pin_a(a1);
        barrier();
        products(b0, a1, acc[0][1]);
        barrier();

        read_b(b1, H1{}, SP{});
        if (kind == 0) request_a(H1{}, kt + 2);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kind == 0 ? 12 : kind == 1 ? 6 : 0) : "memory");
        pin_b(b1);
        barrier();
        products(b1, a1, acc[1][1]);
        barrier();

        if (kind != 2) read_b(b0, H0{}, NP{});
        if (kind == 0) request_b(H1{}, kt + 2);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kind == 0 ? 12 : kind == 1 ? 4 : 0) : "memory");
        if (kind != 2) pin_b(b0);
        barrier();
        products(b1, a0, acc[1][0]);
        barrier();
    };
    wait_vm<12>();                                                 // B0 and A0 of stage 0 have landed
    barrier();
    read_b(b0, H0{}, vg_int<0>{});
    wait_lds();
    pin_b(b0);
    barrier();
    if (grp) barrier();                                            // half a phase behind
    int kt = 0;
    for (; kt + 3 < nst; kt += 2) {
        stage(vg_int<0>{}, vg_int<0>{}, kt);
        stage(vg_int<1>{}, vg_int<0>{}, kt + 1);
    }
    stage(vg_int<0>{}, vg_int<1>{}, kt);
    stage(vg_int<1>{}, vg_int<2>{}, kt + 1);
    if (!grp) barrier();
}

// The tiles of a launch of as many workgroups as run at once: each XCD (workgroups b, b + 8, ...) has one run of them, in which its
// workgroups go side by side, so that tiles which share an operand meet in its L2.
struct TileRun {
    int start, size, next, step;
    __device__ __forceinline__ TileRun(int tiles) {
        const int x = blockIdx.x & 7, per = tiles >> 3, rem = tiles & 7;
        start = x * per + min(x, rem);
        size = per + (x < rem);
        next = blockIdx.x >> 3;
        step = ((int)gridDim.x - x + 7) >> 3;
    }
    __device__ __forceinline__ bool done() const { return next >= size; }
    __device__ __forceinline__ int tile() const { return start + next; }
};

__device__ __forceinline__ void clear(f32x16_t (&acc)[2][2][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[h][j][i][v] = 0.f;
}

constexpr float LOG2E = 1.44269504088896341f;

// 16 accumulator registers as bf16 to 32 consecutive entries, 8 at a time: lanes g = 0 and 1 hold entries 0..3 and 4..7 of every
// eight; exchanged, each has all of one: g = 0 of the first of a pair of eights, g = 1 of the second.  `out`: of lane g's
// first eight.
__device__ __forceinline__ void store_eights(bf16* out, const f32x16_t& d, bool low = true, bool high = true) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    unsigned w[4][2];                                              // [v / 4][pair]
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const bf16x2_t b = {(__bf16)d[4 * q + 2 * k], (__bf16)d[4 * q + 2 * k + 1]};
            w[q][k] = __builtin_bit_cast(unsigned, b);
        }
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
        const u32x2_t x0 = __builtin_amdgcn_permlane32_swap(w[q][0], w[q + 1][0], false, false);
        const u32x2_t x1 = __builtin_amdgcn_permlane32_swap(w[q][1], w[q + 1][1], false, false);
        if (q == 0 ? low : high) *reinterpret_cast<u32x4_t*>(out + 8 * q) = u32x4_t{x0[0], x1[0], x0[1], x1[1]};
    }
}

// Maximum of a row's logits (N blocks of 16 of each of the lanes g = 0, 1) and the sums of exp2((z - maximum) e) for one or two e.
template <bool DUAL, int N>
__device__ __forceinline__ void row_stats(const f32x16_t (&z)[N], float e0, float e1, float* out, int64_t kind, bool store) {
    float m = -INFINITY;
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) m = fmaxf(m, z[b][v]);
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float ref = m == -INFINITY ? 0.f : m;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const float d = z[b][v] - ref;                         // first: a lowest value times a scale may overflow
            s0 += __builtin_amdgcn_exp2f(d * e0);
            if (DUAL) s1 += __builtin_amdgcn_exp2f(d * e1);
        }
    s0 += __shfl_xor(s0, 32, 64);
    if (DUAL) s1 += __shfl_xor(s1, 32, 64);
    if (store) {
        out[0] = m;
        out[kind] = s0;
        if (DUAL) out[2 * kind] = s1;
    }
}

// dz of 16 entries of a row, those of lane g of 32, from its coefficients (without DUAL: the one exponential's; both losses have the
// same at tau = 1), less the row's weight at its label, entry `at` of the lane's; to `out`, where lane g's first eight of them go.
template <bool DUAL, int P>
__device__ __forceinline__ void dz_block(const f32x16_t& z, const float4& c, float rate0, float inv_tau, int at, bf16* out, int64_t part_dz) {
    f32x16_t d;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        d[v] = c.x * __builtin_amdgcn_exp2f(fmaf(z[v], rate0, -c.y) * LOG2E);
        if (DUAL) d[v] = fmaf(c.z, __builtin_amdgcn_exp2f(fmaf(z[v], inv_tau, -c.w) * LOG2E), d[v]);
    }
    if (__any((unsigned)at < 28u)) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
            if (at == 8 * (v >> 2) + (v & 3)) d[v] -= c.x;
    }
#pragma unroll
    for (int part = 0; part < P; ++part) {
        store_eights(out + part * part_dz, d);
        if (part + 1 < P)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float r = d[v] - to_f(from_f<bf16>(d[v]));
                d[v] = fabsf(r) < INFINITY ? r : 0.f;
            }
    }
    __builtin_amdgcn_sched_barrier(0);                             // one block's registers at a time
}
__device__ __forceinline__ float4 one_coef(float4 c, int losses) {
    if (losses == LOSS_KD) { c.x = c.z; c.y = c.w; }
    if (losses == (LOSS_CE | LOSS_KD)) { c.x += c.z; c.y = c.y == INFINITY ? c.w : c.y; }    // the one that the row has, NaN too, or both alike
    return c;
}
// what replaces the accumulators' start at entry c0 + 8 (v / 4) + v % 4 of a tile that the vocabulary does not fill, or with biased
// quads that it does not: -infinity beyond entry n, the bias from `from`
template <int P>
__device__ __forceinline__ void start_at_end(f32x16_t& z, int c0, int n, int part_quad, const void* from) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int c = 8 * (v >> 2) + (v & 3);
        if (c >= n - c0) z[v] = -INFINITY;
        else if (from && c >= part_quad - c0) z[v] = P == 1 ? to_f(reinterpret_cast<const bf16*>(from)[c0 + c]) : reinterpret_cast<const float*>(from)[c0 + c];
    }
}

// The logits of tiles of 256 rows and 256 entries.  The accumulators start at the bias, and at -infinity beyond the vocabulary, so
// that neither costs the epilogue anything.  An accumulator's lane has one row of X in each half and 64 entries of it.  Forward: the
// sums are of exp(z - maximum), or exp((z - maximum) / tau) if only the teacher's loss is wanted; with DUAL the two are
// kept side by side.  Backward: dz, its label's entry p - 1 before it is rounded where labels alone are named.
// What bounds it: see the file's head; the epilogue is 128 exponentials a lane (twice that with DUAL), in which the matrix cores wait.  The first two
// stages of the next tile are under way meanwhile, and its bias.  8192 rows of 1024 to 131072 entries: forward 1.80 ms, 1.22 PFLOP/s, matrix cores busy
// 72 % of the time; backward 2.08 ms, 60 %, with 2.1 GB of dz to write.
template <bool GRAD, bool DUAL, int P>
__global__ __launch_bounds__(512, 2) void vocab_logits_kernel(VocabGemm p) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const TileLane t;
    const VocabPlan pl = *p.plan;
    const int tiles_m = __builtin_amdgcn_readfirstlane(pl.rows >> 8);
    const int width = GRAD ? __builtin_amdgcn_readfirstlane(pl.width) : p.span;
    const Piece piece = piece_of(p.piece, width, p.V);
    const int v0 = piece.v0, n = piece.n;
    const int tiles_n = (n + 255) >> 8;
    TileRun run(tiles_m * tiles_n);
    if (run.done()) return;
    const int gn = tiles_n <= 6 ? tiles_n : 4, per_group = gn * tiles_m;
    const int64_t lda = p.Dp, ldb = p.Dp;
    const unsigned va = (unsigned)(t.row_along() * lda * 2 + t.byte_along());
    const Parts<P> parts{p.Dp >> 6};
    const int64_t part_a = p.Mp * lda * 2, part_b = p.V * ldb * 2;

    // the tile whose operands are being requested, and what its epilogue will need
    int m0, n0;
    const char *a_base, *b_base;
    unsigned vb[2][2];
    // The rest goes to 2 KB of LDS of the wavefront's own: the bias of its 2 x 64 entries, coefficients and label of its 2 x 32 rows.  (Registers for it would be short of 20 in the main loop.)
    typedef typename std::conditional<P == 1, u32x2_t, f32x4_t>::type quad_t;
    unsigned char* side = smem + VG_LDS + t.wave * VG_SIDE;
    const unsigned side_lds = (unsigned)(uintptr_t)LDS_PTR(unsigned char, side);
    const int quad_end = p.V - v0 - 4;
    const bool biased = p.bias != nullptr, biased_quads = biased && p.V >= 4;
    auto take_tile = [&]() {
        const int tile = run.tile(), tg = tile / per_group, in_grp = tile - tg * per_group, gw = min(gn, tiles_n - tg * gn);
        m0 = __builtin_amdgcn_readfirstlane((in_grp / gw) * 256);
        n0 = __builtin_amdgcn_readfirstlane((tg * gn + in_grp % gw) * 256);
        a_base = reinterpret_cast<const char*>(p.x + m0 * lda);
        b_base = reinterpret_cast<const char*>(p.wp + (int64_t)(v0 + n0) * ldb);
        const int last = n - 1 - n0;                               // rows of W beyond it read that one again
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 2; ++q) vb[h][q] = (unsigned)(min(h * 128 + q * 64 + t.row_along(), last) * ldb * 2 + t.byte_along());
        if (biased_quads) {                                        // words beyond the vocabulary's whole quads are not used: its first
            const int c = v0 + n0 + (t.lane >> 5) * 128 + t.wm * 64 + (P == 1 ? 2 : 1) * t.fr;
#pragma unroll
            for (int q = 0; q < (P == 1 ? 1 : 2); ++q) {
                const int at = c + 32 * q;
                dma4_sbase(p.bias, (at <= p.V - (P == 1 ? 2 : 1) ? at : 0) * (P == 1 ? 2 : 4), side_lds + 256 * q);
            }
        }
        if (GRAD) {
            const int row = m0 + (t.lane >> 5) * 128 + t.wn * 32 + t.fr;
            dma16_sbase(p.coef, row * 16, side_lds + 512);
            if (p.label) dma4_sbase(p.label, row * 4, side_lds + 1536);
        }
    };
    auto issue_a = [&](auto half, int kt, unsigned lds) {
        const int term = parts.term(kt);
        const char* src = a_base + parts.a(term) * part_a + decltype(half)::value * 256 * lda + parts.within(kt, term) * 128;
        dma16_sbase(src, va, lds);
        dma16_sbase(src + 128 * lda, va, lds + 8192);
    };
    auto issue_b = [&](auto half, int kt, unsigned lds) {
        constexpr int h = decltype(half)::value;
        const int term = parts.term(kt);
        const char* src = b_base + parts.b(term) * part_b + parts.within(kt, term) * 128;
        dma16_sbase(src, vb[h][0], lds);
        dma16_sbase(src, vb[h][1], lds + 8192);
    };
    take_tile();
    request_stages(smem, t, issue_a, issue_b);
    for (;;) {
        f32x16_t acc[2][2][2];
        wait_vm<16>();                                             // what was asked for ahead of the two stages
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    // in memory's order for bf16 (two entries per word, 32 words of each half), by 32 entries for float32
                    const int c = i * 32 + 8 * k + 4 * t.g;
                    quad_t b = quad_t{};
                    if (biased_quads) b = *reinterpret_cast<const quad_t*>(side + (P == 1 ? h * 128 + c * 2 : i * 256 + h * 128 + (c & 31) * 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (P == 1) acc[h][0][i][4 * k + e] = __uint_as_float(e & 1 ? b[e >> 1] & 0xFFFF0000u : b[e >> 1] << 16);
                        else acc[h][0][i][4 * k + e] = b[e];
                    }
                }
        if (n0 + 256 > n) {                                        // the vocabulary's or the piece's last tile
            const char* from = biased ? reinterpret_cast<const char*>(p.bias) + (int64_t)v0 * (P == 1 ? 2 : 4) : nullptr;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) start_at_end<P>(acc[h][0][i], n0 + h * 128 + t.wm * 64 + i * 32 + 4 * t.g, n, (quad_end + 4) & ~3, from);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[h][1][i] = acc[h][0][i];
        const int tm0 = m0, tn0 = n0;
        tile_products<false, false>(smem, t, issue_a, issue_b, parts.total(), acc);
        float4 tc[2];
        int ty[2];
        if (GRAD) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // rows behind the last one that counts: 0 exp(z - infinity)
                tc[j] = make_float4(0.f, INFINITY, 0.f, INFINITY);
                ty[j] = -1;
                if (tm0 + j * 128 + t.wn * 32 + t.fr < pl.count) {
                    tc[j] = *reinterpret_cast<const float4*>(side + 512 + (j * 32 + t.fr) * 16);
                    if (p.label) ty[j] = *reinterpret_cast<const int*>(side + 1536 + (j * 32 + t.fr) * 4);
                }
            }
            wait_lds();                                            // the next tile's take their place
        }
        run.next += run.step;
        const bool more = !run.done();
        if (more) {
            take_tile();
            request_stages(smem, t, issue_a, issue_b);
        }

        if constexpr (!GRAD) {
            const float e1 = p.inv_tau * LOG2E, e0 = !DUAL && p.losses == LOSS_KD ? e1 : LOG2E;
            float* out = p.stats + (int64_t)((tn0 >> 7) + t.wm) * (DUAL ? 3 : 2) * p.Mp + tm0 + t.wn * 32 + t.fr;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const f32x16_t z[4] = {acc[0][j][0], acc[0][j][1], acc[1][j][0], acc[1][j][1]};
                row_stats<DUAL>(z, e0, e1, out + j * 128, p.Mp, t.g == 0);
            }
        } else {
            const float rate0 = !DUAL && p.losses == LOSS_KD ? p.inv_tau : 1.f;
            const int dz_rows = (pl.count + 127) & ~127;           // dW goes over whole 128 rows
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 c = DUAL ? tc[j] : one_coef(tc[j], p.losses);
                const int64_t row = tm0 + j * 128 + t.wn * 32 + t.fr;
                if (row - t.fr >= dz_rows) continue;
                bf16* out = p.dz + row * width + tn0 + t.wm * 64 + 8 * t.g;
                const int at = ty[j] - (v0 + tn0 + t.wm * 64 + 4 * t.g);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        dz_block<DUAL, P>(acc[h][j][i], c, rate0, p.inv_tau, at - h * 128 - i * 32, out + h * 128 + i * 32, p.dz_part);
            }
        }
        if (!more) break;
    }
}

// The same in tiles of 128 rows and 128 entries, a workgroup of four wavefronts each, two on a CU, for launches that have too few of the
// large ones (mid_tiles_pay, vocab_loss.hip).  Both operands of a stage of 64 travel through two stages of LDS; a stage is read as
// a whole, asked for again and then multiplied.
constexpr int VM_STAGE = 32768, VM_LDS = 2 * VM_STAGE;
template <bool GRAD, bool DUAL, int P>
__global__ __launch_bounds__(256, 2) void vocab_logits_mid_kernel(VocabGemm p) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int lane = threadIdx.x & 63, g = lane >> 5, fr = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
    const VocabPlan pl = *p.plan;
    const int rows_m = __builtin_amdgcn_readfirstlane((pl.count + 127) >> 7);
    const int width = GRAD ? __builtin_amdgcn_readfirstlane(pl.width) : p.span;
    const Piece piece = piece_of(p.piece, width, p.V);
    const int v0 = piece.v0, n = piece.n;
    const int tiles_n = GRAD ? (n + 255) / 256 * 2 : (n + 127) >> 7, tiles = rows_m * tiles_n;    // dz is whole tiles of 256
    if ((int)blockIdx.x >= tiles) return;
    const int tile = xcd_remap(blockIdx.x, tiles), gn = tiles_n <= 8 ? tiles_n : 8, per_group = gn * rows_m, tg = tile / per_group;
    const int in_grp = tile - tg * per_group, gw = min(gn, tiles_n - tg * gn);
    const int m0 = __builtin_amdgcn_readfirstlane((in_grp / gw) * 128), n0 = __builtin_amdgcn_readfirstlane((tg * gn + in_grp % gw) * 128);

    f32x16_t acc[2][2];                                            // [32-entry block of B][32-row block of A]
    const bool biased = p.bias != nullptr;
    const int es = P == 1 ? 2 : 4;
    const char* bias = biased ? reinterpret_cast<const char*>(p.bias) + (int64_t)v0 * es : nullptr;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c0 = n0 + wm * 64 + i * 32 + 4 * g;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f32x4_t b = {0.f, 0.f, 0.f, 0.f};
            if (biased && c0 + 8 * k + 4 <= p.V - v0) {
                if (P == 1) {
                    const u32x2_t u = *reinterpret_cast<const u32x2_t*>(bias + (c0 + 8 * k) * 2);
                    b = f32x4_t{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xFFFF0000u), __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xFFFF0000u)};
                } else {
                    b = *reinterpret_cast<const f32x4_t*>(bias + (c0 + 8 * k) * 4);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][0][4 * k + e] = b[e];
        }
        if (n0 + 128 > n) start_at_end<P>(acc[i][0], c0, n, (p.V - v0) & ~3, bias);
        acc[i][1] = acc[i][0];
    }
    if (m0 < pl.count && n0 < n) {
        // a wavefront-wide load takes 8 rows of 8 chunks; four per operand and wavefront, 32 rows apart
        const int row = wave * 8 + (lane >> 3), ch = ((lane & 7) ^ ((row >> 1) & 7)) << 4;
        const int64_t ld = p.Dp;
        const char* a_base = reinterpret_cast<const char*>(p.x + m0 * ld);
        const char* b_base = reinterpret_cast<const char*>(p.wp + (int64_t)(v0 + n0) * ld);
        const unsigned va = (unsigned)(row * ld * 2 + ch);
        unsigned vb[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) vb[q] = (unsigned)(min(q * 32 + row, n - 1 - n0) * ld * 2 + ch);
        const Parts<P> parts{p.Dp >> 6};
        const int64_t part_a = p.Mp * ld * 2, part_b = p.V * ld * 2;
        const unsigned lds0 = (unsigned)(uintptr_t)LDS_PTR(unsigned char, smem);
        auto issue = [&](int kt) {
            const int term = parts.term(kt);
            const char* a = a_base + parts.a(term) * part_a + parts.within(kt, term) * 128;
            const char* b = b_base + parts.b(term) * part_b + parts.within(kt, term) * 128;
            const unsigned at = lds0 + (kt & 1) * VM_STAGE + wave * 1024;
#pragma unroll
            for (int q = 0; q < 4; ++q) dma16_sbase(b, vb[q], at + q * 4096);
#pragma unroll
            for (int q = 0; q < 4; ++q) dma16_sbase(a + q * 64 * ld, va, at + 16384 + q * 4096);
        };
        const int nst = parts.total();
        issue(0);
        issue(1);
        for (int kt = 0; kt < nst; ++kt) {
            if (kt + 1 < nst) wait_vm<8>();
            else wait_vm<0>();
            asm volatile("s_barrier" ::: "memory");                // everybody's loads of this stage have landed
            const unsigned char* at = smem + (kt & 1) * VM_STAGE;
            bf16x8_t bf[4][2], af[4][2];
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const int koff = ((2 * kk + g) ^ ((fr >> 1) & 7)) << 4;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    bf[kk][i] = *reinterpret_cast<const bf16x8_t*>(at + (wm * 64 + i * 32 + fr) * 128 + koff);
                    af[kk][i] = *reinterpret_cast<const bf16x8_t*>(at + 16384 + (wn * 64 + i * 32 + fr) * 128 + koff);
                }
            }
            wait_lds();
            asm volatile("s_barrier" ::: "memory");                // and it has been read
            if (kt + 2 < nst) issue(kt + 2);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = mfma32(bf[kk][i], af[kk][j], acc[i][j]);
        }
    }
    if constexpr (!GRAD) {
        const float e1 = p.inv_tau * LOG2E, e0 = !DUAL && p.losses == LOSS_KD ? e1 : LOG2E;
        float* out = p.stats + (int64_t)((n0 >> 6) + wm) * (DUAL ? 3 : 2) * p.Mp + m0 + wn * 64 + fr;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f32x16_t z[2] = {acc[0][j], acc[1][j]};
            row_stats<DUAL>(z, e0, e1, out + j * 32, p.Mp, g == 0);
        }
    } else {
        const float rate0 = !DUAL && p.losses == LOSS_KD ? p.inv_tau : 1.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t row = m0 + wn * 64 + j * 32 + fr;
            float4 c = make_float4(0.f, INFINITY, 0.f, INFINITY);  // rows behind the last one that counts: 0 exp(z - infinity)
            int y = -1;
            if (row < pl.count) {
                c = p.coef[row];
                if (p.label) y = p.label[row];
            }
            if (!DUAL) c = one_coef(c, p.losses);
            bf16* out = p.dz + row * width + n0 + wm * 64 + 8 * g;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                dz_block<DUAL, P>(acc[i][j], c, rate0, p.inv_tau, y - (v0 + n0 + wm * 64 + 4 * g) - i * 32, out + i * 32, p.dz_part);
        }
    }
}

// dx of 256 rows and 256 columns over a range of a piece of the vocabulary, in float32, to a place of the range's own, in the order of
// the accumulators (vocab_dx_rows_kernel reads it); later pieces add to it.
template <int P>
__device__ __forceinline__ void dx_block(const VocabGemm& p, unsigned char* smem, int block) {
    const TileLane t;
    const VocabPlan pl = *p.plan;
    const int tiles_d = (p.D + 255) >> 8, tiles = __builtin_amdgcn_readfirstlane((pl.rows >> 8) * tiles_d);
    const int width = __builtin_amdgcn_readfirstlane(pl.width);
    const Piece piece = piece_of(p.piece, width, p.V);
    const int v0 = piece.v0, n = piece.n;
    if (n == 0 || block >= tiles * pl.splits) return;
    const int lin = xcd_remap(block, tiles * pl.splits);
    const int split = __builtin_amdgcn_readfirstlane(lin / tiles), tile = __builtin_amdgcn_readfirstlane(lin - split * tiles);
    const int m0 = __builtin_amdgcn_readfirstlane((tile / tiles_d) * 256), n0 = __builtin_amdgcn_readfirstlane((tile % tiles_d) * 256);
    const int st0 = split * __builtin_amdgcn_readfirstlane(pl.stages), nst = min(__builtin_amdgcn_readfirstlane(pl.stages), ((n + 127) >> 7) * 2 - st0);
    float* out = p.acc + (int64_t)lin * 65536 + t.wave * 8192 + t.lane * 4;
    f32x16_t acc[2][2][2];
    clear(acc);
    if (nst > 0) {
        const int64_t lda = width, ldb = p.ldw;
        // rows of dz behind the last one that counts read that one again, their dx is not stored
        unsigned va[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 2; ++q) va[h][q] = (unsigned)(min(h * 128 + q * 64 + t.row_along(), pl.count - 1 - m0) * lda * 2 + t.byte_along());
        const char* a_base = reinterpret_cast<const char*>(p.dz + m0 * lda + st0 * 64);
        const char* b_base = reinterpret_cast<const char*>(p.w + (int64_t)v0 * ldb + n0);
        unsigned col[2];                                           // columns beyond a row read its last eight again (never used)
#pragma unroll
        for (int h = 0; h < 2; ++h) col[h] = (unsigned)min(h * 256 + t.byte_across(), (p.ldw - 8 - n0) * 2);
        const unsigned vrow = (unsigned)(t.row_across() * ldb * 2);
        const Parts<P> parts{nst};
        const int64_t part_a = p.dz_part * 2, part_b = p.V * ldb * 2;
        auto issue_a = [&](auto half, int kt, unsigned lds) {
            const int term = parts.term(kt);
            constexpr int h = decltype(half)::value;
            const char* src = a_base + parts.a(term) * part_a + parts.within(kt, term) * 128;
            dma16_sbase(src, va[h][0], lds);
            dma16_sbase(src, va[h][1], lds + 8192);
        };
        auto issue_b = [&](auto half, int kt, unsigned lds) {
            constexpr int h = decltype(half)::value;
            const int term = parts.term(kt), k0 = (st0 + parts.within(kt, term)) * 64;
            const char* of = b_base + parts.b(term) * part_b;
            if (k0 + 64 <= n) {
                const char* src = of + k0 * ldb * 2;
                dma16_sbase(src, vrow + col[h], lds);
                dma16_sbase(src + 64 * ldb, vrow + col[h], lds + 8192);
            } else {                                               // rows beyond the piece, where dz is 0, read its last one
                const int first = min(k0, n - 1), left = n - 1 - first;
                const char* src = of + first * ldb * 2;
                dma16_sbase(src, (unsigned)(min(t.row_across(), left) * ldb * 2) + col[h], lds);
                dma16_sbase(src, (unsigned)(min(t.row_across() + 32, left) * ldb * 2) + col[h], lds + 8192);
            }
        };
        request_stages(smem, t, issue_a, issue_b);
        tile_products<false, true>(smem, t, issue_a, issue_b, parts.total(), acc);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (m0 + j * 128 + t.wn * 32 >= pl.count) continue;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16_t& c = acc[h][j][i];
                    f32x4_t v = {c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
                    f32x4_t* at = reinterpret_cast<f32x4_t*>(out + ((h * 4 + j * 2 + i) * 4 + q) * 256);
                    if (p.piece > 0) v += *at;
                    *at = v;
                }
        }
}

// dX of the rows that count, 32 columns per thread: the ranges' sums of the row's place added in order.  The workgroups behind `sums`
// of them clear the rows that do not.  Bound by reading the ranges' sums: 8192 rows of 1024, one range, 14 us, 3.6 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void vocab_dx_rows_kernel(VocabGemm p, const int* __restrict__ list, const int* __restrict__ place, int M, int sums,
                                                            T* __restrict__ dX) {
    const int blocks = (p.D + 31) >> 5, lane = threadIdx.x & 63, w = threadIdx.x >> 6, groups = (blocks + 3) >> 2;
    if ((int)blockIdx.x >= sums) {                                 // four rows per wavefront
        constexpr int E = 16 / sizeof(T);
        const int r0 = (blockIdx.x - sums) * 16 + w * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (r0 + k < M && place[r0 + k] < 0)
                for (int d = lane * E; d < p.D; d += 64 * E) *reinterpret_cast<u32x4_t*>(dX + (int64_t)(r0 + k) * p.D + d) = u32x4_t{0, 0, 0, 0};
        return;
    }
    const VocabPlan pl = *p.plan;
    const int rb = blockIdx.x / groups, cb = (blockIdx.x - rb * groups) * 4 + w, i = rb * 64 + lane;
    if (i >= pl.count || cb >= blocks) return;
    const int d0 = cb * 32;
    f32x4_t s[8] = {};
    const int tiles_d = (p.D + 255) >> 8, tiles = (pl.rows >> 8) * tiles_d, tile = (i >> 8) * tiles_d + (d0 >> 8);
    const int h = d0 >> 7 & 1, wm = d0 >> 6 & 1, ib = d0 >> 5 & 1, j = i >> 7 & 1, wn = i >> 5 & 3, fr = i & 31;
    const float* at = p.acc + (int64_t)tile * 65536 + (wn * 2 + wm) * 8192 + (h * 4 + j * 2 + ib) * 1024 + fr * 4;
    for (int k = 0; k < pl.splits; k += 4) {
        f32x4_t v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[u][e] = k + u < pl.splits ? *reinterpret_cast<const f32x4_t*>(at + (int64_t)(k + u) * tiles * 65536 + (e >> 1) * 256 + (e & 1) * 128)
                                            : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += v[u][e];
    }
    T* out = dX + (int64_t)list[i] * p.D + d0;
#pragma unroll
    for (int e = 0; e < 8; e += 2)
        if (d0 + e * 4 < p.D) {
            if constexpr (sizeof(T) == 2) {
                typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
                bf16x8 b;
#pragma unroll
                for (int k = 0; k < 4; ++k) { b[k] = (__bf16)s[e][k]; b[4 + k] = (__bf16)s[e + 1][k]; }
                *reinterpret_cast<bf16x8*>(out + e * 4) = b;
            } else {
                *reinterpret_cast<f32x4_t*>(out + e * 4) = s[e];
                *reinterpret_cast<f32x4_t*>(out + e * 4 + 4) = s[e + 1];
            }
        }
}

// dW of 256 entries of a piece and 256 columns over a range of the rows, all of them unless there are few tiles, and, in the workgroups
// behind the tiles, db of 256 entries each: these find the CUs that the last round of tiles leaves idle.  The sums of several ranges go to
// places of their own, in float32 (vocab_dw_sum_kernel).
template <typename TG, int P>
__device__ __forceinline__ void dw_block(const VocabGemm& p, unsigned char* smem, TG* dparams, int db, int block) {
    const TileLane t;
    const VocabPlan pl = *p.plan;
    const int width = __builtin_amdgcn_readfirstlane(pl.width);
    const Piece piece = piece_of(p.piece, width, p.V);
    const int v0 = piece.v0, n = piece.n;
    if (n == 0) return;
    const int tiles_v = (n + 255) >> 8, tiles_d = (p.D + 255) >> 8, tiles = tiles_v * tiles_d;
    const int64_t ldz = width;
    const int pairs = (pl.count + 127) >> 7, per = (pairs + p.dw_splits - 1) / p.dw_splits;
    const bool whole = p.dw_splits == 1;
    if (block >= tiles * p.dw_splits) {
        const int lin = block - tiles * p.dw_splits, split = lin / tiles_v, b = lin - split * tiles_v;
        if (!db || split >= p.dw_splits) return;
        const int end = min(pl.count, (split + 1) * per * 128);
        const int c = threadIdx.x & 31, lane_row = threadIdx.x >> 5;
        float s[8] = {};
#pragma unroll
        for (int part = P - 1; part >= 0; --part) {
            const bf16* src = p.dz + part * p.dz_part + b * 256 + c * 8;
            for (int r0 = split * per * 128 + lane_row; r0 < end; r0 += 128) {    // eight rows in flight (up to whole 128 rows, zeros at the end)
                u32x4_t v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const u32x4_t*>(src + (r0 + 16 * u) * ldz);
#pragma unroll
                for (int u = 0; u < 8; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[2 * e] += __uint_as_float(v[u][e] << 16);
                        s[2 * e + 1] += __uint_as_float(v[u][e] & 0xFFFF0000u);
                    }
            }
        }
        float* sh = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int e = 0; e < 8; ++e) sh[lane_row * 256 + c * 8 + e] = s[e];
        __syncthreads();
        if (threadIdx.x < 256 && b * 256 + (int)threadIdx.x < n) {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 16; ++k) sum += sh[k * 256 + threadIdx.x];
            const int64_t at = (int64_t)p.V * p.D + v0 + b * 256 + threadIdx.x;
            if (whole) dparams[at] = from_f<TG>(sum);
            else p.dw_parts[split * p.dw_stride + at] = sum;
        }
        return;
    }
    const int lin = xcd_remap(block, tiles * p.dw_splits), split = __builtin_amdgcn_readfirstlane(lin / tiles), tile = lin - split * tiles;
    const int m0 = __builtin_amdgcn_readfirstlane((tile / tiles_d) * 256), n0 = __builtin_amdgcn_readfirstlane((tile % tiles_d) * 256);
    const int first = __builtin_amdgcn_readfirstlane(split * per), nst = __builtin_amdgcn_readfirstlane(min(per, pairs - first)) * 2;
    f32x16_t acc[2][2][2];
    clear(acc);
    if (nst > 0) {
        const int64_t ldb = p.Dp;
        const unsigned va = (unsigned)(t.row_across() * ldz * 2 + t.byte_across());
        unsigned vb[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) vb[h] = (unsigned)(t.row_across() * ldb * 2 + min(h * 256 + t.byte_across(), (p.Dp - 8 - n0) * 2));
        const char* a_base = reinterpret_cast<const char*>(p.dz + first * 128 * ldz + m0);
        const char* b_base = reinterpret_cast<const char*>(p.x + first * 128 * ldb + n0);
        const Parts<P> parts{nst};
        const int64_t part_a = p.dz_part * 2, part_b = p.Mp * ldb * 2;
        auto issue_a = [&](auto half, int kt, unsigned lds) {
            const int term = parts.term(kt);
            const char* src = a_base + parts.a(term) * part_a + decltype(half)::value * 256 + parts.within(kt, term) * 128 * ldz;
            dma16_sbase(src, va, lds);
            dma16_sbase(src + 64 * ldz, va, lds + 8192);
        };
        auto issue_b = [&](auto half, int kt, unsigned lds) {
            const int term = parts.term(kt);
            const char* src = b_base + parts.b(term) * part_b + parts.within(kt, term) * 128 * ldb;
            dma16_sbase(src, vb[decltype(half)::value], lds);
            dma16_sbase(src + 64 * ldb, vb[decltype(half)::value], lds + 8192);
        };
        request_stages(smem, t, issue_a, issue_b);
        tile_products<true, true>(smem, t, issue_a, issue_b, parts.total(), acc);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int v = m0 + j * 128 + t.wn * 32 + t.fr;
        const int64_t at = (int64_t)(v0 + v) * p.D + n0 + t.wm * 64;
        if (sizeof(TG) == 4 || !whole) {
            if (v >= n) continue;
            float* out = (whole ? reinterpret_cast<float*>(dparams) : p.dw_parts + split * p.dw_stride) + at;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16_t& c = acc[h][j][i];
                        const int d = h * 128 + i * 32 + 8 * q + 4 * t.g;
                        if (n0 + t.wm * 64 + d < p.D)
                            *reinterpret_cast<f32x4_t*>(out + d) = f32x4_t{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
                    }
        } else if constexpr (sizeof(TG) == 2) {
            TG* out = dparams + at;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int d = n0 + t.wm * 64 + h * 128 + i * 32 + 8 * t.g;
                    store_eights(out + h * 128 + i * 32 + 8 * t.g, acc[h][j][i], v < n && d < p.D, v < n && d + 16 < p.D);
                }
        }
    }
}

// dparams from the sums of the ranges of rows, in their order, four elements per thread.  Bound by reading them.
template <typename TG>
__global__ __launch_bounds__(256) void vocab_dw_sum_kernel(const float* __restrict__ parts, int64_t stride, int splits, int64_t n, TG* __restrict__ dparams) {
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= n) return;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < splits; k += 8) {
        f32x4_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = k + u < splits ? *reinterpret_cast<const f32x4_t*>(parts + (k + u) * stride + at) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (at + e < n) dparams[at + e] = from_f<TG>(s[e]);
}

// Both, which need dz alone: the first dx_blocks workgroups take dx, whose ranges are the longer ones, and dW's tiles fill the CUs
// as these end.  Bound by the matrix cores: 8192 rows of 1024, 131072 entries 3.27 ms, 1.35 PFLOP/s, 85 % busy.
template <typename TG, int P>
__global__ __launch_bounds__(512, 2) void vocab_grads_kernel(VocabGemm p, int dx_blocks, TG* dparams, int db) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int block = blockIdx.x;
    if (block < dx_blocks) dx_block<P>(p, smem, block);
    else dw_block<TG, P>(p, smem, dparams, db, block - dx_blocks);
}

template <typename... A>
static int launch_tiles(void (*kern)(A...), LdsLimit& lim, int64_t blocks, int threads, int lds, hipStream_t s, A... args) {
    if (int rc = lim.ensure(reinterpret_cast<const void*>(kern), lds)) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(threads), lds, s, args...);
    REV_HIP(hipGetLastError());
    return REV_OK;
}

template <typename T> constexpr int parts_of = sizeof(T) == 2 ? 1 : 3;

template <typename T>
int vocab_logits(hipStream_t s, const VocabGemm& p, bool grad, bool dual, bool mid, int64_t blocks) {
    constexpr int P = parts_of<T>;
    ProfScope ps(K_VOCAB, s, p.work);
    const int64_t large = std::min<int64_t>(blocks, 256);          // one per CU
#define FORM(G, U) if (grad == G && dual == U) {                                                                          \
        static LdsLimit lim[2];                                                                                          \
        return mid ? launch_tiles(vocab_logits_mid_kernel<G, U, P>, lim[0], 4 * blocks, 256, VM_LDS, s, p)               \
                   : launch_tiles(vocab_logits_kernel<G, U, P>, lim[1], large, 512, VG_LDS + 8 * VG_SIDE, s, p); }
    FORM(false, false) FORM(false, true) FORM(true, false) FORM(true, true)
#undef FORM
    return REV_OK;
}
template <typename T>
int vocab_dx_rows(hipStream_t s, const VocabGemm& p, const int* list, const int* place, int M, T* dX) {
    ProfScope ps(K_REDUCE, s, (4.0 + sizeof(T)) * M * p.D);
    const int sums = (M + 63) / 64 * (((p.D + 31) / 32 + 3) / 4);
    hipLaunchKernelGGL(vocab_dx_rows_kernel<T>, dim3((unsigned)(sums + (M + 15) / 16)), dim3(256), 0, s, p, list, place, M, sums, dX);
    REV_HIP(hipGetLastError());
    return REV_OK;
}
// dx_blocks (a multiple of 8: the tiles of dW begin on the first XCD), dw_blocks: most that there may be; 0: not wanted
template <typename T>
int vocab_grads(hipStream_t s, const VocabGemm& p, int64_t dx_blocks, int64_t dw_blocks, void* dparams, bool grad_bf16, bool db) {
    ProfScope ps(K_VOCAB, s, p.work * ((dx_blocks > 0) + (dw_blocks > 0)));
    static LdsLimit lim[2];
    const int first = (int)dx_blocks;
    if constexpr (sizeof(T) == 2)
        if (grad_bf16) return launch_tiles(vocab_grads_kernel<bf16, 1>, lim[0], dx_blocks + dw_blocks, 512, VG_LDS, s, p, first, (bf16*)dparams, (int)db);
    return launch_tiles(vocab_grads_kernel<float, parts_of<T>>, lim[1], dx_blocks + dw_blocks, 512, VG_LDS, s, p, first, (float*)dparams, (int)db);
}
int vocab_dw_sum(hipStream_t s, const VocabGemm& p, void* dparams, bool grad_bf16, int64_t n) {
    ProfScope ps(K_REDUCE, s, 4.0 * p.dw_splits * n);
    const dim3 grid((unsigned)((n + 1023) / 1024)), block(256);
    if (grad_bf16) hipLaunchKernelGGL(vocab_dw_sum_kernel<bf16>, grid, block, 0, s, p.dw_parts, p.dw_stride, p.dw_splits, n, (bf16*)dparams);
    else hipLaunchKernelGGL(vocab_dw_sum_kernel<float>, grid, block, 0, s, p.dw_parts, p.dw_stride, p.dw_splits, n, (float*)dparams);
    REV_HIP(hipGetLastError());
    return REV_OK;
}
#define BOTH(T)                                                                                   \
    template int vocab_logits<T>(hipStream_t, const VocabGemm&, bool, bool, bool, int64_t);       \
    template int vocab_grads<T>(hipStream_t, const VocabGemm&, int64_t, int64_t, void*, bool, bool); \
    template int vocab_dx_rows<T>(hipStream_t, const VocabGemm&, const int*, const int*, int, T*);
BOTH(bf16)
BOTH(float)
#undef BOTH

}  // namespace rev
