// Gated feed-forward block Y = (act(X Wg) * (X Wu)) Wd, forward and backward.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "bpt_internal.h"
#include "gemm_tiles.h"

namespace bpt {
namespace {

// act(g) and act'(g)
// (v_exp_f32 and v_rcp_f32 are good to 1 unit in the last place; the results are rounded to bf16)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& value, float& slope) {
    if constexpr (ACT == BPT_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504088896341f));
        value = g * s;
        slope = s * (1.f + g * (1.f - s));
    } else if constexpr (ACT == BPT_ACT_GELU) {
        // Phi(-|g|) = exp(-g^2 / 2) t q(t), t = 1 / (1 + 0.3 |g|): q is a polynomial of degree 7 fitted (least squares, weights
        // moved to level the error) to the scaled complementary error function over |g| <= 14, 1.5e-7 relative; with fp32
        // arithmetic below 3e-6 relative for |g| <= 6, where erff and the exponential of the slope would cost twice the instructions
        const float e = __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f);
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(g), 1.f));
        float q = 0.035674779f;
        q = fmaf(q, t, -0.157203101f);
        q = fmaf(q, t, 0.206353537f);
        q = fmaf(q, t, -0.053683671f);
        q = fmaf(q, t, 0.128561640f);
        q = fmaf(q, t, 0.099913488f);
        q = fmaf(q, t, 0.120753957f);
        q = fmaf(q, t, 0.119629299f);
        const float below = q * t * e;
        const float s = g > 0.f ? 1.f - below : below;
        value = g * s;
        slope = s + g * 0.39894228040143268f * e;
    } else {
        value = g <= 0.f ? 0.f : g;   // (a NaN stays one)
        slope = g <= 0.f ? 0.f : 1.f;
    }
}

// Order of the tiles: workgroups go round robin over the 8 XCDs, each of which has an L2 of its own, so every XCD gets
// a contiguous run of tiles; within a run, bands of kBand rows of tiles are walked column by column.
constexpr int kXcds = 8, kBand = 4;
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int total = tiles_m * tiles_n, each = total / kXcds, more = total % kXcds;
    const int xcd = id % kXcds, at = id / kXcds;
    const int t = xcd * each + min(xcd, more) + at;
    const int band = t / (kBand * tiles_n), first = band * kBand, rows = min(kBand, tiles_m - first);
    const int in = t - band * kBand * tiles_n;
    tm = first + in % rows;
    tn = in / rows;
}

__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
    *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}

// ---- F = act(X Wg) * (X Wu) ---------------------------------------------------------------------------------
// One product whose tiles hold the same columns of both projections, so that activation and product are formed from the fp32
// sums where they lie.  65 532 rows, d = 512, f = 2048: 300 to 314 us over devices, 0.92 to 0.88 PFLOP/s (250 us without what follows
// the sums: an exponential and a reciprocal at a quarter of the rate for each value, and 268 MB written); 9001 rows, d = 2048,
// f = 5464: 384 us, 1.05 PFLOP/s.
// F is rounded to bf16, the type of the next product's operand.  That rounding and Y's own are alike in size and independent: Y is off
// by sqrt(2) times its own rounding in the 2-norm (2.3e-3 instead of 1.7e-3 measured, whatever the size).  A second bf16 part, as the
// strips for few rows write it, would take this away and cost the next product twice its operations and F twice its bytes.
struct UpArgs {
    const bf16_t *X, *Wg, *Wu;
    bf16_t *F, *F_low;    // (F_low: strips only)
    int64_t M, ldx;
    int32_t d, f, tiles_m, tiles_n;
};
template <typename C, int ACT>
__global__ void __launch_bounds__(C::kThreads, C::kWavesPerSimd) gated_up_kernel(const UpArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[C::kLds];
    int tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * C::kBM;
    const int n0 = tn * (C::kBN / 2);
    C t;
    t.init(shared, g.ldx, g.M - m0, g.f, g.f - n0);
    typename C::Acc acc = {};
    const bf16_t *X = g.X + m0 * g.ldx, *Wg = g.Wg + n0, *Wu = g.Wu + n0;
    t.run(acc, (g.d + C::kSlab - 1) / C::kSlab, [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
        a = X + s * C::kSlab;
        b0 = Wg + (int64_t)s * C::kSlab * g.f;
        b1 = Wu + (int64_t)s * C::kSlab * g.f;
        k_left = g.d - s * C::kSlab;
    });
    constexpr int kHalf = C::kCols / 2;
    const RowBlock<kHalf * 32> block(t.lds, t.wave, t.lane);
    const int col = n0 + t.col_of(0);
#pragma unroll
    for (int i = 0; i < C::kRows; ++i) {
#pragma unroll
        for (int j = 0; j < kHalf; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float value, slope;
                    activation<ACT>(acc[i][j][4 * q + e], value, slope);
                    v[e] = value * acc[i][kHalf + j][4 * q + e];
                }
                block.put(j * 32 + 8 * q, v[0], v[1], v[2], v[3]);
            }
        const int64_t m = m0 + t.row_of(i);
        block.write(g.F + m * g.f + col, g.f, g.M - m, g.f - col);
    }
}

// ---- few rows ---------------------------------------------------------------------------------------------------
// Neighbouring strips of 32 columns share cache lines, so an XCD gets a run of them.
__device__ __forceinline__ int strip_of(int id, int strips) {
    const int each = strips / kXcds, more = strips % kXcds, xcd = id % kXcds;
    return xcd * each + min(xcd, more) + id / kXcds;
}
// F leaves in two bf16 parts, the second what the first's rounding left over: for few rows the second costs nothing that
// would show (the weights are what is read), and Y is then as good as with F in fp32.
using UpStrip = Strip<4, 4, 1, 2>;
template <int ACT>
__global__ void __launch_bounds__(UpStrip::kThreads) gated_up_strip_kernel(const UpArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[UpStrip::kLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = strip_of(blockIdx.x, gridDim.x) * 32;
    const int64_t m0 = (int64_t)blockIdx.y * 32;
    const bf16_t *x[1] = {g.X + m0 * g.ldx}, *w[2] = {g.Wg + n0, g.Wu + n0};
    float4 sum[2];
    UpStrip::run(shared, wave, lane, x, g.ldx, g.M - m0, w, g.f, g.f - n0, g.d, sum);
    const int64_t m = m0 + (lane & 31);
    const int n = n0 + 8 * wave + 4 * (lane >> 5);
    if (wave >= 4 || m >= g.M || n >= g.f) return;
    const float gate[4] = {sum[0].x, sum[0].y, sum[0].z, sum[0].w}, up[4] = {sum[1].x, sum[1].y, sum[1].z, sum[1].w};
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float value, slope;
        activation<ACT>(gate[e], value, slope);
        v[e] = value * up[e];
    }
    const uint2 hi = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    *reinterpret_cast<uint2*>(g.F + m * g.f + n) = hi;
    if (!g.F_low) return;
    // (an infinite F has no rest: inf - inf)
    const float h[4] = {bf16_as_f32(hi.x & 0xFFFFu), __uint_as_float(hi.x & 0xFFFF0000u), bf16_as_f32(hi.y & 0xFFFFu), __uint_as_float(hi.y & 0xFFFF0000u)};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fabsf(h[e]) < INFINITY ? v[e] - h[e] : 0.f;
    *reinterpret_cast<uint2*>(g.F_low + m * g.f + n) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}

// (blockIdx.z: a slice of k, where the strips leave most of the device idle; its sums go to `part` and are added in order)
struct DownArgs {
    const bf16_t *F[2], *Wd;
    bf16_t* Y;
    int64_t M, ldy;
    int32_t d, f, slices, slice_k;
    float* part;          // [slice][M][d]
};
template <int PARTS>   // of F
using DownStrip = Strip<8, PARTS == 2 ? 3 : 4, PARTS, 1>;
template <int PARTS>
__global__ void __launch_bounds__(DownStrip<PARTS>::kThreads) down_strip_kernel(const DownArgs g) {
    using S = DownStrip<PARTS>;
    __shared__ __attribute__((aligned(1024))) unsigned char shared[S::kLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = strip_of(blockIdx.x, gridDim.x) * 32;
    const int64_t m0 = (int64_t)blockIdx.y * 32;
    const int k0 = blockIdx.z * g.slice_k;
    const bf16_t *x[2] = {g.F[0] + m0 * g.f + k0, PARTS == 2 ? g.F[1] + m0 * g.f + k0 : nullptr}, *w[1] = {g.Wd + (int64_t)k0 * g.d + n0};
    float4 sum[1];
    S::run(shared, wave, lane, x, g.f, g.M - m0, w, g.d, g.d - n0, min(g.slice_k, g.f - k0), sum);
    const int64_t m = m0 + (lane & 31);
    const int n = n0 + 8 * wave + 4 * (lane >> 5);
    if (wave >= 4 || m >= g.M || n >= g.d) return;
    if (g.slices > 1) store4(g.part + ((int64_t)blockIdx.z * g.M + m) * g.d + n, sum[0].x, sum[0].y, sum[0].z, sum[0].w);
    else *reinterpret_cast<uint2*>(g.Y + m * g.ldy + n) = make_uint2(bf16_pair(sum[0].x, sum[0].y), bf16_pair(sum[0].z, sum[0].w));
}
__global__ void __launch_bounds__(256) down_sum_kernel(const DownArgs g) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, elems = g.M * g.d;
    if (i >= elems) return;
    float4 x = *reinterpret_cast<const float4*>(g.part + i);
#pragma unroll 4
    for (int s = 1; s < g.slices; ++s) {
        const float4 v = *reinterpret_cast<const float4*>(g.part + s * elems + i);
        x.x += v.x; x.y += v.y; x.z += v.z; x.w += v.w;
    }
    const int64_t m = i / g.d;
    *reinterpret_cast<uint2*>(g.Y + m * g.ldy + (i - m * g.d)) = make_uint2(bf16_pair(x.x, x.y), bf16_pair(x.z, x.w));
}

// ---- C = A0 B0 (+ A1 B1), or several products side by side ------------------------------------------------------
// The first `full` tiles are computed whole; what is left over is less than the device holds at once and is cut into
// `slices` of k, whose sums go to `part` and are added by product_sum_kernel, in order.  65 532 rows, d = 512, f = 2048: Y 139 us
// (1.0 PFLOP/s), dX 264 us, dWg and dWu 269 + 13 us; 9001 rows, d = 2048, f = 5464: dX 429 us in 256 whole tiles and 32 in
// eight slices each (608 us in two rounds of whole tiles).
struct ProductArgs {
    const bf16_t *A[2], *B[2];
    void* C[2];
    int64_t M, lda, ldb, ldc;
    int64_t K;               // of each of the `terms` products that are added up
    int32_t N, terms, matrices;   // matrices: products with the same A (terms = 1), one behind the other in the grid
    int32_t tiles_m, tiles_n;     // (tiles_n: of one matrix)
    int32_t full, slices, slice_slabs;
    float4* part;            // [left-over tile][slice][block of 32 x 32][4][thread]: as the threads hold the sums
};
struct ProductTile {
    int mat, n0;
    int64_t m0;
};
template <typename C>
__device__ __forceinline__ ProductTile product_tile(const ProductArgs& g, int id) {
    int tm, tn;
    tile_of(id, g.tiles_m, g.tiles_n * g.matrices, tm, tn);
    const int mat = tn / g.tiles_n;
    return {mat, (tn - mat * g.tiles_n) * C::kBN, (int64_t)tm * C::kBM};
}
template <typename C, bool A_KFIRST, bool B_KFIRST, typename T>
__device__ __forceinline__ void product_body(const ProductArgs& g, int group, unsigned char* shared) {
    const int over = max(group - g.full, 0), slice = group < g.full ? 0 : over % g.slices;
    const bool whole = group < g.full || g.slices == 1;
    const ProductTile at = product_tile<C>(g, min(group, g.full) + over / g.slices);
    C t;
    t.init(shared, g.lda, g.M - at.m0, g.ldb, g.N - at.n0);
    typename C::Acc acc = {};
    const int64_t a_at = A_KFIRST ? at.m0 * g.lda : at.m0, b_at = B_KFIRST ? at.n0 * g.ldb : at.n0;
    const int each = (int)((g.K + C::kSlab - 1) / C::kSlab), slabs = each * g.terms;
    const int first = whole ? 0 : slice * g.slice_slabs, last = whole ? slabs : min(first + g.slice_slabs, slabs);
    t.run(acc, max(last - first, 0), [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
        s += first;
        const int term = s >= each ? 1 : 0;
        const int64_t k = (int64_t)(s - term * each) * C::kSlab;
        a = g.A[term] + a_at + (A_KFIRST ? k : k * g.lda);
        b0 = g.B[term + at.mat] + b_at + (B_KFIRST ? k : k * g.ldb);
        k_left = g.K - k;
    });
    if (!whole) {
        float4* part = g.part + (int64_t)over * C::kBlocks * 4 * C::kThreads + threadIdx.x;
#pragma unroll
        for (int i = 0; i < C::kRows; ++i)
#pragma unroll
            for (int j = 0; j < C::kCols; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    part[((i * C::kCols + j) * 4 + q) * C::kThreads] =
                        make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        return;
    }
    const int col = at.n0 + t.col_of(0);
    if constexpr (sizeof(T) == 2) {
        const RowBlock<C::kCols * 32> block(t.lds, t.wave, t.lane);
#pragma unroll
        for (int i = 0; i < C::kRows; ++i) {
#pragma unroll
            for (int j = 0; j < C::kCols; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    block.put(j * 32 + 8 * q, acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
            const int64_t m = at.m0 + t.row_of(i);
            block.write(static_cast<bf16_t*>(g.C[at.mat]) + m * g.ldc + col, g.ldc, g.M - m, g.N - col);
        }
    } else {
#pragma unroll
        for (int i = 0; i < C::kRows; ++i) {
            const int64_t m = at.m0 + t.row_of(i) + (t.lane & 31);
            float* out = static_cast<float*>(g.C[at.mat]) + m * g.ldc;
#pragma unroll
            for (int j = 0; j < C::kCols; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = col + j * 32 + 8 * q + 4 * (t.lane >> 5);
                    if (m < g.M && n < g.N) store4(out + n, acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                }
        }
    }
}

template <typename C, bool A_KFIRST, bool B_KFIRST, typename T>
__global__ void __launch_bounds__(C::kThreads, C::kWavesPerSimd) product_kernel(const ProductArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[C::kLds];
    product_body<C, A_KFIRST, B_KFIRST, T>(g, blockIdx.x, shared);
}

// The three products of the backward at once, the longest sums first: for few rows none of them fills the device.
struct GradArgs {
    ProductArgs dx, wgu, wd;   // whole tiles only
    int32_t dx_last;
};
template <typename CX, typename CW, typename T>
__global__ void __launch_bounds__(CX::kThreads, CX::kWavesPerSimd) grads_kernel(const GradArgs g) {
    static_assert(CX::kThreads == CW::kThreads && CX::kLds == CW::kLds, "one launch");
    __shared__ __attribute__((aligned(1024))) unsigned char shared[CX::kLds];
    const int weights = g.wgu.full + g.wd.full, group = blockIdx.x;
    const int dx = g.dx_last ? group - weights : group, w = g.dx_last ? group : group - g.dx.full;
    if (g.dx_last ? dx >= 0 : w < 0) return product_body<CX, true, true, bf16_t>(g.dx, dx, shared);
    const int wd = w - g.wgu.full;
    product_body<CW, false, false, T>(wd < 0 ? g.wgu : g.wd, wd < 0 ? w : wd, shared);
}

// The left-over tiles: sums of their slices in order; a workgroup takes one 32 x 32 block of each wavefront.
template <typename C, typename T>
__global__ void __launch_bounds__(C::kThreads) product_sum_kernel(const ProductArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[RowBlock<32>::kBytes * C::kWaves];
    const ProductTile at = product_tile<C>(g, g.full + blockIdx.x);
    C t;
    t.place(shared);
    const int i = blockIdx.y / C::kCols, j = blockIdx.y % C::kCols;
    const int64_t pitch = (int64_t)C::kBlocks * 4 * C::kThreads;
    const float4* p = g.part + blockIdx.x * g.slices * pitch + blockIdx.y * 4 * C::kThreads + threadIdx.x;
    float4 x[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = p[q * C::kThreads];
#pragma unroll 4
    for (int s = 1; s < g.slices; ++s) {
        p += pitch;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 v = p[q * C::kThreads];
            x[q].x += v.x; x[q].y += v.y; x[q].z += v.z; x[q].w += v.w;
        }
    }
    const int col = at.n0 + t.col_of(j);
    if constexpr (sizeof(T) == 2) {
        const int64_t m = at.m0 + t.row_of(i);
        const RowBlock<32> block(t.lds, t.wave, t.lane);
#pragma unroll
        for (int q = 0; q < 4; ++q) block.put(8 * q, x[q].x, x[q].y, x[q].z, x[q].w);
        block.write(static_cast<bf16_t*>(g.C[at.mat]) + m * g.ldc + col, g.ldc, g.M - m, g.N - col);
    } else {
        const int64_t m = at.m0 + t.row_of(i) + (t.lane & 31);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = col + 8 * q + 4 * (t.lane >> 5);
            if (m < g.M && n < g.N) store4(static_cast<float*>(g.C[at.mat]) + m * g.ldc + n, x[q].x, x[q].y, x[q].z, x[q].w);
        }
    }
}

// ---- backward up to the hidden gradients ----------------------------------------------------------------------
struct HiddenArgs {
    const bf16_t *X, *dY, *Wg, *Wu, *Wd;
    bf16_t *F, *dG, *dU;
    int64_t M, ldx, ldy;   // (ldy: of dY)
    int32_t d, f, tiles_m, tiles_n;
};
// G = X Wg and U = X Wu are formed again, then dF = dY Wd^T on the same tile: F, dG and dU are written, rounded once.  G and U could
// be kept by the forward instead, but not rounded to bf16 (with both rounded dX is off by 1.9 times the rounding of dX itself;
// now 1.4 times), and in fp32 they cost 16 bytes of traffic per value against 4 d operations: even at d = 800 or so, below which
// most widths here lie, and no gigabyte of activations is held per layer.  F, dG and dU are rounded to bf16 as the forward's F is.
// 65 532 rows, d = 512, f = 2048: 567 to 589 us over devices, 0.73 to 0.70 PFLOP/s (805 MB written); 9001 rows, d = 2048, f = 5464:
// 664 to 688 us, 0.91 to 0.88 PFLOP/s.  The matrix cores are busy 34 % of the cycles, the least of the block's large products at no lower
// a clock: one workgroup per compute unit lets its loads run dry between the two sums and writes with nothing else running.
template <typename C, typename C2, int ACT>
__global__ void __launch_bounds__(C::kThreads, C::kWavesPerSimd) gated_hidden_bwd_kernel(const HiddenArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[C::kLds > C2::kLds ? C::kLds : C2::kLds];
    int tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * C::kBM;
    const int n0 = tn * (C::kBN / 2);
    constexpr int kHalf = C::kCols / 2;
    typename C::Acc gu = {};
    const int slabs = (g.d + C::kSlab - 1) / C::kSlab;
    {
        C t;
        t.init(shared, g.ldx, g.M - m0, g.f, g.f - n0);
        const bf16_t *X = g.X + m0 * g.ldx, *Wg = g.Wg + n0, *Wu = g.Wu + n0;
        t.run(gu, slabs, [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
            a = X + s * C::kSlab;
            b0 = Wg + (int64_t)s * C::kSlab * g.f;
            b1 = Wu + (int64_t)s * C::kSlab * g.f;
            k_left = g.d - s * C::kSlab;
        });
    }
    C2 t;
    t.init(shared, g.ldy, g.M - m0, g.d, g.f - n0);
    typename C2::Acc df = {};
    const bf16_t *dY = g.dY + m0 * g.ldy, *Wd = g.Wd + (int64_t)n0 * g.d;
    t.run(df, slabs, [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
        a = dY + s * C::kSlab;
        b0 = Wd + s * C::kSlab;
        k_left = g.d - s * C::kSlab;
    });
    // the three results, one behind the other through the same LDS; G and U make way for act(G) and U act'(G)
    const RowBlock<kHalf * 32> block(t.lds, t.wave, t.lane);
    const int col = n0 + t.col_of(0);
#pragma unroll
    for (int i = 0; i < C::kRows; ++i) {
        const int64_t m = m0 + t.row_of(i), at = m * g.f + col;
#pragma unroll
        for (int j = 0; j < kHalf; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float value, slope;
                    const float up = gu[i][kHalf + j][4 * q + e];
                    activation<ACT>(gu[i][j][4 * q + e], value, slope);
                    v[e] = value * up;
                    gu[i][j][4 * q + e] = value;
                    gu[i][kHalf + j][4 * q + e] = up * slope;
                    if (e & 1) __builtin_amdgcn_sched_barrier(0);   // (192 sums are in registers: few activations at a time)
                }
                block.put(j * 32 + 8 * q, v[0], v[1], v[2], v[3]);
            }
        block.write(g.F + at, g.f, g.M - m, g.f - col);
#pragma unroll
        for (int half = 1; half >= 0; --half) {
#pragma unroll
            for (int j = 0; j < kHalf; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = df[i][j][4 * q + e] * gu[i][half * kHalf + j][4 * q + e];
                    block.put(j * 32 + 8 * q, v[0], v[1], v[2], v[3]);
                }
            block.write((half ? g.dG : g.dU) + at, g.f, g.M - m, g.f - col);
        }
    }
}

// ---- host side --------------------------------------------------------------------------------------------------
constexpr int kCus = 256;

// Sizes of a workgroup's tile.  kBig: 256 x 256, slabs of 64, one workgroup of 8 wavefronts per compute unit; kWide: 128 x 256,
// slabs of 32, three deep, and kMid: 128 x 128, slabs of 64: two workgroups of 4 wavefronts per compute unit, of which
// one multiplies while the other starts up or writes; kSmall and kSmallAcross: 64 x 64, slabs of 128, two deep, or of 64, four deep,
// where A lies across k (the weights' gradients, whose sums over rows are short): for products of few tiles, whose
// time is a slab's start, four dependent matrix instructions and its barrier (forward and backward of 700 rows, d = 1024,
// f = 2736: 108 us with slabs of 64 throughout, 98 us so; 400 rows, d = 2048, f = 5464, slabs of 128 throughout: 192 -> 216 us; a
// fifth slab in flight changes nothing).  Times measured on all four products of the block (both operands' orders differ by 10 %).
enum TileSize { kBig, kWide, kMid, kSmall, kSmallAcross };
struct TileCost {
    int m, n, slab, per_cu;
    float us, us_one, us_few;   // of 64 k: the device full; one workgroup on every compute unit; few compute units busy
};
constexpr TileCost kTileCost[] = {{256, 256, 64, 1, 2.1f, 2.1f, 1.45f}, {128, 256, 32, 2, 2.35f, 1.7f, 1.15f}, {128, 128, 64, 2, 1.25f, 0.92f, 0.60f},
                                  {64, 64, 128, 2, 0.53f, 0.43f, 0.35f}, {64, 64, 64, 2, 0.53f, 0.43f, 0.37f}};
float slab_us(const TileCost& t, int64_t groups) {   // in between, in proportion
    if (groups <= kCus) return t.us_few + (t.us_one - t.us_few) * (float)groups / kCus;
    return t.us_one + (t.us - t.us_one) * std::min(1.f, (float)(groups - kCus) / kCus);
}
constexpr float kGapUs = 1.0f;               // between two launches
constexpr float kStartUs = 2.5f;             // a tile's first loads and its results
constexpr float kSumUs = 3.5f, kSumBytesPerUs = 5.0e6f;   // adding up slices: a launch, and their bytes written and read
constexpr int kMaxSlices = 32, kMinSliceK = 128;

struct ProductPlan {
    TileSize size;
    int tiles_m, tiles_n, full, left, slices, slice_slabs;   // tiles: computed whole, and cut into slices
    float us;
};
// The cheapest of the tile sizes and slicings by the costs above: whole tiles run in rounds of what the device holds; the last
// round's, if they leave much of it idle, are cut along k instead.
ProductPlan plan_product(int64_t M, int64_t N, int64_t K, int terms, int matrices, TileSize small) {
    ProductPlan best = {};
    best.us = INFINITY;
    for (TileSize c : {kBig, kWide, kMid, small}) {
        const TileCost& t = kTileCost[c];
        ProductPlan p = {};
        p.size = c;
        p.tiles_m = (int)((M + t.m - 1) / t.m);
        p.tiles_n = (int)((N + t.n - 1) / t.n);
        const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * matrices, slots = (int64_t)kCus * t.per_cu;
        const int64_t slabs = (K + t.slab - 1) / t.slab * terms;
        auto rounds = [&](int64_t groups, int64_t n) {   // of workgroups with n slabs each
            const float one = (float)n * t.slab / 64 * slab_us(t, groups) + kStartUs;
            return groups <= kCus ? one : (float)((groups + slots - 1) / slots) * one;
        };
        for (int64_t s = 1; s <= kMaxSlices && (s == 1 || slabs * t.slab / s >= kMinSliceK); ++s) {
            const int64_t over = s == 1 ? 0 : tiles % slots;
            if (s > 1 && (over == 0 || over * s > slots)) break;
            p.full = (int)(tiles - over);
            p.left = (int)over;
            p.slice_slabs = (int)std::max<int64_t>(1, (slabs + s - 1) / s);
            p.slices = s == 1 ? 1 : (int)((slabs + p.slice_slabs - 1) / p.slice_slabs);
            p.us = p.full ? rounds(p.full, slabs) : 0.f;
            if (p.left) {
                p.us += rounds((int64_t)p.left * p.slices, p.slice_slabs);
                p.us += kSumUs + (float)((double)p.left * p.slices * t.m * t.n * 8 / kSumBytesPerUs);
            }
            if (p.us < best.us) best = p;
        }
    }
    return best;
}
size_t part_bytes(const ProductPlan& p) {
    return p.slices > 1 ? align256((size_t)p.left * p.slices * kTileCost[p.size].m * kTileCost[p.size].n * 4) : 0;
}

template <typename C, bool AK, bool BK, typename T>
int launch_product(const ProductArgs& g, int left, hipStream_t st) {
    BPT_LAUNCH("product_kernel", (product_kernel<C, AK, BK, T>), dim3((unsigned)(g.full + left * g.slices)), dim3(C::kThreads), 0, st, g);
    BPT_HIP(hipGetLastError());
    if (g.slices > 1) {
        BPT_LAUNCH("product_sum_kernel", (product_sum_kernel<C, T>), dim3((unsigned)left, C::kBlocks), dim3(C::kThreads), 0, st, g);
        BPT_HIP(hipGetLastError());
    }
    return BPT_OK;
}
template <bool AK, bool BK, typename T>
int launch_product(ProductArgs& g, const ProductPlan& p, void* part, hipStream_t st) {
    g.tiles_m = p.tiles_m; g.tiles_n = p.tiles_n; g.full = p.full; g.slices = p.slices; g.slice_slabs = p.slice_slabs;
    g.part = static_cast<float4*>(part);
    if (p.size == kBig) return launch_product<Tile<256, 256, 2, 4, 64, 2, AK, BK, false>, AK, BK, T>(g, p.left, st);
    if (p.size == kWide) return launch_product<Tile<128, 256, 1, 4, 32, 3, AK, BK, false>, AK, BK, T>(g, p.left, st);
    if (p.size == kMid) return launch_product<Tile<128, 128, 2, 2, 64, 2, AK, BK, false>, AK, BK, T>(g, p.left, st);
    return launch_product<Tile<64, 64, 2, 2, AK ? 128 : 64, AK ? 2 : 4, AK, BK, false>, AK, BK, T>(g, p.left, st);
}

// Strips of 32 x 32 serve as long as every one has a compute unit to itself (d = 512, f = 1368: 1 row, both products 6.7 + 9.9
// -> 3.8 + 4.3 us; 128 rows 7.0 + 10.2 -> 4.3 + 4.6 us; d = 2048, f = 5464: 1 row 25 + 17 -> 10 + 8.5 us, 64 rows 26 + 16 ->
// 24 + 12 us; with two per compute unit they are no faster than the tiles)
bool use_strips(int64_t rows, int cols) { return ((rows + 31) / 32) * ((cols + 31) / 32) <= kCus; }
dim3 strip_grid(int64_t rows, int cols) { return dim3((unsigned)((cols + 31) / 32), (unsigned)((rows + 31) / 32)); }

// Tiles of the hidden activations: 128 rows by 128 columns of both halves, or by 64 where these leave compute units idle, or
// 64 rows by 64 columns where those have a compute unit each (d = 512, f = 1368, 300 rows: 7.2 -> 6.0 us forward, 11.8 -> 9.5 us
// backward; 1023 rows 7.6 -> 10.9 us, 13.6 -> 18.1 us); backward 256 rows by 128 columns for two rounds and more (65 532 rows,
// d = 512, f = 2048: 573 -> 560 us; forward 309 -> 319 us, 9001 rows, d = 2048, f = 5464: 383 -> 392 us).  How full the last
// round is does not enter, here or in the forward: 65 532 rows are 16.0 rounds of the backward's tiles; the 9001 are 6.05, which cost seven.
enum HiddenSize { kHiddenBig, kHiddenWide, kHiddenMid, kHiddenSmall };
HiddenSize hidden_tiles(int64_t M, int f, bool backward, int32_t& tiles_m, int32_t& tiles_n) {
    auto count = [&](int m, int n) {
        tiles_m = (int)((M + m - 1) / m);
        tiles_n = (f + n - 1) / n;
        return (int64_t)tiles_m * tiles_n;
    };
    if (count(64, 64) <= kCus) return kHiddenSmall;
    if (backward && count(256, 128) >= 2 * kCus) return kHiddenBig;
    if (count(128, 128) >= kCus) return kHiddenWide;
    count(128, 64);
    return kHiddenMid;
}

template <int ACT, typename C>
int launch_up_as(const UpArgs& g, hipStream_t st) {
    BPT_LAUNCH("gated_up_kernel", (gated_up_kernel<C, ACT>), dim3((unsigned)((int64_t)g.tiles_m * g.tiles_n)), dim3(C::kThreads), 0, st, g);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}
template <int ACT>
int launch_up(UpArgs& g, hipStream_t st) {
    if (use_strips(g.M, g.f)) {
        BPT_LAUNCH("gated_up_strip_kernel", gated_up_strip_kernel<ACT>, strip_grid(g.M, g.f), dim3(UpStrip::kThreads), 0, st, g);
        BPT_HIP(hipGetLastError());
        return BPT_OK;
    }
    const HiddenSize size = hidden_tiles(g.M, g.f, false, g.tiles_m, g.tiles_n);
    if (size == kHiddenWide) return launch_up_as<ACT, Tile<128, 256, 2, 2, 32, 3, true, false, true>>(g, st);
    if (size == kHiddenMid) return launch_up_as<ACT, Tile<128, 128, 2, 2, 64, 2, true, false, true>>(g, st);
    return launch_up_as<ACT, Tile<64, 128, 2, 2, 128, 2, true, false, true>>(g, st);
}

template <int ACT, typename C, typename C2>
int launch_hidden_as(const HiddenArgs& g, hipStream_t st) {
    BPT_LAUNCH("gated_hidden_bwd_kernel", (gated_hidden_bwd_kernel<C, C2, ACT>), dim3((unsigned)((int64_t)g.tiles_m * g.tiles_n)),
               dim3(C::kThreads), 0, st, g);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}
template <int ACT>
int launch_hidden(HiddenArgs& g, hipStream_t st) {
    const HiddenSize size = hidden_tiles(g.M, g.f, true, g.tiles_m, g.tiles_n);
    if (size == kHiddenBig)
        return launch_hidden_as<ACT, Tile<256, 256, 2, 4, 64, 2, true, false, true>, Tile<256, 128, 2, 4, 64, 2, true, true, false>>(g, st);
    if (size == kHiddenWide)
        return launch_hidden_as<ACT, Tile<128, 256, 1, 4, 32, 3, true, false, true>, Tile<128, 128, 1, 4, 32, 3, true, true, false>>(g, st);
    if (size == kHiddenMid)
        return launch_hidden_as<ACT, Tile<128, 128, 2, 2, 64, 2, true, false, true>, Tile<128, 64, 2, 2, 64, 2, true, true, false>>(g, st);
    return launch_hidden_as<ACT, Tile<64, 128, 2, 2, 128, 2, true, false, true>, Tile<64, 64, 2, 2, 128, 2, true, true, false>>(g, st);
}

constexpr int64_t kMostStride = ((int64_t)1 << 20) - 1;   // (offsets within a tile are 32 bits)
int check_ffn(const bpt_gated_ffn_t* s) {
    if (!s || s->rows < 0) return BPT_ERR_INVALID_ARG;
    if (s->dtype != BPT_BF16 || s->rows >= INT32_MAX) return BPT_ERR_UNSUPPORTED;
    if (s->d < 8 || s->f < 8 || (s->d & 7) || (s->f & 7) || s->d > 65536 || s->f > 65536) return BPT_ERR_UNSUPPORTED;
    if (!stride_ok(s->stride, s->d, kMostStride)) return BPT_ERR_INVALID_ARG;
    if (s->activation < BPT_ACT_SILU || s->activation > BPT_ACT_RELU) return BPT_ERR_INVALID_ARG;
    if (s->grad_dtype != BPT_F32 && s->grad_dtype != BPT_BF16) return BPT_ERR_INVALID_ARG;
    // a launch has fewer than 2^32 threads, 512 for a tile at most
    if (((s->rows + 63) / 64) * ((s->d + 63) / 64) >= 1 << 23 || ((s->rows + 127) / 128) * ((s->f + 127) / 128) >= 1 << 23) return BPT_ERR_UNSUPPORTED;
    return BPT_OK;
}

// Slices of k for the strips of the second product: a compute unit takes in about 50 KB a microsecond, its columns of Wd and all of F's
// rows; with few strips the others help, for the price of a launch that adds the slices.
int down_slices(int64_t rows, int d, int f, int parts) {
    const int64_t strips = ((rows + 31) / 32) * ((d + 31) / 32), slices = std::min<int64_t>(kCus / strips, f / 512);
    const float us = (float)f * 2 * (32 + (float)(parts * std::min<int64_t>(rows, 32))) / 50e3f;
    return slices > 1 && us * (1.f - 1.f / (float)slices) > kSumUs + 1.f ? (int)slices : 1;
}

struct FwdBuffers {
    ProductPlan down;
    bool up_strips, down_strips;
    int slices, slice_k;      // of the strips
    size_t F, F_low, part, total;
};
FwdBuffers fwd_buffers(const bpt_gated_ffn_t* s) {
    FwdBuffers b = {};
    b.up_strips = use_strips(s->rows, s->f);
    b.down_strips = use_strips(s->rows, s->d);
    if (!b.down_strips) b.down = plan_product(s->rows, s->d, s->f, 1, 1, kSmall);
    const size_t hidden = align256((size_t)s->rows * s->f * 2);
    b.F = 0;
    b.F_low = hidden;
    const bool two_parts = b.up_strips && b.down_strips;
    b.part = b.F_low + (two_parts ? hidden : 0);
    if (b.down_strips) {
        b.slices = down_slices(std::max<int64_t>(s->rows, 1), s->d, s->f, two_parts ? 2 : 1);
        b.slice_k = ((s->f + b.slices - 1) / b.slices + 31) / 32 * 32;
        b.slices = (s->f + b.slice_k - 1) / b.slice_k;
    }
    b.total = b.part + (b.down_strips ? (b.slices > 1 ? align256((size_t)b.slices * s->rows * s->d * 4) : 0) : part_bytes(b.down));
    return b;
}
struct BwdBuffers {
    ProductPlan wd, wgu, dx;
    size_t F, dG, dU, part, total;
};
BwdBuffers bwd_buffers(const bpt_gated_ffn_t* s) {
    BwdBuffers b = {};
    b.wd = plan_product(s->f, s->d, s->rows, 1, 1, kSmallAcross);
    b.wgu = plan_product(s->d, s->f, s->rows, 1, 2, kSmallAcross);
    b.dx = plan_product(s->rows, s->d, s->f, 2, 1, kSmall);
    const size_t hidden = align256((size_t)s->rows * s->f * 2);
    b.F = 0;
    b.dG = hidden;
    b.dU = 2 * hidden;
    b.part = 3 * hidden;
    b.total = b.part + std::max(std::max(part_bytes(b.wd), part_bytes(b.wgu)), part_bytes(b.dx));
    return b;
}

ProductArgs wd_product(const bpt_gated_ffn_t* s, const bpt_row_strides_t& apart, const bf16_t* F, const bf16_t* dY, void* dWd) {
    ProductArgs g = {};
    g.A[0] = g.A[1] = F; g.B[0] = g.B[1] = dY; g.C[0] = g.C[1] = dWd;
    g.M = s->f; g.N = s->d; g.K = s->rows;
    g.lda = s->f; g.ldb = apart.grad; g.ldc = s->d;
    g.terms = g.matrices = 1;
    return g;
}
ProductArgs wgu_product(const bpt_gated_ffn_t* s, const bpt_row_strides_t& apart, const bf16_t* X, const bf16_t* dG, const bf16_t* dU, void* dWg,
                        void* dWu) {
    ProductArgs g = {};
    g.A[0] = g.A[1] = X; g.B[0] = dG; g.B[1] = dU; g.C[0] = dWg; g.C[1] = dWu;
    g.M = s->d; g.N = s->f; g.K = s->rows;
    g.lda = apart.x; g.ldb = s->f; g.ldc = s->f;
    g.terms = 1; g.matrices = 2;
    return g;
}
ProductArgs dx_product(const bpt_gated_ffn_t* s, const bpt_row_strides_t& apart, const bf16_t* dG, const bf16_t* dU, const bf16_t* Wg,
                       const bf16_t* Wu, void* dX) {
    ProductArgs g = {};
    g.A[0] = dG; g.A[1] = dU; g.B[0] = Wg; g.B[1] = Wu; g.C[0] = g.C[1] = dX;
    g.M = s->rows; g.N = s->d; g.K = s->f;
    g.lda = g.ldb = s->f; g.ldc = apart.out;
    g.terms = 2; g.matrices = 1;
    return g;
}

// whole tiles of all three products in one launch, dX in one size and the weights' gradients in another, where that is estimated
// shorter than the three one by one
float plan_together(GradArgs& g, TileSize x, TileSize w) {
    ProductArgs* const product[3] = {&g.dx, &g.wgu, &g.wd};
    int64_t groups = 0, slabs[3];
    for (int i = 0; i < 3; ++i) {
        ProductArgs& p = *product[i];
        const TileCost& t = kTileCost[i == 0 ? x : w];
        const int64_t tm = (p.M + t.m - 1) / t.m, tn = (p.N + t.n - 1) / t.n;
        if (tm * tn * p.matrices > 1 << 20) return INFINITY;
        slabs[i] = (p.K + t.slab - 1) / t.slab * p.terms;
        p.tiles_m = (int)tm;
        p.tiles_n = (int)tn;
        p.full = (int)(tm * tn * p.matrices);
        p.slices = 1;
        p.slice_slabs = (int)slabs[i];
        groups += p.full;
    }
    float longest = 0.f, work = 0.f;
    for (int i = 0; i < 3; ++i) {
        const TileCost& t = kTileCost[i == 0 ? x : w];
        const float us = (float)slabs[i] * t.slab / 64 * slab_us(t, groups);
        longest = std::max(longest, us);
        work += (float)product[i]->full * us;
    }
    g.dx_last = slabs[0] * kTileCost[x].slab < slabs[1] * kTileCost[w].slab;
    if (groups <= 2 * kCus) return kStartUs + longest;   // (two of either size per compute unit)
    // several rounds of unequal lengths: measured up to 28 % over their mean
    return kStartUs + std::max(longest, 1.28f * work / (2 * kCus));
}

template <typename CX, typename CW, typename T>
int launch_grads(const GradArgs& g, hipStream_t st) {
    BPT_LAUNCH("grads_kernel", (grads_kernel<CX, CW, T>), dim3((unsigned)(g.dx.full + g.wgu.full + g.wd.full)), dim3(CX::kThreads), 0, st, g);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}

template <typename T>
int grads(const bpt_gated_ffn_t* s, const BwdBuffers& b, GradArgs& g, bool dx_alone, void* part, hipStream_t st) {
    if (s->rows > 0 && !dx_alone) {
        GradArgs best = g;
        float us = b.dx.us + b.wgu.us + b.wd.us + 2 * kGapUs;
        TileSize size[2] = {kBig, kBig};
        for (TileSize x : {kMid, kSmall})
            for (TileSize w : {kMid, kSmallAcross}) {
                GradArgs a = g;
                const float t = plan_together(a, x, w);
                if (t >= us) continue;
                us = t;
                best = a;
                size[0] = x;
                size[1] = w;
            }
        using MidX = Tile<128, 128, 2, 2, 64, 2, true, true, false>;
        using MidW = Tile<128, 128, 2, 2, 64, 2, false, false, false>;
        using SmallX = Tile<64, 64, 2, 2, 128, 2, true, true, false>;
        using SmallW = Tile<64, 64, 2, 2, 64, 4, false, false, false>;
        if (size[0] == kMid) return size[1] == kMid ? launch_grads<MidX, MidW, T>(best, st) : launch_grads<MidX, SmallW, T>(best, st);
        if (size[0] == kSmall) return size[1] == kMid ? launch_grads<SmallX, MidW, T>(best, st) : launch_grads<SmallX, SmallW, T>(best, st);
    }
    // (no rows: products of nothing, zero gradients)
    if (const int rc = launch_product<false, false, T>(g.wd, b.wd, part, st)) return rc;
    if (const int rc = launch_product<false, false, T>(g.wgu, b.wgu, part, st)) return rc;
    // (dX last: it may overwrite dY or X)
    return s->rows > 0 ? launch_product<true, true, bf16_t>(g.dx, b.dx, part, st) : BPT_OK;
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" {

size_t bpt_gated_ffn_fwd_workspace(const bpt_gated_ffn_t* s) {
    if (check_ffn(s)) return SIZE_MAX;
    return fwd_buffers(s).total;
}

int bpt_gated_ffn_fwd_strided(const bpt_gated_ffn_t* s, const bpt_row_strides_t* strides, const void* X, const void* Wg, const void* Wu,
                              const void* Wd, void* Y, void* workspace, size_t workspace_bytes, void* stream) {
    if (const int rc = check_ffn(s)) return rc;
    if (s->rows == 0) return BPT_OK;
    const bpt_row_strides_t apart = row_strides(strides, s->stride);
    if (!stride_ok(apart.x, s->d, kMostStride) || !stride_ok(apart.out, s->d, kMostStride)) return BPT_ERR_INVALID_ARG;
    if (!X || !Wg || !Wu || !Wd || !Y || !workspace || off_boundary(X, Wg, Wu, Wd, Y, workspace)) return BPT_ERR_INVALID_ARG;
    const FwdBuffers b = fwd_buffers(s);
    if (workspace_bytes < b.total) return BPT_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    bf16_t* F = reinterpret_cast<bf16_t*>(ws + b.F);
    UpArgs u = {};
    u.X = static_cast<const bf16_t*>(X); u.Wg = static_cast<const bf16_t*>(Wg); u.Wu = static_cast<const bf16_t*>(Wu);
    u.F = F;
    u.F_low = b.up_strips && b.down_strips ? reinterpret_cast<bf16_t*>(ws + b.F_low) : nullptr;
    u.M = s->rows; u.ldx = apart.x; u.d = s->d; u.f = s->f;
    const int rc = s->activation == BPT_ACT_SILU ? launch_up<BPT_ACT_SILU>(u, st)
                   : s->activation == BPT_ACT_GELU ? launch_up<BPT_ACT_GELU>(u, st) : launch_up<BPT_ACT_RELU>(u, st);
    if (rc) return rc;
    if (b.down_strips) {
        const DownArgs g = {{F, u.F_low}, static_cast<const bf16_t*>(Wd), static_cast<bf16_t*>(Y), s->rows, apart.out, s->d, s->f, b.slices, b.slice_k,
                            reinterpret_cast<float*>(ws + b.part)};
        dim3 grid = strip_grid(s->rows, s->d);
        grid.z = b.slices;
        if (u.F_low)
            BPT_LAUNCH("down_strip_kernel", down_strip_kernel<2>, grid, dim3(DownStrip<2>::kThreads), 0, st, g);
        else
            BPT_LAUNCH("down_strip_kernel", down_strip_kernel<1>, grid, dim3(DownStrip<1>::kThreads), 0, st, g);
        BPT_HIP(hipGetLastError());
        if (b.slices > 1) {
            BPT_LAUNCH("down_sum_kernel", down_sum_kernel, dim3((unsigned)((s->rows * s->d / 4 + 255) / 256)), dim3(256), 0, st, g);
            BPT_HIP(hipGetLastError());
        }
        return BPT_OK;
    }
    ProductArgs g = {};
    g.A[0] = g.A[1] = F; g.B[0] = g.B[1] = static_cast<const bf16_t*>(Wd); g.C[0] = g.C[1] = Y;
    g.M = s->rows; g.N = s->d; g.K = s->f;
    g.lda = s->f; g.ldb = s->d; g.ldc = apart.out;
    g.terms = g.matrices = 1;
    return launch_product<true, false, bf16_t>(g, b.down, ws + b.part, st);
}

int bpt_gated_ffn_fwd(const bpt_gated_ffn_t* s, const void* X, const void* Wg, const void* Wu, const void* Wd, void* Y, void* workspace,
                      size_t workspace_bytes, void* stream) {
    return bpt_gated_ffn_fwd_strided(s, nullptr, X, Wg, Wu, Wd, Y, workspace, workspace_bytes, stream);
}

size_t bpt_gated_ffn_bwd_workspace(const bpt_gated_ffn_t* s) {
    if (check_ffn(s)) return SIZE_MAX;
    return bwd_buffers(s).total;
}

int bpt_gated_ffn_bwd_strided(const bpt_gated_ffn_t* s, const bpt_row_strides_t* strides, const void* X, const void* Wg, const void* Wu,
                              const void* Wd, const void* dY, void* dX, void* dWg, void* dWu, void* dWd, void* workspace,
                              size_t workspace_bytes, void* stream) {
    if (const int rc = check_ffn(s)) return rc;
    const bpt_row_strides_t apart = row_strides(strides, s->stride);
    if (!Wg || !Wu || !Wd || !dWg || !dWu || !dWd || off_boundary(X, Wg, Wu, Wd, dY, dX, dWg, dWu, dWd, workspace)) return BPT_ERR_INVALID_ARG;
    const BwdBuffers b = bwd_buffers(s);
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const bf16_t *x = static_cast<const bf16_t*>(X), *dy = static_cast<const bf16_t*>(dY);
    if (s->rows > 0) {
        if (!X || !dY || !dX || !workspace || workspace_bytes < b.total) return BPT_ERR_INVALID_ARG;
        for (int64_t x : {apart.x, apart.out, apart.grad})
            if (!stride_ok(x, s->d, kMostStride)) return BPT_ERR_INVALID_ARG;
        if (!same_place(dX, dY, s->rows, apart.out, apart.grad) || !same_place(dX, X, s->rows, apart.out, apart.x)) return BPT_ERR_INVALID_ARG;
        HiddenArgs h = {};
        h.X = x; h.dY = dy;
        h.Wg = static_cast<const bf16_t*>(Wg); h.Wu = static_cast<const bf16_t*>(Wu); h.Wd = static_cast<const bf16_t*>(Wd);
        h.F = reinterpret_cast<bf16_t*>(ws + b.F);
        h.dG = reinterpret_cast<bf16_t*>(ws + b.dG);
        h.dU = reinterpret_cast<bf16_t*>(ws + b.dU);
        h.M = s->rows; h.ldx = apart.x; h.ldy = apart.grad; h.d = s->d; h.f = s->f;
        const int rc = s->activation == BPT_ACT_SILU ? launch_hidden<BPT_ACT_SILU>(h, st)
                       : s->activation == BPT_ACT_GELU ? launch_hidden<BPT_ACT_GELU>(h, st) : launch_hidden<BPT_ACT_RELU>(h, st);
        if (rc) return rc;
    }
    const bf16_t *F = reinterpret_cast<const bf16_t*>(ws + b.F), *dG = reinterpret_cast<const bf16_t*>(ws + b.dG),
                 *dU = reinterpret_cast<const bf16_t*>(ws + b.dU);
    GradArgs g = {dx_product(s, apart, dG, dU, static_cast<const bf16_t*>(Wg), static_cast<const bf16_t*>(Wu), dX),
                  wgu_product(s, apart, x, dG, dU, dWg, dWu), wd_product(s, apart, F, dy, dWd), 0};
    const bool dx_alone = dX == dY || dX == X;
    return s->grad_dtype == BPT_BF16 ? grads<bf16_t>(s, b, g, dx_alone, ws + b.part, st) : grads<float>(s, b, g, dx_alone, ws + b.part, st);
}

int bpt_gated_ffn_bwd(const bpt_gated_ffn_t* s, const void* X, const void* Wg, const void* Wu, const void* Wd, const void* dY, void* dX,
                      void* dWg, void* dWu, void* dWd, void* workspace, size_t workspace_bytes, void* stream) {
    return bpt_gated_ffn_bwd_strided(s, nullptr, X, Wg, Wu, Wd, dY, dX, dWg, dWu, dWd, workspace, workspace_bytes, stream);
}

}  // extern "C"
