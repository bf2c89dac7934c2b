// Gated feed-forward block Y = (act(X Wg) * (X Wu)) Wd, forward and backward.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "bpt_internal.h"
#include "gemm_tiles.h"

namespace bpt {
namespace {

// act(g) and act'(g)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& value, float& slope) {
    if constexpr (ACT == BPT_ACT_SILU) {
        const float s = 1.f / (1.f + __expf(-g));
        value = g * s;
        slope = s * (1.f + g * (1.f - s));
    } else if constexpr (ACT == BPT_ACT_GELU) {
        const float s = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        value = g * s;
        slope = s + g * 0.39894228040143268f * __expf(-0.5f * g * g);
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

__device__ __forceinline__ void store4(bf16_t* p, float a, float b, float c, float d) {
    *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(a, b), bf16_pair(c, d));
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
    *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}

// ---- F = act(X Wg) * (X Wu) ---------------------------------------------------------------------------------
struct UpArgs {
    const bf16_t *X, *Wg, *Wu;
    bf16_t* F;
    int64_t M, ldx;
    int32_t d, f, tiles_m, tiles_n;
};
template <typename C, int BM, int BN, int ACT>
__global__ void __launch_bounds__(C::kThreads, 2) gated_up_kernel(const UpArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[C::kLds];
    int tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * (BN / 2);
    C t;
    t.init(shared, g.ldx, g.M - m0, g.f, g.f - n0);
    typename C::Acc acc = {};
    const bf16_t *X = g.X + m0 * g.ldx, *Wg = g.Wg + n0, *Wu = g.Wu + n0;
    t.run(acc, (g.d + kSlab - 1) / kSlab, [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
        a = X + s * kSlab;
        b0 = Wg + (int64_t)s * kSlab * g.f;
        b1 = Wu + (int64_t)s * kSlab * g.f;
        k_left = g.d - s * kSlab;
    });
    constexpr int kHalf = C::kCols / 2;
#pragma unroll
    for (int i = 0; i < C::kRows; ++i) {
        const int64_t m = m0 + t.row_of(i) + (t.lane & 31);
#pragma unroll
        for (int j = 0; j < kHalf; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + t.col_of(j) + 8 * q + 4 * (t.lane >> 5);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float value, slope;
                    activation<ACT>(acc[i][j][4 * q + e], value, slope);
                    v[e] = value * acc[i][kHalf + j][4 * q + e];
                }
                if (m < g.M && n < g.f) store4(g.F + m * g.f + n, v[0], v[1], v[2], v[3]);
            }
    }
}

// ---- C = A0 B0 (+ A1 B1), or several products side by side, in slices of k -----------------------------------
struct ProductArgs {
    const bf16_t *A[2], *B[2];
    void* C[2];
    int64_t M, lda, ldb, ldc;
    int64_t K;               // of each of the `terms` products that are added up
    int32_t N, terms, matrices;   // matrices: products with the same A (terms = 1), one behind the other in the grid
    int32_t tiles_m, tiles_n, slices, slice_slabs;
    float* part;             // [slices][matrices][M][N], with slices > 1
};
template <typename C, int BM, int BN, bool A_KFIRST, bool B_KFIRST, typename T>
__global__ void __launch_bounds__(C::kThreads, 2) product_kernel(const ProductArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[C::kLds];
    int tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n * g.matrices, tm, tn);
    const int mat = tn / g.tiles_n;
    tn -= mat * g.tiles_n;
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * BN;
    C t;
    t.init(shared, g.lda, g.M - m0, g.ldb, g.N - n0);
    typename C::Acc acc = {};
    const int64_t a_at = A_KFIRST ? m0 * g.lda : m0, b_at = B_KFIRST ? n0 * g.ldb : n0;
    const int each = (int)((g.K + kSlab - 1) / kSlab);
    const int first = blockIdx.y * g.slice_slabs, last = min(first + g.slice_slabs, each * g.terms);
    t.run(acc, max(last - first, 0), [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
        s += first;
        const int term = s >= each ? 1 : 0;
        const int64_t k = (int64_t)(s - term * each) * kSlab;
        a = g.A[term] + a_at + (A_KFIRST ? k : k * g.lda);
        b0 = g.B[term + mat] + b_at + (B_KFIRST ? k : k * g.ldb);
        k_left = g.K - k;
    });
    float* part = g.part + ((int64_t)blockIdx.y * g.matrices + mat) * g.M * g.N;
    T* out = static_cast<T*>(g.C[mat]);
#pragma unroll
    for (int i = 0; i < C::kRows; ++i) {
        const int64_t m = m0 + t.row_of(i) + (t.lane & 31);
#pragma unroll
        for (int j = 0; j < C::kCols; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + t.col_of(j) + 8 * q + 4 * (t.lane >> 5);
                const f32x16_t& x = acc[i][j];
                if (m < g.M && n < g.N) {
                    if (g.slices > 1) store4(part + m * g.N + n, x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                    else store4(out + m * g.ldc + n, x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                }
            }
    }
}

// C = sum of the slices, in order, 4 values per thread
template <typename T>
__global__ void __launch_bounds__(256) product_sum_kernel(const float* __restrict__ part, int slices, int64_t elems, int N, int64_t ldc,
                                                          T* C0, T* C1) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= elems) return;
    const int matrices = gridDim.y;
    const float* p = part + blockIdx.y * elems + i;
    float4 acc = *reinterpret_cast<const float4*>(p);
#pragma unroll 4
    for (int s = 1; s < slices; ++s) {
        const float4 v = *reinterpret_cast<const float4*>(p + (int64_t)s * matrices * elems);
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
    }
    const int64_t row = i / N;
    store4((blockIdx.y ? C1 : C0) + row * ldc + (i - row * N), acc.x, acc.y, acc.z, acc.w);
}

// ---- backward up to the hidden gradients ----------------------------------------------------------------------
struct HiddenArgs {
    const bf16_t *X, *dY, *Wg, *Wu, *Wd;
    bf16_t *F, *dG, *dU;
    int64_t M, ldx;
    int32_t d, f, tiles_m, tiles_n;
};
// G = X Wg and U = X Wu are formed again, then dF = dY Wd^T on the same tile: F, dG and dU are written, rounded once.
template <typename C, typename C2, int BM, int BN, int ACT>
__global__ void __launch_bounds__(C::kThreads, 2) gated_hidden_bwd_kernel(const HiddenArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char shared[C::kLds > C2::kLds ? C::kLds : C2::kLds];
    int tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * (BN / 2);
    constexpr int kHalf = C::kCols / 2;
    typename C::Acc gu = {};
    const int slabs = (g.d + kSlab - 1) / kSlab;
    {
        C t;
        t.init(shared, g.ldx, g.M - m0, g.f, g.f - n0);
        const bf16_t *X = g.X + m0 * g.ldx, *Wg = g.Wg + n0, *Wu = g.Wu + n0;
        t.run(gu, slabs, [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
            a = X + s * kSlab;
            b0 = Wg + (int64_t)s * kSlab * g.f;
            b1 = Wu + (int64_t)s * kSlab * g.f;
            k_left = g.d - s * kSlab;
        });
    }
    C2 t;
    t.init(shared, g.ldx, g.M - m0, g.d, g.f - n0);
    typename C2::Acc df = {};
    const bf16_t *dY = g.dY + m0 * g.ldx, *Wd = g.Wd + (int64_t)n0 * g.d;
    t.run(df, slabs, [&](int s, const bf16_t*& a, const bf16_t*& b0, const bf16_t*& b1, int64_t& k_left) {
        a = dY + s * kSlab;
        b0 = Wd + s * kSlab;
        k_left = g.d - s * kSlab;
    });
#pragma unroll
    for (int i = 0; i < C::kRows; ++i) {
        const int64_t m = m0 + t.row_of(i) + (t.lane & 31);
#pragma unroll
        for (int j = 0; j < kHalf; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + t.col_of(j) + 8 * q + 4 * (t.lane >> 5);
                float vf[4], vg[4], vu[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float value, slope;
                    const float u = gu[i][kHalf + j][4 * q + e], x = df[i][j][4 * q + e];
                    activation<ACT>(gu[i][j][4 * q + e], value, slope);
                    vf[e] = value * u;
                    vg[e] = x * u * slope;
                    vu[e] = x * value;
                }
                if (m < g.M && n < g.f) {
                    const int64_t at = m * g.f + n;
                    store4(g.F + at, vf[0], vf[1], vf[2], vf[3]);
                    store4(g.dG + at, vg[0], vg[1], vg[2], vg[3]);
                    store4(g.dU + at, vu[0], vu[1], vu[2], vu[3]);
                }
            }
    }
}

// ---- host side --------------------------------------------------------------------------------------------------
constexpr int kCus = 256;

// tiles of 256 x 256 where they, with slices of at least kMinSlice k, fill three quarters of the compute units, else
// 128 x 128 (two workgroups per compute unit)
constexpr int kMinSlice = 512, kMaxSlices = 32;
struct ProductPlan {
    bool big;
    int tiles_m, tiles_n, slices, slice_slabs;
};
ProductPlan plan_product(int64_t M, int64_t N, int64_t K, int terms, int matrices) {
    auto cut = [&](int b, int want) {
        ProductPlan p = {};
        p.big = b == 256;
        p.tiles_m = (int)((M + b - 1) / b);
        p.tiles_n = (int)((N + b - 1) / b);
        const int64_t tiles = std::max<int64_t>(1, (int64_t)p.tiles_m * p.tiles_n * matrices), slabs = (K + kSlab - 1) / kSlab * terms;
        int64_t s = std::min<int64_t>(kMaxSlices, std::max<int64_t>(1, std::min(want / tiles, slabs * kSlab / kMinSlice)));
        p.slice_slabs = (int)std::max<int64_t>(1, (slabs + s - 1) / s);
        p.slices = (int)std::max<int64_t>(1, (slabs + p.slice_slabs - 1) / p.slice_slabs);
        return p;
    };
    const ProductPlan p = cut(256, kCus);
    if ((int64_t)p.tiles_m * p.tiles_n * matrices * p.slices >= 3 * kCus / 4) return p;
    return cut(128, 2 * kCus);
}
size_t part_bytes(const ProductPlan& p, int64_t M, int64_t N, int matrices) {
    return p.slices > 1 ? align256((size_t)p.slices * matrices * M * N * 4) : 0;
}

template <bool AK, bool BK, typename T>
int launch_product(ProductArgs& g, const ProductPlan& p, void* part, hipStream_t st) {
    g.tiles_m = p.tiles_m; g.tiles_n = p.tiles_n; g.slices = p.slices; g.slice_slabs = p.slice_slabs;
    g.part = static_cast<float*>(part);
    const dim3 grid((unsigned)((int64_t)p.tiles_m * p.tiles_n * g.matrices), (unsigned)p.slices);
    using Big = Tile<256, 256, 2, 4, AK, BK, false>;
    using Mid = Tile<128, 128, 2, 2, AK, BK, false>;
    if (p.big) BPT_LAUNCH("product_kernel", (product_kernel<Big, 256, 256, AK, BK, T>), grid, dim3(Big::kThreads), 0, st, g);
    else BPT_LAUNCH("product_kernel", (product_kernel<Mid, 128, 128, AK, BK, T>), grid, dim3(Mid::kThreads), 0, st, g);
    BPT_HIP(hipGetLastError());
    if (p.slices > 1) {
        const int64_t elems = g.M * g.N;
        BPT_LAUNCH("product_sum_kernel", product_sum_kernel<T>, dim3((unsigned)((elems / 4 + 255) / 256), (unsigned)g.matrices), dim3(256), 0,
                   st, g.part, p.slices, elems, g.N, g.ldc, static_cast<T*>(g.C[0]), static_cast<T*>(g.C[1]));
        BPT_HIP(hipGetLastError());
    }
    return BPT_OK;
}

template <int ACT>
int launch_up(UpArgs& g, hipStream_t st) {
    const int64_t big = ((g.M + 255) / 256) * ((g.f + 127) / 128);
    const bool is_big = big >= 3 * kCus / 4;
    const int bm = is_big ? 256 : 128, bn = is_big ? 128 : 64;
    g.tiles_m = (int)((g.M + bm - 1) / bm);
    g.tiles_n = (g.f + bn - 1) / bn;
    const dim3 grid((unsigned)((int64_t)g.tiles_m * g.tiles_n));
    using Big = Tile<256, 256, 2, 4, true, false, true>;
    using Mid = Tile<128, 128, 2, 2, true, false, true>;
    if (is_big) BPT_LAUNCH("gated_up_kernel", (gated_up_kernel<Big, 256, 256, ACT>), grid, dim3(Big::kThreads), 0, st, g);
    else BPT_LAUNCH("gated_up_kernel", (gated_up_kernel<Mid, 128, 128, ACT>), grid, dim3(Mid::kThreads), 0, st, g);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}

template <int ACT>
int launch_hidden(HiddenArgs& g, hipStream_t st) {
    const int64_t big = ((g.M + 255) / 256) * ((g.f + 127) / 128);
    const bool is_big = big >= 3 * kCus / 4;
    const int bm = is_big ? 256 : 128, bn = is_big ? 128 : 64;
    g.tiles_m = (int)((g.M + bm - 1) / bm);
    g.tiles_n = (g.f + bn - 1) / bn;
    const dim3 grid((unsigned)((int64_t)g.tiles_m * g.tiles_n));
    using Big = Tile<256, 256, 2, 4, true, false, true>;
    using Big2 = Tile<256, 128, 2, 4, true, true, false>;
    using Mid = Tile<128, 128, 2, 2, true, false, true>;
    using Mid2 = Tile<128, 64, 2, 2, true, true, false>;
    if (is_big) BPT_LAUNCH("gated_hidden_bwd_kernel", (gated_hidden_bwd_kernel<Big, Big2, 256, 256, ACT>), grid, dim3(Big::kThreads), 0, st, g);
    else BPT_LAUNCH("gated_hidden_bwd_kernel", (gated_hidden_bwd_kernel<Mid, Mid2, 128, 128, ACT>), grid, dim3(Mid::kThreads), 0, st, g);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}

int check_ffn(const bpt_gated_ffn_t* s) {
    if (!s || s->rows < 0) return BPT_ERR_INVALID_ARG;
    if (s->dtype != BPT_BF16 || s->rows >= INT32_MAX) return BPT_ERR_UNSUPPORTED;
    if (s->d < 8 || s->f < 8 || (s->d & 7) || (s->f & 7) || s->d > 65536 || s->f > 65536) return BPT_ERR_UNSUPPORTED;
    if (s->stride < s->d || (s->stride & 7) || s->stride >= ((int64_t)1 << 20)) return BPT_ERR_INVALID_ARG;
    if (s->activation < BPT_ACT_SILU || s->activation > BPT_ACT_RELU) return BPT_ERR_INVALID_ARG;
    if (s->grad_dtype != BPT_F32 && s->grad_dtype != BPT_BF16) return BPT_ERR_INVALID_ARG;
    // tiles are numbered in 31 bits (of 128 x 64 at least)
    if (((s->rows + 127) / 128) * ((std::max(s->d, s->f) + 63) / 64) > INT32_MAX) return BPT_ERR_UNSUPPORTED;
    return BPT_OK;
}

struct FwdBuffers {
    ProductPlan down;
    size_t F, part, total;
};
FwdBuffers fwd_buffers(const bpt_gated_ffn_t* s) {
    FwdBuffers b = {};
    b.down = plan_product(s->rows, s->d, s->f, 1, 1);
    b.F = 0;
    b.part = align256((size_t)s->rows * s->f * 2);
    b.total = b.part + part_bytes(b.down, s->rows, s->d, 1);
    return b;
}
struct BwdBuffers {
    ProductPlan wd, wgu, dx;
    size_t F, dG, dU, part, total;
};
BwdBuffers bwd_buffers(const bpt_gated_ffn_t* s) {
    BwdBuffers b = {};
    b.wd = plan_product(s->f, s->d, s->rows, 1, 1);
    b.wgu = plan_product(s->d, s->f, s->rows, 1, 2);
    b.dx = plan_product(s->rows, s->d, s->f, 2, 1);
    const size_t hidden = align256((size_t)s->rows * s->f * 2);
    b.F = 0;
    b.dG = hidden;
    b.dU = 2 * hidden;
    b.part = 3 * hidden;
    b.total = b.part + std::max(std::max(part_bytes(b.wd, s->f, s->d, 1), part_bytes(b.wgu, s->d, s->f, 2)), part_bytes(b.dx, s->rows, s->d, 1));
    return b;
}

template <typename T>
int weight_grads(const bpt_gated_ffn_t* s, const BwdBuffers& b, const bf16_t* X, const bf16_t* dY, unsigned char* ws, void* dWg, void* dWu,
                 void* dWd, hipStream_t st) {
    const bf16_t *F = reinterpret_cast<const bf16_t*>(ws + b.F), *dG = reinterpret_cast<const bf16_t*>(ws + b.dG),
                 *dU = reinterpret_cast<const bf16_t*>(ws + b.dU);
    ProductArgs g = {};
    g.A[0] = g.A[1] = F; g.B[0] = g.B[1] = dY; g.C[0] = g.C[1] = dWd;
    g.M = s->f; g.N = s->d; g.K = s->rows;
    g.lda = s->f; g.ldb = s->stride; g.ldc = s->d;
    g.terms = g.matrices = 1;
    if (const int rc = launch_product<false, false, T>(g, b.wd, ws + b.part, st)) return rc;
    g.A[0] = g.A[1] = X; g.B[0] = dG; g.B[1] = dU; g.C[0] = dWg; g.C[1] = dWu;
    g.M = s->d; g.N = s->f;
    g.lda = s->stride; g.ldb = s->f; g.ldc = s->f;
    g.matrices = 2;
    return launch_product<false, false, T>(g, b.wgu, ws + b.part, st);
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" {

size_t bpt_gated_ffn_fwd_workspace(const bpt_gated_ffn_t* s) {
    if (check_ffn(s)) return SIZE_MAX;
    return fwd_buffers(s).total;
}

int bpt_gated_ffn_fwd(const bpt_gated_ffn_t* s, const void* X, const void* Wg, const void* Wu, const void* Wd, void* Y, void* workspace,
                      size_t workspace_bytes, void* stream) {
    if (const int rc = check_ffn(s)) return rc;
    if (s->rows == 0) return BPT_OK;
    if (!X || !Wg || !Wu || !Wd || !Y || !workspace || off_boundary(X, Wg, Wu, Wd, Y, workspace)) return BPT_ERR_INVALID_ARG;
    const FwdBuffers b = fwd_buffers(s);
    if (workspace_bytes < b.total) return BPT_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    bf16_t* F = reinterpret_cast<bf16_t*>(ws + b.F);
    UpArgs u = {};
    u.X = static_cast<const bf16_t*>(X); u.Wg = static_cast<const bf16_t*>(Wg); u.Wu = static_cast<const bf16_t*>(Wu);
    u.F = F;
    u.M = s->rows; u.ldx = s->stride; u.d = s->d; u.f = s->f;
    const int rc = s->activation == BPT_ACT_SILU ? launch_up<BPT_ACT_SILU>(u, st)
                   : s->activation == BPT_ACT_GELU ? launch_up<BPT_ACT_GELU>(u, st) : launch_up<BPT_ACT_RELU>(u, st);
    if (rc) return rc;
    ProductArgs g = {};
    g.A[0] = g.A[1] = F; g.B[0] = g.B[1] = static_cast<const bf16_t*>(Wd); g.C[0] = g.C[1] = Y;
    g.M = s->rows; g.N = s->d; g.K = s->f;
    g.lda = s->f; g.ldb = s->d; g.ldc = s->stride;
    g.terms = g.matrices = 1;
    return launch_product<true, false, bf16_t>(g, b.down, ws + b.part, st);
}

size_t bpt_gated_ffn_bwd_workspace(const bpt_gated_ffn_t* s) {
    if (check_ffn(s)) return SIZE_MAX;
    return bwd_buffers(s).total;
}

int bpt_gated_ffn_bwd(const bpt_gated_ffn_t* s, const void* X, const void* Wg, const void* Wu, const void* Wd, const void* dY, void* dX,
                      void* dWg, void* dWu, void* dWd, void* workspace, size_t workspace_bytes, void* stream) {
    if (const int rc = check_ffn(s)) return rc;
    if (!Wg || !Wu || !Wd || !dWg || !dWu || !dWd || off_boundary(X, Wg, Wu, Wd, dY, dX, dWg, dWu, dWd, workspace)) return BPT_ERR_INVALID_ARG;
    const BwdBuffers b = bwd_buffers(s);
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const bf16_t *x = static_cast<const bf16_t*>(X), *dy = static_cast<const bf16_t*>(dY);
    if (s->rows > 0) {
        if (!X || !dY || !dX || !workspace || workspace_bytes < b.total) return BPT_ERR_INVALID_ARG;
        HiddenArgs h = {};
        h.X = x; h.dY = dy;
        h.Wg = static_cast<const bf16_t*>(Wg); h.Wu = static_cast<const bf16_t*>(Wu); h.Wd = static_cast<const bf16_t*>(Wd);
        h.F = reinterpret_cast<bf16_t*>(ws + b.F);
        h.dG = reinterpret_cast<bf16_t*>(ws + b.dG);
        h.dU = reinterpret_cast<bf16_t*>(ws + b.dU);
        h.M = s->rows; h.ldx = s->stride; h.d = s->d; h.f = s->f;
        const int rc = s->activation == BPT_ACT_SILU ? launch_hidden<BPT_ACT_SILU>(h, st)
                       : s->activation == BPT_ACT_GELU ? launch_hidden<BPT_ACT_GELU>(h, st) : launch_hidden<BPT_ACT_RELU>(h, st);
        if (rc) return rc;
    }
    // (no rows: products of nothing, zero gradients)
    int rc = s->grad_dtype == BPT_BF16 ? weight_grads<bf16_t>(s, b, x, dy, ws, dWg, dWu, dWd, st)
                                       : weight_grads<float>(s, b, x, dy, ws, dWg, dWu, dWd, st);
    if (rc || s->rows == 0) return rc;
    // (dX last: it may overwrite dY or X)
    ProductArgs g = {};
    g.A[0] = reinterpret_cast<const bf16_t*>(ws + b.dG); g.A[1] = reinterpret_cast<const bf16_t*>(ws + b.dU);
    g.B[0] = static_cast<const bf16_t*>(Wg); g.B[1] = static_cast<const bf16_t*>(Wu);
    g.C[0] = g.C[1] = dX;
    g.M = s->rows; g.N = s->d; g.K = s->f;
    g.lda = g.ldb = s->f; g.ldc = s->stride;
    g.terms = 2; g.matrices = 1;
    return launch_product<true, true, bf16_t>(g, b.dx, ws + b.part, st);
}

}  // extern "C"
