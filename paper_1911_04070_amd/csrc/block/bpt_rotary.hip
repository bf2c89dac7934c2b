// Rotary positions on Q and K, and the positions of a graph's nodes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "bpt_internal.h"
#include "row_device.h"

namespace bpt {
namespace {

struct RotaryArgs {
    const void* in[2];
    void* out[2];
    const float* pos;
    int64_t pos_sb;
    int64_t sb, sh, sn, ob, oh, on;   // elements
    int64_t rows;                     // B * N
    int32_t N, H, rot;
    int32_t each;                     // rows of a workgroup, a power of two
    int32_t heads_first;              // the heads of a row lie closer together than its neighbours
    double turns[kD / 2];             // w_i' / (2 pi), negative for the inverse
};

// 16 bytes of a row
template <typename T>
struct Piece {
    static constexpr int kCount = 16 / sizeof(T);
    T x[kCount];
    __device__ __forceinline__ void load(const T* p) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        __builtin_memcpy(x, &w, 16);
    }
    __device__ __forceinline__ void store(T* p) const {
        uint4 w;
        __builtin_memcpy(&w, x, 16);
        *reinterpret_cast<uint4*>(p) = w;
    }
};
__device__ __forceinline__ float to_f32(bf16_t x) { return bf16_as_f32(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void from_f32(float v, bf16_t& x) { x = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void from_f32(float v, float& x) { x = v; }

enum PairLayout { kNeighbours, kHalves, kHalvesApart };   // kHalvesApart: a half is not a whole number of 16-byte pieces

// A workgroup forms the sines and cosines of its `each` rows once, one or a few per thread, into LDS (64-bit product, reduced to a
// turn, then fp32), and turns all heads of Q and K with them.  A thread takes 16 bytes of a row; 8 (fp32: 16) lanes cover a
// head's row, the next lanes the next head or the next row, whichever lies behind it, so that loads and stores are whole cache
// lines.  With halves a thread also loads the 16 bytes its features are paired with, which its neighbours have just asked
// for, and computes its own side of the pairs only.  Bound by HBM: 4 x 16 383 rows of 8 heads of Q and K in bf16, out of the rows a
// projection writes: 64 us, 4.2 TB/s (lanes that hold both halves of a pair, in 64 bytes of two cache lines, and form the
// angles of their own pairs: 80 us); 2 x 4095 rows of 8 heads in fp32: 13 us, out of the memory-side cache.
// A result may overwrite its input: a pair's threads are lanes of one wavefront, which loads before it stores.
constexpr int kRotaryRows = 16;
template <typename T, PairLayout LAYOUT, int NT>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
    constexpr int kPieces = kD / Piece<T>::kCount, kCount = Piece<T>::kCount, kSlots = 256 / kPieces;
    __shared__ float2 table[kRotaryRows][kD / 2 + 2];   // (two more: rows start in different banks)
    __shared__ int64_t in_row[kRotaryRows], out_row[kRotaryRows];
    const int64_t first = (int64_t)blockIdx.x * a.each;
    const int rows = (int)min((int64_t)a.each, a.rows - first);
    for (int t = threadIdx.x; t < rows * (kD / 2); t += 256) {
        const int r = t / (kD / 2), i = t % (kD / 2);
        const uint32_t row = (uint32_t)(first + r), b = row / (uint32_t)a.N, n = row - b * (uint32_t)a.N;
        if (i == 0) {
            in_row[r] = (int64_t)b * a.sb + (int64_t)n * a.sn;
            out_row[r] = (int64_t)b * a.ob + (int64_t)n * a.on;
        }
        float2 v = make_float2(1.f, 0.f);
        if (i < a.rot / 2) {
            const double x = (double)a.pos[(int64_t)b * a.pos_sb + n] * a.turns[i];
            sincospif(2.f * (float)(x - rint(x)), &v.y, &v.x);
        }
        table[r][i] = v;
    }
    __syncthreads();
    // slot = (row, head), heads or rows running fastest; a thread steps kSlots slots at a time
    const int f0 = (int)(threadIdx.x % kPieces) * kCount, slots = rows * a.H, half = a.rot / 2;
    int slot = threadIdx.x / kPieces;
    const int inner = a.heads_first ? a.H : rows;
    int lo = slot % inner, hi = slot / inner;
    const int lo_step = kSlots % inner, hi_step = kSlots / inner;
    const bool second = f0 >= half;
#pragma unroll 2
    for (; slot < slots; slot += kSlots) {
        const int h = a.heads_first ? lo : hi, r = a.heads_first ? hi : lo;
        const int64_t in_at = in_row[r] + h * a.sh + f0, out_at = out_row[r] + h * a.oh + f0;
        Piece<T> x[NT], y[NT];
#pragma unroll
        for (int w = 0; w < NT; ++w) {
            const T* p = static_cast<const T*>(a.in[w]) + in_at;
            x[w].load(p);
            if (LAYOUT == kHalves && f0 < a.rot) y[w].load(second ? p - half : p + half);
            if (LAYOUT == kHalvesApart)
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    const int f = f0 + e;
                    if (f < a.rot) y[w].x[e] = f < half ? p[e + half] : p[e - half];
                }
        }
#pragma unroll
        for (int w = 0; w < NT; ++w) {
            Piece<T> o = x[w];
            if (LAYOUT == kNeighbours) {
#pragma unroll
                for (int e = 0; e < kCount; e += 2)
                    if (f0 + e < a.rot) {
                        const float2 t = table[r][(f0 + e) / 2];
                        const float u = to_f32(x[w].x[e]), v = to_f32(x[w].x[e + 1]);
                        from_f32(u * t.x - v * t.y, o.x[e]);
                        from_f32(v * t.x + u * t.y, o.x[e + 1]);
                    }
            } else {
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    const int f = f0 + e;
                    const bool is_second = LAYOUT == kHalves ? second : f >= half;
                    if (LAYOUT == kHalves ? f0 < a.rot : f < a.rot) {
                        const float2 t = table[r][is_second ? f - half : f];
                        from_f32(to_f32(x[w].x[e]) * t.x + to_f32(y[w].x[e]) * (is_second ? t.y : -t.y), o.x[e]);
                    }
                }
            }
            o.store(static_cast<T*>(a.out[w]) + out_at);
        }
        lo += lo_step;
        hi += hi_step;
        if (lo >= inner) {
            lo -= inner;
            ++hi;
        }
    }
}

// rows of a workgroup: 16, fewer where that leaves compute units idle (a decoding step is one row of every sequence)
int rotary_rows(int64_t rows) {
    int each = kRotaryRows;
    while (each > 1 && rows / each < 1024) each /= 2;
    return each;
}

template <typename T, PairLayout LAYOUT>
int launch_rotary(RotaryArgs& a, hipStream_t st) {
    a.each = rotary_rows(a.rows);
    const dim3 grid((unsigned)((a.rows + a.each - 1) / a.each));
    if (a.in[1])
        BPT_LAUNCH("rotary_kernel", (rotary_kernel<T, LAYOUT, 2>), grid, dim3(256), 0, st, a);
    else
        BPT_LAUNCH("rotary_kernel", (rotary_kernel<T, LAYOUT, 1>), grid, dim3(256), 0, st, a);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}
template <typename T>
int launch_rotary(RotaryArgs& a, bool interleaved, hipStream_t st) {
    if (interleaved) return launch_rotary<T, kNeighbours>(a, st);
    return (a.rot / 2) % Piece<T>::kCount ? launch_rotary<T, kHalvesApart>(a, st) : launch_rotary<T, kHalves>(a, st);
}

// no two rows of [B][H][N][kD] with these strides overlap: see bpt_rotary_t
bool rows_apart(int64_t B, int64_t H, int64_t N, int64_t sb, int64_t sh, int64_t sn) {
    std::pair<int64_t, int64_t> s[3] = {{sb, B}, {sh, H}, {sn, N}};
    std::sort(s, s + 3);
    int64_t least = kD;
    for (const auto& x : s) {
        if (x.second == 1) continue;
        if (x.first < least || x.first > INT64_MAX / x.second) return false;
        least = x.first * x.second;
    }
    return true;
}

struct PositionArgs {
    const int32_t* delta;   // [level][sequence] first row minus first id, or null: one sequence, rows are ids
    float* pos;
    int32_t n, lg, rows, batch, levels;
};
__global__ void __launch_bounds__(256) node_positions_kernel(const PositionArgs a) {
    const int row = blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    int level, m;
    if (a.delta) {
        // the last (level, sequence) whose first row is not behind this one (first rows ascend in that order; a
        // sequence without nodes of a level has the first row of the next one, so the last such entry holds the row)
        int lo = 0, hi = a.levels * a.batch - 1;
        auto first_row = [&](int i) { return a.delta[i] + (2 * a.n - ((2 * a.n) >> (i / a.batch))); };
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first_row(mid) <= row) lo = mid;
            else hi = mid - 1;
        }
        level = lo / a.batch;
        m = row - first_row(lo);
    } else {
        const int x = 2 * a.n - row;               // (n >> l) < x <= (2n >> l) on level l
        level = a.lg - (31 - __clz(x - 1));
        m = ((2 * a.n) >> level) - x;
    }
    a.pos[row] = (float)m * (float)(1 << level) + 0.5f * (float)((1 << level) - 1);
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" {

int bpt_rotary(const bpt_rotary_t* s, const float* pos, int64_t pos_stride_b, const void* Q, const void* K, void* Qr, void* Kr,
               void* stream) {
    if (!s || s->B < 0 || s->H < 0 || s->N < 0) return BPT_ERR_INVALID_ARG;
    if (s->D != kD || (s->dtype != BPT_F32 && s->dtype != BPT_BF16)) return BPT_ERR_UNSUPPORTED;
    if (s->rot < 2 || s->rot > kD || (s->rot & 1)) return BPT_ERR_INVALID_ARG;
    int64_t in[3] = {s->stride_b, s->stride_h, s->stride_n}, out[3] = {s->out_stride_b, s->out_stride_h, s->out_stride_n};
    const int32_t count[3] = {s->B, s->H, s->N};
    for (int i = 0; i < 3; ++i) {
        if (count[i] == 1) in[i] = out[i] = 0;   // (one entry: its stride says nothing)
        if (in[i] < 0 || out[i] < 0 || ((in[i] | out[i]) & 7)) return BPT_ERR_INVALID_ARG;
    }
    const double base = s->base > 0 ? s->base : 10000.0, factor = s->factor > 0 ? s->factor : 1.0;
    const double low = s->low == 0 && s->high == 0 ? 1.0 : s->low, high = s->low == 0 && s->high == 0 ? 32.0 : s->high;
    if (!(std::isfinite(base) && std::isfinite(factor) && std::isfinite(s->context) && s->context >= 0 && low < high) ||
        !std::isfinite(high - low) || std::isnan(s->base) || std::isnan(s->factor) || pos_stride_b < 0)
        return BPT_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)s->B * s->N;
    if (rows > (1 << 28) - 32 || s->H > 65535) return BPT_ERR_UNSUPPORTED;   // a launch has fewer than 2^32 threads, 256 for 16 rows
    if (rows == 0 || s->H == 0) return BPT_OK;
    if (!pos || !Q || !Qr || !K != !Kr || (reinterpret_cast<uintptr_t>(pos) & 3) || off_boundary(Q, K, Qr, Kr) || Qr == Kr) return BPT_ERR_INVALID_ARG;
    if (!rows_apart(s->B, s->H, s->N, out[0], out[1], out[2])) return BPT_ERR_INVALID_ARG;
    const bool same = in[0] == out[0] && in[1] == out[1] && in[2] == out[2];
    if (((Q == Qr || (K && K == Kr)) && !same) || Qr == K || (Kr && Kr == Q)) return BPT_ERR_INVALID_ARG;
    RotaryArgs a = {};
    a.in[0] = Q; a.in[1] = K;
    a.out[0] = Qr; a.out[1] = Kr;
    a.pos = pos; a.pos_sb = pos_stride_b;
    a.sb = in[0]; a.sh = in[1]; a.sn = in[2];
    a.ob = out[0]; a.oh = out[1]; a.on = out[2];
    a.N = s->N; a.H = s->H; a.rot = s->rot;
    a.rows = rows;
    a.heads_first = in[1] < (s->N == 1 ? in[0] : in[2]);
    const double kTwoPi = 6.283185307179586476925286766559;
    const double step = std::pow(base, -2.0 / s->rot);
    double w = 1.0;   // 32 products of the step at most: relative error below 32 * 2^-53
    for (int i = 0; i < s->rot / 2; ++i, w *= step) {
        const double turns = s->context * w / kTwoPi;
        const double keep = s->context > 0 ? std::min(1.0, std::max(0.0, (turns - low) / (high - low))) : 0.0;
        a.turns[i] = w * (keep + (1.0 - keep) / factor) / kTwoPi * (s->inverse ? -1.0 : 1.0);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    return s->dtype == BPT_BF16 ? launch_rotary<bf16_t>(a, s->interleaved != 0, st) : launch_rotary<float>(a, s->interleaved != 0, st);
}

int bpt_node_positions(const bpt_graph_t* g, float* pos, void* stream) {
    if (!g || !pos || off_boundary(pos)) return BPT_ERR_INVALID_ARG;
    int device = 0;
    BPT_HIP(hipGetDevice(&device));
    if (device != g->device) return BPT_ERR_INVALID_ARG;   // (a batch graph's tables are the memory of its own)
    hipStream_t st = static_cast<hipStream_t>(stream);
    const UseOnReturn use = {g, st};
    PositionArgs a = {};
    a.delta = g->batch > 0 ? g->d_delta : nullptr;
    a.pos = pos;
    a.n = g->n;
    a.lg = 31 - __builtin_clz((unsigned)g->n);
    a.rows = g->num_nodes;
    a.batch = std::max(g->batch, 1);
    a.levels = g->num_levels;
    BPT_LAUNCH("node_positions_kernel", node_positions_kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, st, a);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}

}  // extern "C"
