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
    int64_t items;                    // B * N * items per row
    int32_t N, H, heads_each, rot;
    double turns[kD / 2];             // w_i' / (2 pi), negative for the inverse
};

// V consecutive values of a row
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T x[V];
};
__device__ __forceinline__ float to_f32(bf16_t x) { return bf16_as_f32(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void from_f32(float v, bf16_t& x) { x = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void from_f32(float v, float& x) { x = v; }

// A thread owns one item of a row -- V pairs, 2 V features -- and turns it in `heads_each` heads of Q and K, so that
// an angle's sine and cosine (64-bit product, reduced to a turn, then fp32) are formed once for up to 2 H uses.
// HALVES: the pairs' first features are V consecutive ones, the second ones V more, rot / 2 further on; else a pair
// is two neighbours.  Items behind rot / (2 V) are features that are copied.  V is the largest of 8 (fp32: 4), 4, 2, 1
// that divides rot / 2, so that an access is 16 bytes wherever the layout allows it.
template <typename T, int V, bool HALVES, int NT>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
    constexpr int kItems = kD / (2 * V);
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= a.items) return;
    const int item = (int)(t % kItems);
    const uint32_t row = (uint32_t)(t / kItems);
    const uint32_t b = row / (uint32_t)a.N, n = row - b * (uint32_t)a.N;
    const int h0 = blockIdx.y * a.heads_each, h1 = min(a.H, h0 + a.heads_each);
    const bool turned = item * 2 * V < a.rot;
    const int at0 = turned && HALVES ? item * V : item * 2 * V;
    const int at1 = turned && HALVES ? a.rot / 2 + item * V : item * 2 * V + V;
    float c[V], s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = 1.f;
        s[v] = 0.f;
    }
    if (turned) {
        const double p = (double)a.pos[(int64_t)b * a.pos_sb + n];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const double x = p * a.turns[item * V + v];
            sincospif(2.f * (float)(x - rint(x)), &s[v], &c[v]);
        }
    }
    const int64_t in_at = (int64_t)b * a.sb + (int64_t)n * a.sn, out_at = (int64_t)b * a.ob + (int64_t)n * a.on;
#pragma unroll 2
    for (int h = h0; h < h1; ++h) {
        Pack<T, V> x0[NT], x1[NT];
#pragma unroll
        for (int w = 0; w < NT; ++w) {
            const T* p = static_cast<const T*>(a.in[w]) + in_at + h * a.sh;
            x0[w] = *reinterpret_cast<const Pack<T, V>*>(p + at0);
            x1[w] = *reinterpret_cast<const Pack<T, V>*>(p + at1);
        }
#pragma unroll
        for (int w = 0; w < NT; ++w) {
            T* p = static_cast<T*>(a.out[w]) + out_at + h * a.oh;
            if (turned) {
                T x[2 * V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    x[v] = x0[w].x[v];
                    x[V + v] = x1[w].x[v];
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int i = HALVES ? v : 2 * v, j = HALVES ? V + v : 2 * v + 1;
                    const float f = to_f32(x[i]), g = to_f32(x[j]);
                    from_f32(f * c[v] - g * s[v], x[i]);
                    from_f32(g * c[v] + f * s[v], x[j]);
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    x0[w].x[v] = x[v];
                    x1[w].x[v] = x[V + v];
                }
            }
            *reinterpret_cast<Pack<T, V>*>(p + at0) = x0[w];
            *reinterpret_cast<Pack<T, V>*>(p + at1) = x1[w];
        }
    }
}

// heads per thread: all of them where the rows alone fill the device, fewer for few rows (a decoding step is one row
// of every sequence), down to one
int heads_each(int64_t items, int H) {
    const int64_t threads = (int64_t)256 * 2048;   // what 256 compute units hold
    const int64_t parts = std::min<int64_t>(H, std::max<int64_t>(1, threads / std::max<int64_t>(items, 1)));
    return (int)((H + parts - 1) / parts);
}

template <typename T, int V, bool HALVES>
int launch_rotary(RotaryArgs& a, int64_t rows, hipStream_t st) {
    constexpr int kItems = kD / (2 * V);
    a.items = rows * kItems;
    a.heads_each = heads_each(a.items, a.H);
    const dim3 grid((unsigned)((a.items + 255) / 256), (unsigned)((a.H + a.heads_each - 1) / a.heads_each));
    if (a.in[1])
        BPT_LAUNCH("rotary_kernel", (rotary_kernel<T, V, HALVES, 2>), grid, dim3(256), 0, st, a);
    else
        BPT_LAUNCH("rotary_kernel", (rotary_kernel<T, V, HALVES, 1>), grid, dim3(256), 0, st, a);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}
template <typename T, int V>
int launch_rotary(RotaryArgs& a, int64_t rows, bool interleaved, hipStream_t st) {
    return interleaved ? launch_rotary<T, V, false>(a, rows, st) : launch_rotary<T, V, true>(a, rows, st);
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
    const int64_t in[3] = {s->stride_b, s->stride_h, s->stride_n}, out[3] = {s->out_stride_b, s->out_stride_h, s->out_stride_n};
    for (int i = 0; i < 3; ++i)
        if (in[i] < 0 || out[i] < 0 || ((in[i] | out[i]) & 7)) return BPT_ERR_INVALID_ARG;
    const double base = s->base > 0 ? s->base : 10000.0, factor = s->factor > 0 ? s->factor : 1.0;
    const double low = s->low == 0 && s->high == 0 ? 1.0 : s->low, high = s->low == 0 && s->high == 0 ? 32.0 : s->high;
    if (!(std::isfinite(base) && std::isfinite(factor) && std::isfinite(s->context) && s->context >= 0 && low < high) ||
        !std::isfinite(high - low) || std::isnan(s->base) || std::isnan(s->factor) || pos_stride_b < 0)
        return BPT_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)s->B * s->N;
    if (rows >= INT32_MAX || s->H > 65535) return BPT_ERR_UNSUPPORTED;
    if (rows == 0 || s->H == 0) return BPT_OK;
    if (!pos || !Q || !Qr || !K != !Kr || off_boundary(pos, Q, K, Qr, Kr) || Qr == Kr) return BPT_ERR_INVALID_ARG;
    if (!rows_apart(s->B, s->H, s->N, out[0], out[1], out[2])) return BPT_ERR_INVALID_ARG;
    const bool same = (s->B == 1 || in[0] == out[0]) && (s->H == 1 || in[1] == out[1]) && (s->N == 1 || in[2] == out[2]);
    if (((Q == Qr || (K && K == Kr)) && !same) || Qr == K || (Kr && Kr == Q)) return BPT_ERR_INVALID_ARG;
    RotaryArgs a = {};
    a.in[0] = Q; a.in[1] = K;
    a.out[0] = Qr; a.out[1] = Kr;
    a.pos = pos; a.pos_sb = pos_stride_b;
    a.sb = in[0]; a.sh = in[1]; a.sn = in[2];
    a.ob = out[0]; a.oh = out[1]; a.on = out[2];
    a.N = s->N; a.H = s->H; a.rot = s->rot;
    const double kTwoPi = 6.283185307179586476925286766559;
    const double step = std::pow(base, -2.0 / s->rot);
    double w = 1.0;   // 32 products of the step at most: relative error below 32 * 2^-53
    for (int i = 0; i < s->rot / 2; ++i, w *= step) {
        const double turns = s->context * w / kTwoPi;
        const double keep = s->context > 0 ? std::min(1.0, std::max(0.0, (turns - low) / (high - low))) : 0.0;
        a.turns[i] = w * (keep + (1.0 - keep) / factor) / kTwoPi * (s->inverse ? -1.0 : 1.0);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool il = s->interleaved != 0;
    const int half = s->rot / 2;
    if (s->dtype == BPT_BF16) {
        if (half % 8 == 0) return launch_rotary<bf16_t, 8>(a, rows, il, st);
        if (half % 4 == 0) return launch_rotary<bf16_t, 4>(a, rows, il, st);
        if (half % 2 == 0) return launch_rotary<bf16_t, 2>(a, rows, il, st);
        return launch_rotary<bf16_t, 1>(a, rows, il, st);
    }
    if (half % 4 == 0) return launch_rotary<float, 4>(a, rows, il, st);
    if (half % 2 == 0) return launch_rotary<float, 2>(a, rows, il, st);
    return launch_rotary<float, 1>(a, rows, il, st);
}

int bpt_node_positions(const bpt_graph_t* g, float* pos, void* stream) {
    if (!g || !pos || off_boundary(pos)) return BPT_ERR_INVALID_ARG;
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
