// Norms before and after a sublayer with its gate and the residual sum, forward and backward:
//   y = residual_scale * x + gate * post(branch),   h = pre(y).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "bpt_internal.h"
#include "row_device.h"

namespace bpt {
namespace {

// A row is worked on by THREADS threads, 8 consecutive features each: the smallest of 8, 16, 32 (part of a wavefront),
// 64, 128, 256, 512 (1 to 8 wavefronts) that covers d, so that the row stays in registers between its passes whatever d is; a
// workgroup of 256 threads (or THREADS) works on several rows side by side.  (Other multiples of 64 leave fewer threads idle and
// compute units worse filled: 30 000 rows of 1032 in bf16, backward with 192 threads 183 us, with 256 131 us.  500 000 rows of 64 in
// bf16 with 16 threads a row: forward 70 us, with its backward 199 us; with 8: 44 and 143 us.)  Just above a power of two nearly half
// the threads have no columns and as many bytes less are on their way: those 30 000 rows' bytes alone would take the backward 76 us.
struct NormArgs {
    const void *x, *branch, *gate, *dy, *dh;
    const float *post_gain, *post_bias, *pre_gain, *pre_bias;
    const float4* stats;
    void *y, *h, *dx, *d_branch;
    float4* stats_out;
    void* d_gate;          // written by the row kernel where a gate row has one slice, else by the sum over slices
    float* gate_part;      // [units][d]: sums of a slice of a gate row's rows
    float* part;           // [gridDim.x][sums][d]: sums over a workgroup's rows
    int64_t rows, gate_rows;
    bpt_row_strides_t stride;
    int32_t d, post, pre;
    float residual_scale, eps;
    // a workgroup takes units blockIdx.x, + gridDim.x, ..: unit u is slice u % slices of the rows of gate row u / slices
    // (one gate row for all rows where there is no gate, or one for every row)
    int64_t units, unit_rows, group_rows;
    int32_t slices, num_sums;
    int32_t sum_at[4];     // position of post gain, post bias, pre gain, pre bias among the sums, -1: not wanted
};

template <int THREADS>
struct RowTeam {
    static constexpr int kBlock = THREADS < 256 ? 256 : THREADS;
    static constexpr int kRows = kBlock / THREADS;       // rows side by side in a workgroup
    static constexpr int kWaves = THREADS <= 64 ? 1 : THREADS / 64;
};

// Sums of two values over the THREADS threads of a row, in all of them; in a fixed order.  `slot` alternates between two
// buffers, so that one barrier per exchange is enough.
template <int THREADS>
__device__ __forceinline__ void row_sums(float& u, float& v, float2* lds, int& slot) {
    constexpr int kLanes = THREADS < 64 ? THREADS : 64;
#pragma unroll
    for (int s = 1; s < kLanes; s <<= 1) {
        u += __shfl_xor(u, s);
        v += __shfl_xor(v, s);
    }
    if constexpr (THREADS > 64) {
        constexpr int kWaves = THREADS / 64, kBlockWaves = RowTeam<THREADS>::kBlock / 64;
        const int wave = threadIdx.x >> 6, first = wave / kWaves * kWaves;
        float2* mine = lds + slot * kBlockWaves;
        slot ^= 1;
        if ((threadIdx.x & 63) == 0) mine[wave] = make_float2(u, v);
        __syncthreads();
        u = v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 p = mine[first + w];
            u += p.x;
            v += p.y;
        }
    }
}

// Mean and 1 / deviation of a row whose 8 values this thread holds (zeros where it has none, `has` false); the second
// pass subtracts the mean before it squares.
template <int THREADS>
__device__ __forceinline__ float2 row_stats(const float* v, bool has, int kind, float inv_d, float eps, float2* lds, int& slot) {
    float mean = 0.f, sq = 0.f, none = 0.f;
    if (kind == BPT_NORM_LAYER) {
#pragma unroll
        for (int e = 0; e < 8; ++e) mean += v[e];
        row_sums<THREADS>(mean, none, lds, slot);
        mean *= inv_d;
    }
    if (has)
#pragma unroll
        for (int e = 0; e < 8; ++e) sq += (v[e] - mean) * (v[e] - mean);
    none = 0.f;
    row_sums<THREADS>(sq, none, lds, slot);
    return make_float2(mean, 1.f / sqrtf(sq * inv_d + eps));
}

__device__ __forceinline__ void params8(const float* p, int col, bool has, float otherwise, float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = otherwise;
    if (p && has) {
        Raw8<float> w;
        w.load(p + col);
        w.get(v);
    }
}

// Bound by HBM: x and branch in, y and h out, the row in registers in between; parameters of a thread's columns stay in
// registers, the next row is loaded before the current one's sums are exchanged.  65 532 rows of 512 in bf16, a gate row for every
// 16 383: 49 us, 5.5 TB/s (a large copy reaches 4.9 on the same device; part of what it moves is still in the memory-side
// cache); 4095 rows of 2048 in fp32: 28 us, 4.9 TB/s.  92 to 114 registers, none spilled.
template <typename T, int THREADS>
__global__ void __launch_bounds__(RowTeam<THREADS>::kBlock, sizeof(T) == 2 ? 5 : 4) residual_norm_kernel(const NormArgs a) {
    using Team = RowTeam<THREADS>;
    __shared__ float2 lds[2 * Team::kBlock / 64];
    int slot = 0;
    const int col = (int)(threadIdx.x % THREADS) * 8;
    const bool has = col < a.d;
    const float inv_d = 1.f / (float)a.d;
    const int64_t step = (int64_t)gridDim.x * Team::kRows;
    const int64_t first = (int64_t)blockIdx.x * Team::kRows;
    int64_t row = first + threadIdx.x / THREADS;
    float g1[8], b1[8], g2[8], b2[8];
    params8(a.post_gain, col, has, 1.f, g1);
    params8(a.post_bias, col, has, 0.f, b1);
    params8(a.pre_gain, col, has, 1.f, g2);
    params8(a.pre_bias, col, has, 0.f, b2);
    const T *px = static_cast<const T*>(a.x), *pb = static_cast<const T*>(a.branch), *pg = static_cast<const T*>(a.gate);
    Raw8<T> xw = {}, bw = {}, gw = {};
    auto fetch = [&](int64_t r) {
        if (!has || r >= a.rows) return;
        xw.load(px + r * a.stride.x + col);
        if (pb) bw.load(pb + r * a.stride.branch + col);
        if (pg) gw.load(pg + (int64_t)((uint32_t)r / (uint32_t)a.gate_rows) * a.d + col);
    };
    fetch(row);
    // (every thread of a workgroup makes as many turns as its first row needs: the exchanges are barriers)
    for (int64_t at = first; at < a.rows; at += step, row += step) {
        float x[8], b[8], g[8];
        xw.get(x);
        bw.get(b);
        gw.get(g);
        fetch(row + step);
        const bool live = has && row < a.rows;
        float2 sb = make_float2(0.f, 1.f), sy = make_float2(0.f, 1.f);
        if (a.post != BPT_NORM_NONE) sb = row_stats<THREADS>(b, has, a.post, inv_d, a.eps, lds, slot);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = a.post != BPT_NORM_NONE ? (b[e] - sb.x) * sb.y * g1[e] + b1[e] : b[e];
            if (pg) v *= g[e];
            x[e] = has ? a.residual_scale * x[e] + (pb ? v : 0.f) : 0.f;
        }
        if (a.pre != BPT_NORM_NONE) sy = row_stats<THREADS>(x, has, a.pre, inv_d, a.eps, lds, slot);
        if (!live) continue;
        if (a.y) store8(static_cast<T*>(a.y) + row * a.stride.out + col, x);
        if (a.pre != BPT_NORM_NONE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (x[e] - sy.x) * sy.y * g2[e] + b2[e];
            store8(static_cast<T*>(a.h) + row * a.stride.out + col, x);
        }
        if (a.stats_out && col == 0) a.stats_out[row] = make_float4(sb.x, sb.y, sy.x, sy.y);
    }
}

// With bhat, yhat the normalised rows and yhat's gradient t = dh g2:
//   dY = dy + ry (t - [layer] mean(t) - yhat mean(t yhat))     dx = residual_scale dY
//   dN = gate dY,  d_gate = sum over the gate row's rows of dY post(branch)
//   d_branch = rb (s - [layer] mean(s) - bhat mean(s bhat)),  s = dN g1
// and column sums dN bhat, dN, dh yhat, dh for gains and biases.  x and branch are read again (y is formed from them in
// fp32 as the forward did, not from its rounded copy), six values of memory traffic per element; the sums stay in the
// thread's registers over all rows of its workgroup, which leaves two wavefronts per SIMD: rows have to be requested early.
// 65 532 rows of 512 in bf16: 89 us, 4.5 TB/s (one row ahead instead of two: 100 us); 4095 rows of 2048 in fp32: 42 us, 4.7 TB/s.
// A unit's rows are requested when it begins, and its gate row's sum is taken over all teams, so that gates of very few rows leave
// teams idle and wait for memory once per gate row: 65 532 rows of 64, bf16, 27 us with a gate for every row, 263 us with one for
// every two; of 512, 149 us with one for every three.
// A row's number as a new value to the compiler, which else keeps a running offset in registers for every tensor and row on its way
// (with strides of their own for the tensors 256 registers and up to 9 spilled; so 218 to 240 and none)
__device__ __forceinline__ uint32_t hidden(uint32_t v) {
    asm("" : "+v"(v));
    return v;
}
template <typename T, int THREADS>
__global__ void __launch_bounds__(RowTeam<THREADS>::kBlock, 2) residual_norm_bwd_kernel(const NormArgs a) {
    using Team = RowTeam<THREADS>;
    __shared__ float2 lds[2 * Team::kBlock / 64];
    __shared__ float gather[Team::kRows > 1 ? (Team::kRows - 1) * THREADS * 8 : 1];
    int slot = 0;
    const int col = (int)(threadIdx.x % THREADS) * 8, team = threadIdx.x / THREADS;
    const bool has = col < a.d;
    const float inv_d = 1.f / (float)a.d;
    float g1[8], b1[8], g2[8];
    params8(a.post_gain, col, has, 1.f, g1);
    params8(a.post_bias, col, has, 0.f, b1);
    params8(a.pre_gain, col, has, 1.f, g2);
    float sums[4][8] = {}, sum_gate[8] = {};
    const T *px = static_cast<const T*>(a.x), *pb = static_cast<const T*>(a.branch), *pg = static_cast<const T*>(a.gate);
    const T *pdy = static_cast<const T*>(a.dy), *pdh = static_cast<const T*>(a.dh);
    const bool gate_each = pg && a.gate_rows == 1;
    // adds the teams' values in order; the result is the first team's
    auto over_teams = [&](float* v) {
        if constexpr (Team::kRows > 1) {
            __syncthreads();
            if (team > 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) gather[(team - 1) * THREADS * 8 + e * THREADS + threadIdx.x % THREADS] = v[e];
            __syncthreads();
            if (team == 0)
                for (int t = 0; t < Team::kRows - 1; ++t)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += gather[t * THREADS * 8 + e * THREADS + threadIdx.x % THREADS];
        }
    };
    for (int64_t unit = blockIdx.x; unit < a.units; unit += gridDim.x) {
        const int64_t group = unit / a.slices, slice = unit - group * a.slices;
        const int64_t begin = group * a.group_rows + slice * a.unit_rows;
        const int64_t end = min(min(begin + a.unit_rows, (group + 1) * a.group_rows), a.rows);
        // as many rows are on their way as registers allow: two in bf16, one in fp32
        constexpr int kAhead = sizeof(T) == 2 ? 2 : 1;
        struct Row {
            Raw8<T> x, b, g, dy, dh;
            float4 st;
        } rows[kAhead] = {};
        Raw8<T> gate = {};
        if (pg && !gate_each && has && begin < end) gate.load(pg + group * a.d + col);
        auto fetch = [&](Row& w, int64_t r) {
            w.st = make_float4(0.f, 1.f, 0.f, 1.f);
            if (r >= end) return;
            w.st = a.stats[r];
            if (!has) return;
            const uint32_t at_row = hidden((uint32_t)r);
            w.x.load(px + at_row * a.stride.x + col);
            if (pb) w.b.load(pb + at_row * a.stride.branch + col);
            const int64_t at = at_row * a.stride.grad + col;
            if (pdy) w.dy.load(pdy + at);
            if (pdh) w.dh.load(pdh + at);
            if (gate_each) w.g.load(pg + at_row * (int64_t)a.d + col);
        };
        auto work = [&](Row& w, int64_t row) {
            const bool live = has && row < end;
            float x[8], b[8], g[8], dy[8], dh[8];
            w.x.get(x);
            w.b.get(b);
            (gate_each ? w.g : gate).get(g);
            w.dy.get(dy);
            w.dh.get(dh);
            const float4 s = w.st;
            fetch(w, row + kAhead * Team::kRows);
            float bn[8];   // post(branch)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!live) b[e] = x[e] = dy[e] = dh[e] = 0.f;
                if (!pdy) dy[e] = 0.f;
                if (!pdh) dh[e] = 0.f;
                if (!pg) g[e] = 1.f;
                if (a.post != BPT_NORM_NONE) b[e] = (b[e] - s.x) * s.y;
                bn[e] = a.post != BPT_NORM_NONE ? b[e] * g1[e] + b1[e] : b[e];
                x[e] = a.residual_scale * x[e] + (pb ? g[e] * bn[e] : 0.f);   // y
                x[e] = (x[e] - s.z) * s.w;                                    // yhat
            }
            if (a.pre != BPT_NORM_NONE && pdh) {
                float m1 = 0.f, m2 = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float t = dh[e] * g2[e];
                    m1 += t;
                    m2 += live ? t * x[e] : 0.f;
                    if (live) {
                        sums[2][e] += dh[e] * x[e];
                        sums[3][e] += dh[e];
                    }
                }
                row_sums<THREADS>(m1, m2, lds, slot);
                m1 = a.pre == BPT_NORM_LAYER ? m1 * inv_d : 0.f;
                m2 *= inv_d;
#pragma unroll
                for (int e = 0; e < 8; ++e) dy[e] += s.w * (dh[e] * g2[e] - m1 - x[e] * m2);
            }
            if (live) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = a.residual_scale * dy[e];
                store8(static_cast<T*>(a.dx) + hidden((uint32_t)row) * a.stride.out + col, o);
            }
            if (pg) {
                if (gate_each) {
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = dy[e] * bn[e];
                    if (live) store8(static_cast<T*>(a.d_gate) + hidden((uint32_t)row) * (int64_t)a.d + col, o);
                } else if (live) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum_gate[e] += dy[e] * bn[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) dy[e] *= g[e];
            }
            if (a.post != BPT_NORM_NONE) {
                float m1 = 0.f, m2 = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float t = live ? dy[e] * g1[e] : 0.f;
                    m1 += t;
                    m2 += live ? t * b[e] : 0.f;
                    if (live) {
                        sums[0][e] += dy[e] * b[e];
                        sums[1][e] += dy[e];
                    }
                }
                row_sums<THREADS>(m1, m2, lds, slot);
                m1 = a.post == BPT_NORM_LAYER ? m1 * inv_d : 0.f;
                m2 *= inv_d;
#pragma unroll
                for (int e = 0; e < 8; ++e) dy[e] = s.y * (dy[e] * g1[e] - m1 - b[e] * m2);
            }
            if (live && a.d_branch) store8(static_cast<T*>(a.d_branch) + hidden((uint32_t)row) * a.stride.out + col, dy);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(rows[i], begin + team + i * Team::kRows);
        for (int64_t at = begin; at < end; at += kAhead * Team::kRows) {
            work(rows[0], at + team);
            if (kAhead == 2 && at + Team::kRows < end) work(rows[kAhead - 1], at + team + Team::kRows);
        }
        if (pg && !gate_each) {
            over_teams(sum_gate);
            if (team == 0 && has) {
                if (a.slices == 1) store8(static_cast<T*>(a.d_gate) + group * a.d + col, sum_gate);
                else store8(a.gate_part + unit * a.d + col, sum_gate);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum_gate[e] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (a.sum_at[i] >= 0) {
            over_teams(sums[i]);
            if (team == 0 && has) store8(a.part + ((int64_t)blockIdx.x * a.num_sums + a.sum_at[i]) * a.d + col, sums[i]);
        }
}

// Column sums of up to 4 + gate rows of tables: job j < num_sums adds `parts` rows of part, `num_sums` rows apart; job
// num_sums + g adds the `slices` rows of gate row g.  A workgroup takes 32 columns, 8 lanes of 16 bytes per row, 32 rows
// in flight; sums are added across lanes and wavefronts in a fixed tree.  512 rows of 2 x 512 and 4 x 128 of 512: 4 us.
struct SumJobs {
    const float *part, *gate_part;
    float* out[4];
    void* d_gate;
    int32_t num_sums, parts, slices, d;
};
template <typename T>
__global__ void __launch_bounds__(256) norm_column_sum_kernel(const SumJobs a) {
    __shared__ float4 s[32][8];
    const int lane8 = threadIdx.x & 7, rowlane = threadIdx.x >> 3;
    const int c = blockIdx.x * 32 + lane8 * 4;
    const int job = blockIdx.y;
    const bool gate = job >= a.num_sums;
    const float* src = gate ? a.gate_part + (int64_t)(job - a.num_sums) * a.slices * a.d : a.part + (int64_t)job * a.d;
    const int64_t pitch = gate ? a.d : (int64_t)a.num_sums * a.d;
    const int parts = gate ? a.slices : a.parts;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < a.d) {
#pragma unroll 4
        for (int p = rowlane; p < parts; p += 32) {
            const float4 v = *reinterpret_cast<const float4*>(src + p * pitch + c);
            acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
        }
    }
    s[rowlane][lane8] = acc;
    __syncthreads();
    for (int w = 16; w > 0; w >>= 1) {
        if (rowlane < w) {
            const float4 u = s[rowlane][lane8], v = s[rowlane + w][lane8];
            s[rowlane][lane8] = make_float4(u.x + v.x, u.y + v.y, u.z + v.z, u.w + v.w);
        }
        __syncthreads();
    }
    if (rowlane == 0 && c < a.d) {
        const float4 v = s[0][lane8];
        if (gate && sizeof(T) == 2) {
            T* o = static_cast<T*>(a.d_gate) + (int64_t)(job - a.num_sums) * a.d + c;
            *reinterpret_cast<uint2*>(o) = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
        } else {
            float* o = gate ? static_cast<float*>(a.d_gate) + (int64_t)(job - a.num_sums) * a.d + c : a.out[job] + c;
            *reinterpret_cast<float4*>(o) = v;
        }
    }
}

// compute units; wavefronts per SIMD: forward 5 (bf16) and 4 (fp32), backward 2, as the kernels' launch bounds say
constexpr int kNormCus = 256, kNormBwdBlocks = 2 * 256;

int norm_threads(int d) {
    int t = 8;
    while (t * 8 < d) t *= 2;
    return t;
}

constexpr int64_t kMostStride = (int64_t)1 << 40;
int check_norm(const bpt_residual_norm_t* s) {
    if (!s || s->rows < 0) return BPT_ERR_INVALID_ARG;
    if (s->dtype != BPT_F32 && s->dtype != BPT_BF16) return BPT_ERR_UNSUPPORTED;
    if (s->d < 8 || s->d > 4096 || (s->d & 7) || s->rows >= INT32_MAX) return BPT_ERR_UNSUPPORTED;
    if (!stride_ok(s->stride, s->d, kMostStride)) return BPT_ERR_INVALID_ARG;
    for (int k : {s->post, s->pre})
        if (k != BPT_NORM_NONE && k != BPT_NORM_LAYER && k != BPT_NORM_RMS) return BPT_ERR_INVALID_ARG;
    if (s->gate_rows < 0 || s->gate_rows >= INT32_MAX || !std::isfinite(s->residual_scale) || !std::isfinite(s->eps)) return BPT_ERR_INVALID_ARG;
    return BPT_OK;
}

// how the backward cuts its rows, and where its sums lie in the workspace
struct BwdPlan {
    int64_t groups, group_rows, slices, unit_rows, units;
    int blocks;
    bool gate_sums;        // a gate row's gradient is a sum over several slices
    size_t part, gate_part, total;
};
BwdPlan bwd_plan(const bpt_residual_norm_t* s) {
    BwdPlan p = {};
    const int threads = norm_threads(s->d), block = std::max(threads, 256), teams = block / threads;
    const int64_t most = std::max(1, kNormBwdBlocks * 256 / block);
    const bool shared_gate = s->gate_rows > 1;
    p.group_rows = shared_gate ? std::min(s->gate_rows, s->rows) : s->rows;
    p.groups = (s->rows + p.group_rows - 1) / p.group_rows;
    // as many slices of a group as let the workgroups, which are resident together, end together: the first multiple of a round
    // whose last round is nine tenths full (65 532 rows of 512 in bf16, a gate for 100 rows each: forward and backward 168 us with
    // one round at most, 160 us so)
    const int64_t longest = (p.group_rows + teams - 1) / teams;
    p.slices = 1;
    for (int64_t rounds = 1; rounds <= 8; ++rounds) {
        const int64_t cut = std::max<int64_t>(1, std::min(rounds * most / p.groups, longest)), units = p.groups * cut;
        p.slices = cut;
        if (cut == longest || 10 * units >= 9 * ((units + most - 1) / most * most)) break;
    }
    p.unit_rows = (p.group_rows + p.slices - 1) / p.slices;
    p.unit_rows = (p.unit_rows + teams - 1) / teams * teams;
    p.slices = (p.group_rows + p.unit_rows - 1) / p.unit_rows;
    p.units = p.groups * p.slices;
    p.blocks = (int)std::min(p.units, most);
    p.gate_sums = shared_gate && p.slices > 1;
    p.part = 0;
    p.gate_part = align256((size_t)p.blocks * 4 * s->d * 4);
    p.total = p.gate_part + (p.gate_sums ? align256((size_t)p.units * s->d * 4) : 0);
    return p;
}

template <typename T, int THREADS>
int launch_fwd(const NormArgs& a, hipStream_t st) {
    using Team = RowTeam<THREADS>;
    // as many workgroups as are resident, of equal shares of the rows
    const int64_t most = (int64_t)kNormCus * ((sizeof(T) == 2 ? 5 : 4) * 256 / Team::kBlock);
    const int64_t groups = (a.rows + Team::kRows - 1) / Team::kRows, each = (groups + most - 1) / most;
    const dim3 grid((unsigned)((groups + each - 1) / each));
    BPT_LAUNCH("residual_norm_kernel", (residual_norm_kernel<T, THREADS>), grid, dim3(Team::kBlock), 0, st, a);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}
template <typename T, int THREADS>
int launch_bwd(const NormArgs& a, int blocks, hipStream_t st) {
    BPT_LAUNCH("residual_norm_bwd_kernel", (residual_norm_bwd_kernel<T, THREADS>), dim3(blocks), dim3(RowTeam<THREADS>::kBlock), 0, st, a);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}
template <typename T>
int launch_fwd_any(const NormArgs& a, hipStream_t st) {
    switch (norm_threads(a.d)) {
        case 8: return launch_fwd<T, 8>(a, st);
        case 16: return launch_fwd<T, 16>(a, st);
        case 32: return launch_fwd<T, 32>(a, st);
        case 64: return launch_fwd<T, 64>(a, st);
        case 128: return launch_fwd<T, 128>(a, st);
        case 256: return launch_fwd<T, 256>(a, st);
        default: return launch_fwd<T, 512>(a, st);
    }
}
template <typename T>
int launch_bwd_any(const NormArgs& a, int blocks, hipStream_t st) {
    switch (norm_threads(a.d)) {
        case 8: return launch_bwd<T, 8>(a, blocks, st);
        case 16: return launch_bwd<T, 16>(a, blocks, st);
        case 32: return launch_bwd<T, 32>(a, blocks, st);
        case 64: return launch_bwd<T, 64>(a, blocks, st);
        case 128: return launch_bwd<T, 128>(a, blocks, st);
        case 256: return launch_bwd<T, 256>(a, blocks, st);
        default: return launch_bwd<T, 512>(a, blocks, st);
    }
}

NormArgs norm_args(const bpt_residual_norm_t* s, const bpt_row_strides_t& strides, const void* x, const void* branch, const void* gate, const float* post_gain,
                   const float* post_bias, const float* pre_gain, const float* pre_bias) {
    NormArgs a = {};
    a.stride = strides;
    a.x = x; a.branch = branch; a.gate = gate;
    a.post_gain = post_gain; a.post_bias = post_bias; a.pre_gain = pre_gain; a.pre_bias = pre_bias;
    a.rows = s->rows; a.gate_rows = std::max<int64_t>(s->gate_rows, 1);
    a.d = s->d; a.post = s->post; a.pre = s->pre;
    a.residual_scale = s->residual_scale;
    a.eps = s->eps > 0.f ? s->eps : 1e-5f;
    return a;
}
// what both calls ask of their inputs
int check_inputs(const bpt_residual_norm_t* s, const bpt_row_strides_t& strides, const void* x, const void* branch, const void* gate, const float* post_gain,
                 const float* post_bias, const float* pre_gain, const float* pre_bias) {
    if (!stride_ok(strides.x, s->d, kMostStride) || !stride_ok(strides.out, s->d, kMostStride) ||
        (branch && !stride_ok(strides.branch, s->d, kMostStride)))
        return BPT_ERR_INVALID_ARG;
    if (!x || !gate != (s->gate_rows == 0)) return BPT_ERR_INVALID_ARG;
    if (!branch && (gate || s->post != BPT_NORM_NONE)) return BPT_ERR_INVALID_ARG;
    if (s->post == BPT_NORM_NONE && (post_gain || post_bias)) return BPT_ERR_INVALID_ARG;
    if (s->pre == BPT_NORM_NONE && (pre_gain || pre_bias)) return BPT_ERR_INVALID_ARG;
    return off_boundary(x, branch, gate, post_gain, post_bias, pre_gain, pre_bias) ? BPT_ERR_INVALID_ARG : BPT_OK;
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" {

int bpt_residual_norm_fwd_strided(const bpt_residual_norm_t* s, const bpt_row_strides_t* strides, const void* x, const void* branch,
                                  const void* gate, const float* post_gain, const float* post_bias, const float* pre_gain,
                                  const float* pre_bias, void* y, void* h, float* stats, void* stream) {
    if (const int rc = check_norm(s)) return rc;
    if (s->rows == 0) return BPT_OK;
    const bpt_row_strides_t apart = row_strides(strides, s->stride);
    if (const int rc = check_inputs(s, apart, x, branch, gate, post_gain, post_bias, pre_gain, pre_bias)) return rc;
    if (!h != (s->pre == BPT_NORM_NONE) || (!y && !h) || y == h || off_boundary(y, h, stats)) return BPT_ERR_INVALID_ARG;
    for (const void* o : {y, h})
        if (!same_place(o, x, s->rows, apart.out, apart.x) || !same_place(o, branch, s->rows, apart.out, apart.branch)) return BPT_ERR_INVALID_ARG;
    NormArgs a = norm_args(s, apart, x, branch, gate, post_gain, post_bias, pre_gain, pre_bias);
    a.y = y; a.h = h;
    a.stats_out = reinterpret_cast<float4*>(stats);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return s->dtype == BPT_BF16 ? launch_fwd_any<bf16_t>(a, st) : launch_fwd_any<float>(a, st);
}

int bpt_residual_norm_fwd(const bpt_residual_norm_t* s, const void* x, const void* branch, const void* gate, const float* post_gain,
                          const float* post_bias, const float* pre_gain, const float* pre_bias, void* y, void* h, float* stats,
                          void* stream) {
    return bpt_residual_norm_fwd_strided(s, nullptr, x, branch, gate, post_gain, post_bias, pre_gain, pre_bias, y, h, stats, stream);
}

size_t bpt_residual_norm_bwd_workspace(const bpt_residual_norm_t* s) {
    if (check_norm(s)) return SIZE_MAX;
    return s->rows == 0 ? 0 : bwd_plan(s).total;
}

int bpt_residual_norm_bwd_strided(const bpt_residual_norm_t* s, const bpt_row_strides_t* strides, const void* x, const void* branch,
                                  const void* gate, const float* post_gain, const float* post_bias, const float* pre_gain,
                                  const float* pre_bias, const float* stats, const void* dy, const void* dh, void* dx, void* d_branch,
                                  const bpt_residual_norm_grads_t* grads, void* workspace, size_t workspace_bytes, void* stream) {
    if (const int rc = check_norm(s)) return rc;
    const bpt_row_strides_t apart = row_strides(strides, s->stride);
    if (!grads) return BPT_ERR_INVALID_ARG;
    float* const out[4] = {grads->d_post_gain, grads->d_post_bias, grads->d_pre_gain, grads->d_pre_bias};
    const float* const par[4] = {post_gain, post_bias, pre_gain, pre_bias};
    for (int i = 0; i < 4; ++i)
        if (!out[i] != !par[i] || off_boundary(out[i])) return BPT_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    SumJobs j = {};
    NormArgs a = norm_args(s, apart, x, branch, gate, post_gain, post_bias, pre_gain, pre_bias);
    for (int i = 0; i < 4; ++i) {
        a.sum_at[i] = out[i] ? j.num_sums : -1;
        if (out[i]) j.out[j.num_sums++] = out[i];
    }
    j.d = s->d;
    int64_t gate_jobs = 0;
    if (s->rows > 0) {
        if (const int rc = check_inputs(s, apart, x, branch, gate, post_gain, post_bias, pre_gain, pre_bias)) return rc;
        if (!stats || !dx || !d_branch != !branch || !grads->d_gate != !gate || (dh && s->pre == BPT_NORM_NONE) || (!dy && !dh) ||
            dx == d_branch || off_boundary(stats, dy, dh, dx, d_branch, grads->d_gate, workspace))
            return BPT_ERR_INVALID_ARG;
        if (!stride_ok(apart.grad, s->d, kMostStride)) return BPT_ERR_INVALID_ARG;
        for (const void* g : {dy, dh})
            if (!same_place(dx, g, s->rows, apart.out, apart.grad) || !same_place(d_branch, g, s->rows, apart.out, apart.grad)) return BPT_ERR_INVALID_ARG;
        const BwdPlan p = bwd_plan(s);
        if (!workspace || workspace_bytes < p.total) return BPT_ERR_INVALID_ARG;
        unsigned char* ws = static_cast<unsigned char*>(workspace);
        a.stats = reinterpret_cast<const float4*>(stats);
        a.dy = dy; a.dh = dh; a.dx = dx; a.d_branch = d_branch;
        a.d_gate = grads->d_gate;
        a.part = reinterpret_cast<float*>(ws + p.part);
        a.gate_part = reinterpret_cast<float*>(ws + p.gate_part);
        a.units = p.units; a.unit_rows = p.unit_rows; a.group_rows = p.group_rows;
        a.slices = (int)p.slices;
        a.num_sums = j.num_sums;
        j.part = a.part; j.gate_part = a.gate_part;
        j.d_gate = grads->d_gate;
        j.parts = p.blocks; j.slices = (int)p.slices;
        gate_jobs = gate && p.gate_sums ? p.groups : 0;
        const int rc = s->dtype == BPT_BF16 ? launch_bwd_any<bf16_t>(a, p.blocks, st) : launch_bwd_any<float>(a, p.blocks, st);
        if (rc) return rc;
    }
    // (no rows: sums of nothing)
    if (j.num_sums + gate_jobs == 0) return BPT_OK;
    const dim3 grid((unsigned)((s->d + 31) / 32), (unsigned)(j.num_sums + gate_jobs));
    if (s->dtype == BPT_BF16) BPT_LAUNCH("norm_column_sum_kernel", norm_column_sum_kernel<bf16_t>, grid, dim3(256), 0, st, j);
    else BPT_LAUNCH("norm_column_sum_kernel", norm_column_sum_kernel<float>, grid, dim3(256), 0, st, j);
    BPT_HIP(hipGetLastError());
    return BPT_OK;
}

int bpt_residual_norm_bwd(const bpt_residual_norm_t* s, const void* x, const void* branch, const void* gate, const float* post_gain,
                          const float* post_bias, const float* pre_gain, const float* pre_bias, const float* stats, const void* dy,
                          const void* dh, void* dx, void* d_branch, const bpt_residual_norm_grads_t* grads, void* workspace,
                          size_t workspace_bytes, void* stream) {
    return bpt_residual_norm_bwd_strided(s, nullptr, x, branch, gate, post_gain, post_bias, pre_gain, pre_bias, stats, dy, dh, dx, d_branch,
                                         grads, workspace, workspace_bytes, stream);
}

}  // extern "C"
