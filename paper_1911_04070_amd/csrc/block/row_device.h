// Helpers shared by the row operators beside the layer: 8 consecutive values of a row as fp32, checks of pointers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bpt_internal.h"

namespace bpt {
namespace {

typedef uint16_t bf16_t;

__device__ __forceinline__ float bf16_as_f32(uint32_t bits16) { return __uint_as_float(bits16 << 16); }
// two floats -> packed bf16 pair, round to nearest even
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const bf16x2_t v = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, v);
}

// 8 consecutive values as they lie in memory, and as fp32
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16_t> {
    uint4 w;
    __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float* v) const {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = bf16_as_f32(x[e] & 0xFFFFu);
            v[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
        }
    }
};
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const float4*>(p);
        b = *reinterpret_cast<const float4*>(p + 4);
    }
    __device__ __forceinline__ void get(float* v) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
__device__ __forceinline__ void store8(bf16_t* p, const float* v) {
    *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
// every tensor starts on a 16-byte boundary (null passes: optional arguments are checked where they are used)
template <typename... P>
bool off_boundary(P... p) {
    const uintptr_t bits = (... | reinterpret_cast<uintptr_t>(static_cast<const void*>(p)));
    return (bits & 15u) != 0;
}

inline bpt_row_strides_t row_strides(const bpt_row_strides_t* given, int64_t all) {
    return given ? *given : bpt_row_strides_t{all, all, all, all};
}
// rows of d elements may lie `stride` apart: they do not overlap and start on 16-byte boundaries
inline bool stride_ok(int64_t stride, int64_t d, int64_t most) { return stride >= d && !(stride & 7) && stride <= most; }
// a result in the place of an input has its rows in the input's places
inline bool same_place(const void* out, const void* in, int64_t rows, int64_t out_stride, int64_t in_stride) {
    return out != in || !out || rows <= 1 || out_stride == in_stride;
}

}  // namespace
}  // namespace bpt
