// What runs around a block's linear layers besides attention: fused norms and the clipping of gradients.
#pragma once
#include "common.hpp"

namespace onecomp {
namespace block {

// 16 bytes at any address of the element type: the memory system takes them in one load, so that odd widths and offsets cost
// no more than the cache lines they straddle.
typedef uint4v uint4u __attribute__((aligned(2)));
typedef float4v float4u __attribute__((aligned(4)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// eight bf16 or four fp32 values from 16 bytes
__device__ __forceinline__ void load_vector(float (&x)[8], const uint16_t* p) {
    const uint4v v = *reinterpret_cast<const uint4u*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_value(v[i] & 0xffffu);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load_vector(float (&x)[4], const float* p) {
    const float4v v = *reinterpret_cast<const float4u*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
}
__device__ __forceinline__ void store_vector(uint16_t* p, const float (&x)[8]) {
    bf16x8u v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<__bf16>(x[i]);
    *reinterpret_cast<bf16x8u*>(p) = v;
}
__device__ __forceinline__ void store_vector(float* p, const float (&x)[4]) {
    float4v v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x[i];
    *reinterpret_cast<float4u*>(p) = v;
}
__device__ __forceinline__ float load_one(const uint16_t* p) { return bf16_value(*p); }
__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ void store_one(uint16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = static_cast<__bf16>(x); }
__device__ __forceinline__ void store_one(float* p, float x) { *p = x; }

struct Rows {
    void* p;
    int64_t stride;        // elements between rows
};

struct Params {
    Rows h, y, gate;       // forward: h as it comes in; gradients: h' (or h where there is no y)
    Rows h_out, n;
    Rows dn, dh_out, dh, dy, dgate;
    const void *weight, *bias, *post_weight, *post_bias;
    void* d_param[5];      // gradients of weight, bias, post_weight, post_bias, gate per channel
    float *part, *row_numbers;   // scratch; null where no parameter's gradient is wanted
    int64_t rows;
    int width, layer, post, gate_rows, w_bf16, wanted;   // wanted: bits of the d_param that are given
    float scale, eps;
};

onecomp_status norm_run(onecomp_dtype dtype, const Params& P, bool gradient, hipStream_t stream);
size_t gradient_workspace_bytes(int64_t rows, int64_t width, int wanted);

size_t clip_workspace_bytes();
onecomp_status clip_run(const onecomp_gradient* grads, int n, float max_norm, float* norm, void* workspace, hipStream_t stream);

}  // namespace block
}  // namespace onecomp
