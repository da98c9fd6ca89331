// What the head operators (normalisation, gated block, gated recurrence) share: element types, wide loads and stores,
// activations with their slopes.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include "../../include/rrm.h"

namespace rrm {

typedef __nv_bfloat16 bf16;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16_rn(v); }   // the one rounding of an output
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// V neighbouring elements, moved as one access of V * sizeof(T) <= 16 bytes
template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) { return *reinterpret_cast<const Pack<T, V>*>(p); }
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& v) { *reinterpret_cast<Pack<T, V>*>(p) = v; }

// 1 / (1 + e^-z) with the hardware's exponential and division: a few units in the last place of 24 bits, below what any of
// the types stored can tell but fp32, whose outputs it leaves at about 1e-7
__device__ __forceinline__ float sigmoid_f(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }
__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * (1.f + erff(z * 0.70710678118654752f)); }

__device__ __forceinline__ float act_value(int act, float z)
{
    switch (act) {
        case RRM_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
        case RRM_ACT_LEAKY: return z > 0.f ? z : 0.1f * z;
        case RRM_ACT_SIGMOID: return sigmoid_f(z);
        case RRM_ACT_SILU: return z * sigmoid_f(z);
        case RRM_ACT_GELU: return z * normal_cdf(z);
        default: return z;
    }
}

// the value and its derivative by z (at a kink: the slope from below)
__device__ __forceinline__ float act_slope(int act, float z, float& value)
{
    switch (act) {
        case RRM_ACT_RELU: value = z > 0.f ? z : (z != z ? z : 0.f); return z > 0.f ? 1.f : 0.f;
        case RRM_ACT_LEAKY: value = z > 0.f ? z : 0.1f * z; return z > 0.f ? 1.f : 0.1f;
        case RRM_ACT_SIGMOID: { const float q = sigmoid_f(z); value = q; return q * (1.f - q); }
        case RRM_ACT_SILU: { const float q = sigmoid_f(z); value = z * q; return q * fmaf(z, 1.f - q, 1.f); }
        case RRM_ACT_GELU: {
            const float q = normal_cdf(z);
            value = z * q;
            return fmaf(z * 0.39894228040143268f, __expf(-0.5f * z * z), q);
        }
        default: value = z; return 1.f;
    }
}

// host side of the argument checks
inline int head_elem_bytes(int dtype) { return dtype == RRM_F32 ? 4 : 2; }
inline bool head_act_ok(int act)
{
    return act == RRM_ACT_NONE || act == RRM_ACT_RELU || (act >= RRM_ACT_LEAKY && act <= RRM_ACT_GELU);
}
inline bool misaligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

}  // namespace rrm
