// fp32, bf16 and fp16 elements of the entry points that take an lpdt_dtype (not part of the ABI).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"

namespace lpdt {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);        // to nearest, halves to even
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// The elements of a 32-bit word of memory: one fp32, or two of 16 bits (the lower address first).
__device__ __forceinline__ void unpack_word(uint32_t w, float *f, float) { f[0] = __uint_as_float(w); }
__device__ __forceinline__ void unpack_word(uint32_t w, float *f, __nv_bfloat16) {
    f[0] = __uint_as_float(w << 16);
    f[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack_word(uint32_t w, float *f, __half) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    f[0] = v.x;
    f[1] = v.y;
}
__device__ __forceinline__ uint32_t pack_word(const float *f, float) { return __float_as_uint(f[0]); }
__device__ __forceinline__ uint32_t pack_word(const float *f, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f[0], f[1]);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack_word(const float *f, __half) {
    const __half2 v = __floats2half2_rn(f[0], f[1]);
    return *reinterpret_cast<const uint32_t *>(&v);
}

static inline size_t dtype_size(lpdt_dtype t) { return t == LPDT_F32 ? 4 : 2; }
static inline bool dtype_ok(lpdt_dtype t) { return t == LPDT_F32 || t == LPDT_BF16 || t == LPDT_F16; }

// f(a value of the element type) for the type that `t` names
template <typename F>
static inline lpdt_status with_dtype(lpdt_dtype t, F &&f) {
    switch (t) {
        case LPDT_F32: return f(float());
        case LPDT_BF16: return f(__nv_bfloat16());
        case LPDT_F16: return f(__half());
    }
    return LPDT_ERR_INVALID_ARG;
}

}  // namespace lpdt
