// Declarations shared by the operators on cleartext activations (clear_*.cu): element types, checks of descriptors, errors.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "common.cuh"

// These calls have no context: the text of a refused one is kept per host thread.
int clear_fail(int code, const char* what);
#define CLEAR_CUDA(call)                                                       \
    do {                                                                       \
        cudaError_t e_ = (call);                                               \
        if (e_ != cudaSuccess) return clear_fail(FESC_ECUDA, cudaGetErrorString(e_)); \
    } while (0)

// an output at the address of an input or of another output
static inline bool same_buffer(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
    for (auto o = outs.begin(); o != outs.end(); o++) {
        if (!*o) continue;
        for (const void* i : ins)
            if (*o == i) return true;
        for (auto other = outs.begin(); other != o; other++)
            if (*o == *other) return true;
    }
    return false;
}

template <class T>
struct ClearType;
template <>
struct ClearType<__nv_bfloat16> {
    static constexpr int planes = 1;   // bfloat16 numbers that add up to any value exactly
    static __device__ __forceinline__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct ClearType<__half> {
    static constexpr int planes = 2;
    static __device__ __forceinline__ float to(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half from(float v) { return __float2half_rn(v); }
};
template <>
struct ClearType<float> {
    static constexpr int planes = 3;
    static __device__ __forceinline__ float to(float v) { return v; }
    static __device__ __forceinline__ float from(float v) { return v; }
};
// A decay of zero leaves nothing of a state, also of an infinite one or of NaN.
__device__ __forceinline__ float decayed(float f, float v) { return f == 0.f ? 0.f : f * v; }
static inline uint32_t clear_type_bytes(uint32_t type) { return type == FESC_F32 ? 4 : 2; }

// two float32 numbers at a time
struct f2 {
    float x, y;
};
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ f2 both(uint32_t bf16x2) { return {__uint_as_float(bf16x2 << 16), __uint_as_float(bf16x2 & 0xFFFF0000u)}; }

// Eight neighbours at once where the buffer allows 16-byte accesses (`wide`), one by one up to `count` otherwise; what is not there reads as zero.
template <class T>
__device__ __forceinline__ void clear_load8(const T* p, int count, bool wide, float (&v)[8]) {
    if (wide && count >= 8) {
        if constexpr (sizeof(T) == 2) {
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (std::is_same_v<T, __half>) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
                    v[2 * i] = f.x, v[2 * i + 1] = f.y;
                } else {
                    v[2 * i] = __uint_as_float(u[i] << 16), v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
                }
            }
        } else {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < count ? ClearType<T>::to(p[i]) : 0.f;
    }
}
template <class T>
__device__ __forceinline__ void clear_store8(T* p, int count, bool wide, const float (&v)[8]) {
    if (wide && count >= 8) {
        if constexpr (sizeof(T) == 2) {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (std::is_same_v<T, __half>) {
                    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                    u[i] = *reinterpret_cast<const uint32_t*>(&h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                    u[i] = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
            *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
        } else {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < count) p[i] = ClearType<T>::from(v[i]);
    }
}
