// Vectors of bf16 and fp32 values as the kernels load, convert and store them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace orbit {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

struct bf16_t {  // a bf16 value in memory, as a type of its own for templates
    uint16_t bits;
};

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// (a, b) rounded to nearest even: a in the low half
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2_t));
}

// Four values in a row: 8 bytes of bf16 or 16 of fp32.
template <typename T>
struct Vec4;

template <>
struct Vec4<bf16_t> {
    u32x2 r;
    __device__ __forceinline__ void load(const bf16_t* p) { r = *(const u32x2*)p; }
    __device__ __forceinline__ void get(float* v) const {
        v[0] = bf16_low(r.x), v[1] = bf16_high(r.x), v[2] = bf16_low(r.y), v[3] = bf16_high(r.y);
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
        *(u32x2*)p = (u32x2){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
};

template <>
struct Vec4<float> {
    f32x4 r;
    __device__ __forceinline__ void load(const float* p) { r = *(const f32x4*)p; }
    __device__ __forceinline__ void get(float* v) const { v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w; }
    static __device__ __forceinline__ void store(float* p, const float* v) { *(f32x4*)p = (f32x4){v[0], v[1], v[2], v[3]}; }
};

// Eight values in a row.
template <typename T>
struct Vec8;

template <>
struct Vec8<bf16_t> {
    u32x4 r;
    __device__ __forceinline__ void load(const bf16_t* p) { r = *(const u32x4*)p; }
    __device__ __forceinline__ void get(float* v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = bf16_low(r[i]), v[2 * i + 1] = bf16_high(r[i]);
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
        *(u32x4*)p = (u32x4){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
};

template <>
struct Vec8<float> {
    Vec4<float> a, b;
    __device__ __forceinline__ void load(const float* p) { a.load(p), b.load(p + 4); }
    __device__ __forceinline__ void get(float* v) const { a.get(v), b.get(v + 4); }
    static __device__ __forceinline__ void store(float* p, const float* v) {
        Vec4<float>::store(p, v);
        Vec4<float>::store(p + 4, v + 4);
    }
};

}  // namespace orbit
