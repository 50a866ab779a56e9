// Vectors of bf16 and fp32 values as the kernels load, convert and store them.  NT: non-temporally, of data that the
// caches do not hold to the end of a call.
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

template <bool NT, typename V>
__device__ __forceinline__ V load_vec(const void* p) {
    return NT ? __builtin_nontemporal_load((const V*)p) : *(const V*)p;
}

template <bool NT, typename V>
__device__ __forceinline__ void store_vec(void* p, V v) {
    if (NT)
        __builtin_nontemporal_store(v, (V*)p);
    else
        *(V*)p = v;
}

// Four values in a row: 8 bytes of bf16 or 16 of fp32.
template <typename T, bool NT>
struct Vec4;

template <bool NT>
struct Vec4<bf16_t, NT> {
    u32x2 r;
    __device__ __forceinline__ void load(const bf16_t* p) { r = load_vec<NT, u32x2>(p); }
    __device__ __forceinline__ void get(float* v) const {
        v[0] = bf16_low(r.x), v[1] = bf16_high(r.x), v[2] = bf16_low(r.y), v[3] = bf16_high(r.y);
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
        store_vec<NT>(p, (u32x2){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])});
    }
};

template <bool NT>
struct Vec4<float, NT> {
    f32x4 r;
    __device__ __forceinline__ void load(const float* p) { r = load_vec<NT, f32x4>(p); }
    __device__ __forceinline__ void get(float* v) const { v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w; }
    static __device__ __forceinline__ void store(float* p, const float* v) { store_vec<NT>(p, (f32x4){v[0], v[1], v[2], v[3]}); }
};

// Eight bf16 values in a row.
template <bool NT>
struct Vec8 {
    u32x4 r;
    __device__ __forceinline__ void load(const bf16_t* p) { r = load_vec<NT, u32x4>(p); }
    __device__ __forceinline__ void get(float* v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = bf16_low(r[i]), v[2 * i + 1] = bf16_high(r[i]);
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
        store_vec<NT>(p, (u32x4){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
    }
};

}  // namespace orbit
