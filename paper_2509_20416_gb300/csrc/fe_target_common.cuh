// Device helpers shared by the target-side kernels: cache row addresses, e4m3 conversion.
#pragma once

#include "fe_common.cuh"
#include "fe_target_kernels.h"

namespace fe {

// The row index of (sequence b, head 0, slot); the head's row is + h * head_step(). False for
// a slot outside [0, max_seq) or a page id outside the pool.
__device__ __forceinline__ bool cache_row(const CacheView& c, int b, int64_t slot, int64_t& row, int* status) {
    if (slot < 0 || slot >= c.max_seq) {
        atomicOr(status, ST_CAPACITY);
        return false;
    }
    const int s = (int)slot;
    if (c.page_size == 0) {
        row = (int64_t)b * c.Hkv * c.max_seq + s;
        return true;
    }
    const int lp = s / c.page_size;
    const int pg = c.table[(int64_t)b * c.max_pages + lp];
    if (pg < 0 || pg >= c.n_pages) {
        atomicOr(status, ST_DEVICE);
        return false;
    }
    row = (int64_t)pg * c.Hkv * c.page_size + (s - lp * c.page_size);
    return true;
}

__device__ __forceinline__ int64_t head_step(const CacheView& c) {
    return c.page_size == 0 ? c.max_seq : c.page_size;
}

// two e4m3 numbers (low byte first) to floats; exact, NaN stays NaN
__device__ __forceinline__ float2 e4m3x2_to_f32(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    float lo, hi;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
        : "=f"(lo), "=f"(hi)
        : "r"(h));
    return make_float2(lo, hi);
}

// round to nearest even; magnitudes up to 448 (larger finite ones saturate), NaN to e4m3's NaN
__device__ __forceinline__ uint32_t f32x2_to_e4m3(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// two floats to packed bfloat16 (round to nearest even, NaN and infinities kept)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ bool finite_f32(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// 16 bytes of rows, from and to floats
template <typename T> __device__ __forceinline__ uint4 pack16(const float* f);
template <> __device__ __forceinline__ uint4 pack16<float>(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ uint4 pack16<bf16_t>(const float* f) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_one(bf16_t* p, float v) { p->bits = (uint16_t)pack_bf16(v, 0.f); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// packed pairs of floats: d = a * b + c and a + b, elementwise
__device__ __forceinline__ uint64_t pair_f32(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ uint64_t pair_f32(float x) { return pair_f32(__float_as_uint(x), __float_as_uint(x)); }
__device__ __forceinline__ float low_f32(uint64_t a) { return __uint_as_float((uint32_t)a); }
__device__ __forceinline__ float high_f32(uint64_t a) { return __uint_as_float((uint32_t)(a >> 32)); }
__device__ __forceinline__ uint64_t fma_x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul_x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t add_x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

}  // namespace fe
