// The cache that holds 4.5 bits a value: its pages and what a code stands for.
#pragma once

#include "pcg_cache.cuh"

namespace pcg {

// Byte offsets inside a page of 16 tokens of one head.
__host__ __device__ constexpr int page_bytes(int d) { return 18 * d; }
__host__ __device__ constexpr int key_scales_at(int d) { return 8 * d; }
__host__ __device__ constexpr int value_codes_at(int d) { return 9 * d; }
__host__ __device__ constexpr int value_scales_at(int d) { return 17 * d; }

pcg_status check_fourbit(const char *who, const pcg_fourbit_cache *c);

#ifdef __CUDACC__

// Four bytes of codes as eight float16 values, two a register: exact.
__device__ __forceinline__ void widen_codes(uint32_t w, uint32_t (&r)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
        : "r"(w));
}
// Four scales as float16 values, two a register: exact.
__device__ __forceinline__ void widen_scales(uint32_t w, uint32_t (&r)[2]) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(r[0]), "=r"(r[1])
        : "r"(w));
}
__device__ __forceinline__ float widen_scale(uint32_t byte) {
    uint32_t r[2];
    widen_scales(byte, r);
    return __low2float(*reinterpret_cast<__half2 *>(&r[0]));
}
// Two float16 products.
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    const __half2 r = __hmul2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ float2 both_halves(uint32_t h2) { return __half22float2(*reinterpret_cast<__half2 *>(&h2)); }

#endif  // __CUDACC__

}  // namespace pcg
