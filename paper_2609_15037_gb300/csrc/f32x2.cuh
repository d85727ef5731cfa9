// Pairs of fp32 numbers, two operations in one instruction.
#pragma once

#include <cstdint>

namespace moara {

__device__ __forceinline__ uint64_t f32x2(float a, float b) {
    uint64_t y;
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ uint64_t both(float a) { return f32x2(a, a); }
__device__ __forceinline__ void split(uint64_t x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t y;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
    return y;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t y;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
    return y;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t y;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
    return y;
}
// a - b
__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) { return fma2(b, both(-1.0f), a); }

// Two bf16 numbers of a word.
__device__ __forceinline__ uint64_t widen2(uint32_t w) { return f32x2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }

}  // namespace moara
