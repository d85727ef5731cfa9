// Rounding to MXFP4 in registers: a block's scale, codes, and entries of a row in
// fp32 or bf16.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

namespace moara {

// Scale byte of a block from its largest magnitude's bits: the exponent field of
// top / 1.5 rounded up to a power of two, two binades lower (6 = 1.5 * 2^2).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7F800000u) return 255u;
    const int e = static_cast<int>((top + 0x3FFFFFu) >> 23) - 2;
    return static_cast<uint32_t>(max(e, 0));
}

// 2^(127 - byte), the factor into the block's grid (0 for a NaN scale)
__device__ __forceinline__ float inv_scale(uint32_t byte) {
    return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23);
}

// Eight codes, entry 0 in the low half of byte 0; products with a power of two are
// exact, so the conversion is the only rounding (to nearest, ties to even).
__device__ __forceinline__ uint32_t codes8(const float (&v)[8], float f) {
    uint32_t w;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(w)
        : "f"(v[0] * f), "f"(v[1] * f), "f"(v[2] * f), "f"(v[3] * f), "f"(v[4] * f), "f"(v[5] * f), "f"(v[6] * f),
          "f"(v[7] * f));
    return w;
}

// Four codes in the lower half.
__device__ __forceinline__ uint32_t codes4(const float (&v)[4], float f) {
    uint32_t w;
    asm("{\n\t.reg .b8 b0, b1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "mov.b32 %0, {b0, b1, b0, b1};\n\t}"
        : "=r"(w)
        : "f"(v[0] * f), "f"(v[1] * f), "f"(v[2] * f), "f"(v[3] * f));
    return w;
}

// Entries of a row as they lie in memory, their fp32 values, and the largest
// magnitude of several, with a NaN above all (bf16: of two columns at a time).
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}

// The 16 bytes at p, on any boundary of an entry, from the three lines of 8 bytes that
// hold them.  offset: p's place in the first, the same in every thread.  Both orientations
// of 4199 x 12909 take 36.2 us in bf16 and 52.8 in fp32 (12912 columns, whose rows are
// aligned: 31.6 and 44.3); from two lines of 16 bytes 36.9 and 59.5, from words 38.5 and
// 61.1; of 4978 x 5370 in bf16 18.2, entry by entry 25.0.
template <int SIZE> __device__ __forceinline__ void load_lines(const void* p, int offset, uint32_t (&w)[4]) {
    const uint2* line = reinterpret_cast<const uint2*>(reinterpret_cast<uintptr_t>(p) - offset);
    const uint2 a = line[0], b = line[1], c = line[2];
    uint32_t t[6] = {a.x, a.y, b.x, b.y, c.x, c.y};
    const bool four = (offset & 4) != 0;
#pragma unroll
    for (int e = 0; e < 5; ++e) t[e] = four ? t[e + 1] : t[e];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = SIZE == 2 ? __funnelshift_r(t[e], t[e + 1], (offset & 2) * 8) : t[e];
}

template <class T, int N> struct Row;

template <int N> struct Row<float, N> {
    uint32_t w[N];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const uint4 a = *reinterpret_cast<const uint4*>(p + e);
            w[e] = a.x; w[e + 1] = a.y; w[e + 2] = a.z; w[e + 3] = a.w;
        }
    }
    __device__ __forceinline__ void load_any(const float* p, int offset) { load_lines<4>(p, offset, w); }
    __device__ __forceinline__ void load_some(const float* p, int count) {
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = e < count ? __float_as_uint(p[e]) : 0u;
    }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(w[e]); }
    // bits of the largest magnitude of the row's entries
    __device__ __forceinline__ uint32_t top() const {
        float t = fabsf(get(0));
#pragma unroll
        for (int e = 1; e < N; ++e) t = max_nan(t, fabsf(get(e)));
        return __float_as_uint(t);
    }
    // and of each column of eight rows
    static __device__ __forceinline__ void tops(const Row (&x)[8], uint32_t (&t)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float y = fabsf(x[0].get(e));
#pragma unroll
            for (int i = 1; i < 8; ++i) y = max_nan(y, fabsf(x[i].get(e)));
            t[e] = __float_as_uint(y);
        }
    }
};

template <> struct Row<__nv_bfloat16, 8> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    }
    __device__ __forceinline__ void load_any(const __nv_bfloat16* p, int offset) { load_lines<2>(p, offset, w); }
    __device__ __forceinline__ void load_some(const __nv_bfloat16* p, int count) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = (2 * e < count ? h[2 * e] : 0u) | (2 * e + 1 < count ? static_cast<uint32_t>(h[2 * e + 1]) << 16 : 0u);
    }
    __device__ __forceinline__ float get(int e) const {
        return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
    static __device__ __forceinline__ uint32_t size(uint32_t x) { return x & 0x7FFF7FFFu; }
    __device__ __forceinline__ uint32_t top() const {
        const uint32_t t = max_nan2(max_nan2(size(w[0]), size(w[1])), max_nan2(size(w[2]), size(w[3])));
        return max(t << 16, t & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void tops(const Row (&x)[8], uint32_t (&t)[8]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t y = size(x[0].w[e]);
#pragma unroll
            for (int i = 1; i < 8; ++i) y = max_nan2(y, size(x[i].w[e]));
            t[2 * e] = y << 16;
            t[2 * e + 1] = y & 0xFFFF0000u;
        }
    }
};

}  // namespace moara
