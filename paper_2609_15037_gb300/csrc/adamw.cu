// AdamW over many tensors in one launch, with moments in fp32 or in 8 bits, and
// the norm of many gradients.
//
// Both are one pass over the data.  Per entry the step moves 28 bytes (fp32
// parameter and moments, bf16 gradient and copy) or 10 (bf16 parameter and
// gradient, 8-bit moments) and does some twenty to sixty operations, so DRAM
// bounds the first and DRAM and the integer pipe together the second; the norm
// reads its bytes and does one FMA per entry.  Short tensors are all latency:
// every tensor of a call is in the launch's parameter block, so a call costs one
// launch.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "launch.cuh"
#include "ops.h"

namespace moara {
namespace {

// ---------------------------------------------------------------------------
// 8-bit moments.  y = |x| * (1.875 / top) lies in [0, 1.875] up to rounding.
// Scaled by 2^-112 (exp_avg) or 2^-96 (exp_avg_sq) its largest exponent lands on
// the fp32 exponent field 15 or 31 and everything below field 1 is an fp32
// subnormal, so the code is bits >> 20 of an fp32 number: exponent field and 3
// mantissa bits, subnormals included, with no case distinction.  Adding 20
// random bits before the shift rounds up with the probability of the part
// cut off.  The moments themselves take one fp32 rounding per operation (no
// contraction), so that the codes follow from the formulas alone.
// ---------------------------------------------------------------------------
constexpr float kCodeTop = 1.875f;
// The nearest float to 1 / 1.875, 5.2e-8 of itself too large: a block's values grow by so much
// with every step, beside a decay of 1 - beta (1e-4 in 2000 steps without a gradient, 5.2e-8 /
// (1 - beta) where gradients keep coming).
constexpr float kCodeUnit = 1.0f / 1.875f;

// Four codes of exp_avg: sign, 4 exponent and 3 mantissa bits are the upper bits of
// an fp16 number without its top exponent bit, subnormals included.
__device__ __forceinline__ void decode_avg(uint32_t w, float scale, float* v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t x = __byte_perm(w, 0, i == 0 ? 0x1404 : 0x3424);       // each code in the upper byte of a half
        const uint32_t h = (x & 0x80008000u) | ((x >> 1) & 0x3F803F80u);
        const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&h));
        v[2 * i] = __fmul_rn(y.x, scale);
        v[2 * i + 1] = __fmul_rn(y.y, scale);
    }
}

// Four codes of exp_avg_sq, 5 exponent and 3 mantissa bits.
__device__ __forceinline__ void decode_sq(uint32_t w, float scale, float* v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t x = (e < 3 ? w << (20 - 8 * e) : w >> 4) & 0x0FF00000u;
        v[e] = __fmul_rn(__fmul_rn(__uint_as_float(x), 0x1p96f), scale);
    }
}

// The upper bytes of eight words.
__device__ __forceinline__ void upper_bytes(const uint32_t (&u)[8], uint32_t (&w)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = __byte_perm(__byte_perm(u[4 * i], u[4 * i + 1], 0x0073), __byte_perm(u[4 * i + 2], u[4 * i + 3], 0x0073), 0x5410);
}

// Codes of 8 entries in two words.  y is at most two units above 1.875, whose code has
// 20 zero bits below it, so no random number carries it beyond the largest code.
// WIDE (a block whose largest entry is above 2^14 or 2^30): 2^-112 or 2^-96 comes in a
// second product, because the joint factor would be subnormal; such a factor is
// inexact, so that the code is limited too.
template <bool WIDE>
__device__ __forceinline__ void encode_avg(const float (&x)[8], float inv, const uint32_t (&r)[8], uint32_t (&w)[2]) {
    const float f = WIDE ? inv : inv * 0x1p-112f;
    uint32_t u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = __fmul_rn(fabsf(x[e]), f), z = WIDE ? __fmul_rn(y, 0x1p-112f) : y;
        uint32_t t = __float_as_uint(z) + (r[e] & 0xFFFFu) * 16u;
        if (WIDE) t = min(t, 0x07FFFFFFu);
        u[e] = (t << 4) | (__float_as_uint(x[e]) & 0x80000000u);      // the code in the upper byte
    }
    upper_bytes(u, w);
}

template <bool WIDE>
__device__ __forceinline__ void encode_sq(const float (&x)[8], float inv, const uint32_t (&r)[8], uint32_t (&w)[2]) {
    constexpr uint32_t ONE = 1u << 20;                                // the smallest code
    const float f = WIDE ? inv : inv * 0x1p-96f;
    uint32_t u[8], low = ONE;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = __fmul_rn(x[e], f), z = WIDE ? __fmul_rn(y, 0x1p-96f) : y;
        u[e] = __float_as_uint(z) + ((r[e] >> 12) & 0xFFFF0u);
        if (WIDE) u[e] = min(u[e], 0x0FFFFFFFu);
        low = min(low, u[e]);
    }
    if (low < ONE) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (x[e] > 0.0f) u[e] = max(u[e], ONE);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] <<= 4;
    upper_bytes(u, w);
}

// 32-bit xor-shift-multiply mixing: the published finaliser of MurmurHash3 (A. Appleby, public domain)
__host__ __device__ __forceinline__ uint32_t mix32_rest(uint32_t x) {
    x *= 0x85EBCA6Bu;
    x ^= x >> 13;
    x *= 0xC2B2AE35u;
    return x ^ (x >> 16);
}

__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) { return mix32_rest(x ^ (x >> 16)); }

// four consecutive entries at i; those at or behind n read as zero
template <bool FULL> __device__ __forceinline__ void load4(const float* p, long long i, long long n, float (&v)[4]) {
    if (FULL) {
        const float4 w = __ldcs(reinterpret_cast<const float4*>(p + i));
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = i + e < n ? p[i + e] : 0.0f;
    }
}

template <bool FULL>
__device__ __forceinline__ void load4(const __nv_bfloat16* p, long long i, long long n, float (&v)[4]) {
    if (FULL) {
        const uint2 w = __ldcs(reinterpret_cast<const uint2*>(p + i));
        v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
        v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = i + e < n ? __bfloat162float(p[i + e]) : 0.0f;
    }
}

template <bool FULL> __device__ __forceinline__ uint32_t load4(const uint8_t* p, long long i, long long n) {
    if (FULL) return __ldcs(reinterpret_cast<const unsigned int*>(p + i));
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < n) w |= static_cast<uint32_t>(p[i + e]) << (8 * e);
    return w;
}

// eight consecutive entries at i as they lie in memory, and eight codes
template <class T, bool FULL> struct Raw8;

template <bool FULL> struct Raw8<float, FULL> {
    float w[8];
    __device__ __forceinline__ void load(const float* p, long long i, long long n) {
        float a[4], b[4];
        load4<FULL>(p, i, n, a);
        load4<FULL>(p, i + 4, n, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = a[e], w[4 + e] = b[e];
    }
    __device__ __forceinline__ float get(int e) const { return w[e]; }
};

template <bool FULL> struct Raw8<__nv_bfloat16, FULL> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p, long long i, long long n) {
        if (FULL) {
            const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p + i));
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        } else {
            const uint16_t* h = reinterpret_cast<const uint16_t*>(p + i);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = (i + 2 * e < n ? h[2 * e] : 0u) |
                       (i + 2 * e + 1 < n ? static_cast<uint32_t>(h[2 * e + 1]) << 16 : 0u);
        }
    }
    __device__ __forceinline__ float get(int e) const {
        return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
};

template <bool FULL> __device__ __forceinline__ uint2 load8(const uint8_t* p, long long i, long long n) {
    if (FULL) return __ldcs(reinterpret_cast<const uint2*>(p + i));
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (i + e < n) w[e >> 2] |= static_cast<uint32_t>(p[i + e]) << (8 * (e & 3));
    return make_uint2(w[0], w[1]);
}

template <bool FULL> __device__ __forceinline__ void store4(float* p, long long i, long long n, const float (&v)[4]) {
    if (FULL) {
        __stcs(reinterpret_cast<float4*>(p + i), make_float4(v[0], v[1], v[2], v[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = v[e];
    }
}

__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <bool FULL>
__device__ __forceinline__ void store4(__nv_bfloat16* p, long long i, long long n, const float (&v)[4]) {
    if (FULL) {
        __stcs(reinterpret_cast<uint2*>(p + i), make_uint2(bf16x2(v[0], v[1]), bf16x2(v[2], v[3])));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = __float2bfloat16_rn(v[e]);
    }
}

template <bool FULL> __device__ __forceinline__ void store8(float* p, long long i, long long n, const float (&v)[8]) {
    const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
    store4<FULL>(p, i, n, a);
    store4<FULL>(p, i + 4, n, b);
}

template <bool FULL>
__device__ __forceinline__ void store8(__nv_bfloat16* p, long long i, long long n, const float (&v)[8]) {
    if (FULL) {
        __stcs(reinterpret_cast<uint4*>(p + i), make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]),
                                                           bf16x2(v[6], v[7])));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) p[i + e] = __float2bfloat16_rn(v[e]);
    }
}

template <bool FULL>
__device__ __forceinline__ void store8(uint8_t* p, long long i, long long n, const uint32_t (&w)[2]) {
    if (FULL) {
        __stcs(reinterpret_cast<uint2*>(p + i), make_uint2(w[0], w[1]));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) p[i + e] = static_cast<uint8_t>(w[e >> 2] >> (8 * (e & 3)));
    }
}

__device__ __forceinline__ float sqrt_fast(float x) {     // a few ulp, subnormals kept
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The same by one instruction each where nothing below 2^-126 matters.
__device__ __forceinline__ float sqrt_flush(float x) {
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float rcp_flush(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The largest magnitude of a warp's 256 values; a NaN is the largest (over the lanes
// as bits).
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

__device__ __forceinline__ float warp_top(const float (&a)[8]) {
    float top = fabsf(a[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) top = max_nan(top, fabsf(a[e]));
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
}

__device__ __forceinline__ void new_moments(const AdamCall& b, float g, float& m, float& v) {
    m = __fadd_rn(__fmul_rn(m, b.b1), __fmul_rn(g, b.c1));
    v = __fadd_rn(__fmul_rn(v, b.b2), __fmul_rn(__fmul_rn(g, g), b.c2));
}

__device__ __forceinline__ float new_param(const AdamTensor& t, const AdamCall& b, float p, float m, float v) {
    const float den = __fmaf_rn(sqrt_fast(v), b.rbc2, b.eps);
    return __fmaf_rn(p, t.keep, -__fdividef(__fmul_rn(m, t.step), den));
}

// fp32 moments.  One warp, 256 entries from i0 on: lane l has i0 + 4l .. +3 and
// i0 + 128 + 4l .. +3, so that every access is contiguous over the warp.  2 x 131 M
// entries with fp32 parameters, bf16 gradients and copies (28 bytes each): 1.03 ms,
// 7.1 TB/s.
template <class PT, class GT, bool FULL>
__device__ __forceinline__ void adam_tile(const AdamTensor& t, const AdamCall& b, float coef, long long i0, int lane) {
    const long long n = t.n;
    const long long at[2] = {i0 + 4 * lane, i0 + 128 + 4 * lane};
    PT* const pp = static_cast<PT*>(t.p);
    const GT* const gp = static_cast<const GT*>(t.g);
    float* const mp = static_cast<float*>(t.m);
    float* const vp = static_cast<float*>(t.v);
    float p[2][4], g[2][4], m[2][4], v[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        load4<FULL>(gp, at[h], n, g[h]);
        load4<FULL>(pp, at[h], n, p[h]);
        load4<FULL>(mp, at[h], n, m[h]);
        load4<FULL>(vp, at[h], n, v[h]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            new_moments(b, __fmul_rn(g[h][e], coef), m[h][e], v[h][e]);
            p[h][e] = new_param(t, b, p[h][e], m[h][e], v[h][e]);
        }
        store4<FULL>(pp, at[h], n, p[h]);
        if (t.copy != nullptr) store4<FULL>(reinterpret_cast<__nv_bfloat16*>(t.copy), at[h], n, p[h]);
        store4<FULL>(mp, at[h], n, m[h]);
        store4<FULL>(vp, at[h], n, v[h]);
    }
}

// 8-bit moments.  One warp, one block of 256 entries: lane l has i0 + 8l .. +7, so
// that its codes are 8 and its bf16 entries 16 bytes.  What a block reads is loaded
// while the block in front of it is computed.  93.5 M entries in bf16 (10 bytes each): 181
// us, 5.2 TB/s; 68 instructions an entry take 85% of the issue slots, of which the
// hash is 7, the two encodings 13, the update 8 + 8, divisions, addresses and the two
// maxima 14.
template <class PT, class GT, bool FULL> struct Block8 {
    Raw8<PT, FULL> p;
    Raw8<GT, FULL> g;
    uint2 mc, vc;
    float ms, vs;
    __device__ __forceinline__ void load(const AdamTensor& t, long long i0, int lane) {
        const long long at = i0 + 8 * lane;
        g.load(static_cast<const GT*>(t.g), at, t.n);
        p.load(static_cast<const PT*>(t.p), at, t.n);
        mc = load8<FULL>(static_cast<const uint8_t*>(t.m), at, t.n);
        vc = load8<FULL>(static_cast<const uint8_t*>(t.v), at, t.n);
        ms = t.ms[i0 >> 8];
        vs = t.vs[i0 >> 8];
    }
};

template <class PT, class GT, bool FULL>
__device__ __forceinline__ void adam_tile8(const AdamTensor& t, const AdamCall& b, const Block8<PT, GT, FULL>& in,
                                           float coef, long long i0, int lane) {
    const long long n = t.n, at = i0 + 8 * lane;
    PT* const pp = static_cast<PT*>(t.p);
    float p[8], g[8], m[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = in.p.get(e), g[e] = in.g.get(e);
    const uint2 mc = in.mc, vc = in.vc;
    const float ms = in.ms, vs = in.vs;
    decode_avg(mc.x, ms, m);
    decode_avg(mc.y, ms, m + 4);
    decode_sq(vc.x, vs, v);
    decode_sq(vc.y, vs, v + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) new_moments(b, __fmul_rn(g[e], coef), m[e], v[e]);
    if (b.eps >= 1e-10f) {
        // a second moment below 2^-126 is nothing beside eps
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float den = __fmaf_rn(sqrt_flush(v[e]), b.rbc2, b.eps);
            p[e] = __fmaf_rn(p[e], t.keep, -__fmul_rn(__fmul_rn(m[e], t.step), rcp_flush(den)));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = new_param(t, b, p[e], m[e], v[e]);
    }
    store8<FULL>(pp, at, n, p);
    if (t.copy != nullptr) store8<FULL>(reinterpret_cast<__nv_bfloat16*>(t.copy), at, n, p);
    const float mt = warp_top(m), vt = warp_top(v);
    const bool mf = !(mt < 0x1p-100f), vf = !(vt < 0x1p-100f);
    const float mi = mf ? __fdiv_rn(kCodeTop, mt) : 0.0f, vi = vf ? __fdiv_rn(kCodeTop, vt) : 0.0f;
    const uint32_t key = mix32(t.key ^ static_cast<uint32_t>(static_cast<unsigned long long>(i0) >> 32));
    // mix32(entry ^ key): the entries differ in their lowest three bits only, which
    // the first xor-shift does not move
    uint32_t r[8], w[2];
    const uint32_t x = static_cast<uint32_t>(at) ^ key, y = x ^ (x >> 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = mix32_rest(y ^ e);
    if (mt > 0x1p14f) encode_avg<true>(m, mi, r, w);
    else encode_avg<false>(m, mi, r, w);
    store8<FULL>(static_cast<uint8_t*>(t.m), at, n, w);
    if (vt > 0x1p30f) encode_sq<true>(v, vi, r, w);
    else encode_sq<false>(v, vi, r, w);
    store8<FULL>(static_cast<uint8_t*>(t.v), at, n, w);
    if (lane == 0) {
        t.ms[i0 >> 8] = mf ? __fmul_rn(mt, kCodeUnit) : 0.0f;
        t.vs[i0 >> 8] = vf ? __fmul_rn(vt, kCodeUnit) : 0.0f;
    }
}

// A warp's blocks below `end`, `stride` entries apart; returns the first one behind.
template <class PT, class GT, bool FULL>
__device__ __forceinline__ long long adam_blocks8(const AdamTensor& t, const AdamCall& b, float coef, long long i0,
                                                  long long stride, long long end) {
    const int lane = threadIdx.x & 31;
    if (i0 >= end) return i0;
    Block8<PT, GT, FULL> in;
    in.load(t, i0, lane);
    while (true) {
        const long long next = i0 + stride;
        const bool more = next < end;
        Block8<PT, GT, FULL> ahead;
        if (more) ahead.load(t, next, lane);
        adam_tile8<PT, GT, FULL>(t, b, in, coef, i0, lane);
        i0 = next;
        if (!more) return i0;
        in = ahead;
    }
}

template <class PT, class GT, bool B8>
__device__ __forceinline__ void adam_any(const AdamTensor& t, const AdamCall& b, float coef, long long i0, long long stride) {
    if (B8) {
        if (t.kind & kAdamVector) i0 = adam_blocks8<PT, GT, true>(t, b, coef, i0, stride, t.n - MOARA_ADAMW_BLOCK + 1);
        adam_blocks8<PT, GT, false>(t, b, coef, i0, stride, t.n);
    } else {
        if ((t.kind & kAdamVector) && i0 + MOARA_ADAMW_BLOCK <= t.n) adam_tile<PT, GT, true>(t, b, coef, i0, threadIdx.x & 31);
        else adam_tile<PT, GT, false>(t, b, coef, i0, threadIdx.x & 31);
    }
}

// Largest i < count with start(i) <= c.
template <class F> __device__ __forceinline__ int find_tensor(int count, uint32_t c, F start) {
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start(mid) <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <int CAP> __global__ void __launch_bounds__(256, 4) k_adamw(const __grid_constant__ AdamBatchOf<CAP> b) {
    const uint32_t c = blockIdx.x;
    const int q = find_tensor(b.count, c, [&](int i) { return b.start[i]; });
    const AdamTensor& t = b.t[q];
    const long long i0 = static_cast<long long>(c - b.start[q]) * kAdamChunk + (threadIdx.x >> 5) * MOARA_ADAMW_BLOCK;
    const long long stride = static_cast<long long>(b.start[q + 1] - b.start[q]) * kAdamChunk;
    pdl_begin();
    if (i0 >= t.n) return;
    const float coef = b.scale != nullptr ? *b.scale : 1.0f;
    switch (t.kind & 7u) {
        case 0: adam_any<float, float, false>(t, b, coef, i0, stride); break;
        case 1: adam_any<__nv_bfloat16, float, false>(t, b, coef, i0, stride); break;
        case 2: adam_any<float, __nv_bfloat16, false>(t, b, coef, i0, stride); break;
        case 3: adam_any<__nv_bfloat16, __nv_bfloat16, false>(t, b, coef, i0, stride); break;
        case 4: adam_any<float, float, true>(t, b, coef, i0, stride); break;
        case 5: adam_any<__nv_bfloat16, float, true>(t, b, coef, i0, stride); break;
        case 6: adam_any<float, __nv_bfloat16, true>(t, b, coef, i0, stride); break;
        default: adam_any<__nv_bfloat16, __nv_bfloat16, true>(t, b, coef, i0, stride); break;
    }
}

// ---------------------------------------------------------------------------
// Moments as fp32, DRAM-bound: 93.5 M entries of both, from 8 bits, 137 us (6.8 TB/s).
// ---------------------------------------------------------------------------
template <bool AVG>
__device__ __forceinline__ void moment_tile(const void* x, const float* scale, float* out, int block8, long long i0,
                                            long long n, int lane) {
    if (out == nullptr) return;
    const bool full = i0 + MOARA_ADAMW_BLOCK <= n && (reinterpret_cast<uintptr_t>(out) & 15) == 0 &&
                      (reinterpret_cast<uintptr_t>(x) & 15) == 0;
    const long long at[2] = {i0 + 4 * lane, i0 + 128 + 4 * lane};
    float v[2][4];
    if (block8) {
        const uint8_t* c = static_cast<const uint8_t*>(x);
        const float s = scale[i0 >> 8];
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = full ? load4<true>(c, at[h], n) : load4<false>(c, at[h], n);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (AVG) decode_avg(w[h], s, v[h]);
            else decode_sq(w[h], s, v[h]);
        }
    } else {
        const float* c = static_cast<const float*>(x);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (full) load4<true>(c, at[h], n, v[h]);
            else load4<false>(c, at[h], n, v[h]);
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (full) store4<true>(out, at[h], n, v[h]);
        else store4<false>(out, at[h], n, v[h]);
    }
}

__global__ void __launch_bounds__(256) k_moments(const __grid_constant__ MomentBatch b) {
    const uint32_t c = blockIdx.x;
    const int q = find_tensor(b.count, c, [&](int i) { return b.start[i]; });
    const MomentTensor& t = b.t[q];
    const int lane = threadIdx.x & 31;
    const long long i0 = static_cast<long long>(c - b.start[q]) * kAdamChunk + (threadIdx.x >> 5) * MOARA_ADAMW_BLOCK;
    pdl_begin();
    if (i0 >= t.n) return;
    moment_tile<true>(t.m, t.ms, t.om, t.block8, i0, t.n, lane);
    moment_tile<false>(t.v, t.vs, t.ov, t.block8, i0, t.n, lane);
}

// ---------------------------------------------------------------------------
// Gradient norm.  A thread sums at most 32 squares of a chunk in fp32 and adds
// the chunk sums in fp64; CTA sums go to the workspace, and the CTA that draws
// the last ticket adds them in order.  Which CTA that is does not change the
// result: chunks belong to CTAs by index.  DRAM-bound: 374 M bf16 entries 107 us (7.0
// TB/s), fp32 207 us (7.2 TB/s); 65 gradients of 4096 entries 4.3 us, the chain of
// launch, sums, ticket and the last CTA's sum.
// ---------------------------------------------------------------------------
// The sum over 256 threads, in thread 0.
__device__ __forceinline__ double cta_sum(double v, double* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        v = red[threadIdx.x & 7];
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
}

// Adds one at a counter; what this thread wrote before is visible to whoever reads the
// counter this way afterwards.
__device__ __forceinline__ unsigned int draw_ticket(unsigned int* ticket) {
    unsigned int order;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(order) : "l"(ticket) : "memory");
    return order;
}

template <class T>
__device__ __forceinline__ float chunk_squares(const T* g, long long e0, long long n, bool vector) {
    float s = 0.0f;
    if (vector && e0 + kGradChunk <= n) {
        constexpr int V = kGradChunk / 256 / 4;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float v[4];
            load4<true>(g, e0 + 4 * (threadIdx.x + 256 * k), n, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = fmaf(v[e], v[e], s);
        }
    } else {
        const long long e1 = min(e0 + static_cast<long long>(kGradChunk), n);
        long long i = e0;
        if (vector) {
#pragma unroll 4
            for (; i + 1024 <= e1; i += 1024) {
                float v[4];
                load4<true>(g, i + 4 * threadIdx.x, n, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) s = fmaf(v[e], v[e], s);
            }
        }
        for (i += threadIdx.x; i < e1; i += 256) {
            const float x = static_cast<float>(g[i]);
            s = fmaf(x, x, s);
        }
    }
    return s;
}

template <int CAP> __global__ void __launch_bounds__(256) k_grad_norm(const __grid_constant__ NormBatchOf<CAP> b) {
    __shared__ double red[8];
    __shared__ bool finish;
    double acc = 0.0;
    pdl_begin();
    for (uint32_t c = blockIdx.x; c < b.chunks; c += gridDim.x) {
        const int q = find_tensor(b.count, c, [&](int i) { return b.t[i].start; });
        const NormTensor& t = b.t[q];
        const long long e0 = static_cast<long long>(c - t.start) * kGradChunk;
        const bool vec = (t.kind & kAdamVector) != 0;
        acc += (t.kind & kAdamGradBf16) ? chunk_squares(static_cast<const __nv_bfloat16*>(t.g), e0, t.n, vec)
                                        : chunk_squares(static_cast<const float*>(t.g), e0, t.n, vec);
    }
    const double sum = cta_sum(acc, red);
    if (threadIdx.x == 0) {
        b.partials[b.first + blockIdx.x] = sum;
        finish = b.last && draw_ticket(b.ticket) == gridDim.x - 1;
    }
    __syncthreads();
    if (!finish) return;
    double part = 0.0;
    for (int i = threadIdx.x; i < b.first + static_cast<int>(gridDim.x); i += 256) part += __ldcg(b.partials + i);
    const double total = cta_sum(part, red);
    if (threadIdx.x == 0) {
        *b.ticket = 0;
        // an fp64 root and quotient are a microsecond of dependent operations here: fp32 ones,
        // but for a sum that fp32 does not hold
        const double all = total + (b.extra != nullptr ? static_cast<double>(*b.extra) : 0.0);
        const float norm = all < 1e38 ? __fsqrt_rn(static_cast<float>(all)) : static_cast<float>(sqrt(all));
        const float coef = __fdiv_rn(b.max_norm, norm + 1e-6f);
        b.out[0] = static_cast<float>(total);
        b.out[1] = norm;
        b.out[2] = b.max_norm > 0.0f && !(coef >= 1.0f) ? coef : 1.0f;
    }
}

}  // namespace

uint32_t adamw_key(uint64_t seed, uint32_t id, int64_t t) {
    uint32_t k = mix32(mix32(static_cast<uint32_t>(seed)) ^ static_cast<uint32_t>(seed >> 32));
    k = mix32(k ^ id);
    return mix32(k ^ static_cast<uint32_t>(t));
}

cudaError_t launch_adamw(const AdamBatch& b, cudaStream_t s, int64_t* launches) {
    ++*launches;
    if (b.count <= kAdamFew) {
        AdamBatchOf<kAdamFew> f;
        static_cast<AdamCall&>(f) = b;
        for (int i = 0; i < b.count; ++i) f.t[i] = b.t[i];
        for (int i = 0; i <= b.count; ++i) f.start[i] = b.start[i];
        return launch(k_adamw<kAdamFew>, dim3(b.start[b.count]), dim3(256), 0, s, 1, f);
    }
    return launch(k_adamw<kAdamTensors>, dim3(b.start[b.count]), dim3(256), 0, s, 1, b);
}

cudaError_t launch_moments(const MomentBatch& b, cudaStream_t s, int64_t* launches) {
    ++*launches;
    return launch(k_moments, dim3(b.start[b.count]), dim3(256), 0, s, 1, b);
}

cudaError_t launch_grad_norm(const NormBatch& b, int ctas, cudaStream_t s, int64_t* launches) {
    ++*launches;
    if (b.count <= kNormFew) {
        NormBatchOf<kNormFew> f;
        static_cast<NormCall&>(f) = b;
        for (int i = 0; i < b.count; ++i) f.t[i] = b.t[i];
        return launch(k_grad_norm<kNormFew>, dim3(ctas), dim3(256), 0, s, 1, f);
    }
    return launch(k_grad_norm<kNormTensors>, dim3(ctas), dim3(256), 0, s, 1, b);
}

}  // namespace moara
