// MXFP4 operands: quantisation by rows and by columns from one read of the
// matrix, and the values of an operand.  DRAM-bound: per entry 4 or 2 bytes in
// and 17/32 of a byte out per orientation.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ops.h"

namespace moara {
namespace {

struct QuantParams {
    const void* X;
    long long ld;
    int rows, cols;
    int kb, kbt;           // 32-entry blocks of a row, of a column
    int tiles_c, tiles_r;  // 128-column and 128-row tiles
    int vec;               // rows of X may be read 16 bytes at a time
    uint8_t* q;
    uint32_t* sf;          // words of four scales
    uint8_t* qt;
    uint32_t* sft;
};

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

// Eight entries of a row as they lie in memory, their fp32 values, and the largest
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

template <class T> struct Row8;

template <> struct Row8<float> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const float* p) {
        const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
    __device__ __forceinline__ void load_some(const float* p, int count) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = e < count ? __float_as_uint(p[e]) : 0u;
    }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(w[e]); }
    // bits of the largest magnitude of the row's eight entries
    __device__ __forceinline__ uint32_t top() const {
        float t = fabsf(get(0));
#pragma unroll
        for (int e = 1; e < 8; ++e) t = max_nan(t, fabsf(get(e)));
        return __float_as_uint(t);
    }
    // and of each column of eight rows
    static __device__ __forceinline__ void tops(const Row8 (&x)[8], uint32_t (&t)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float y = fabsf(x[0].get(e));
#pragma unroll
            for (int i = 1; i < 8; ++i) y = max_nan(y, fabsf(x[i].get(e)));
            t[e] = __float_as_uint(y);
        }
    }
};

template <> struct Row8<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    }
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
    static __device__ __forceinline__ void tops(const Row8 (&x)[8], uint32_t (&t)[8]) {
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

// One CTA takes a 128 x 128 tile, which is one 512-byte scale tile of either
// orientation, and each warp 32 rows x 64 columns of it: a lane holds 8 rows x 8
// columns in registers, so that a row's block of 32 columns is four lanes, a
// column's block of 32 rows the four lanes 8 apart, and eight codes of either are one
// word of one lane.  The matrix passes through no shared memory (32 x 1 blocks of a
// 64 KB tile there took 67 us where this takes 42 on 11008 x 4096 fp32); only the
// columns' codes do, to leave in whole 64-byte lines.
template <class T, bool ROWS, bool COLS>
__global__ void __launch_bounds__(256, sizeof(T) == 2 && !(ROWS && COLS) ? 3 : 2) k_fp4_quantize(const QuantParams p) {
    __shared__ __align__(16) uint8_t sfr[512];
    __shared__ __align__(16) uint8_t sfc[512];
    __shared__ __align__(16) uint32_t qc[COLS ? 128 * 17 : 1];       // a column's 16 words of codes, and one of padding
    const int tr = blockIdx.x / p.tiles_c, tc = blockIdx.x % p.tiles_c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wr = warp >> 1, sub = (warp & 1) * 8 + (lane & 7);     // 32-row group, 8-column group of the tile
    const int lr = wr * 32 + (lane >> 3) * 8, lc = sub * 8;          // the lane's 8 x 8 entries inside the tile
    const int row0 = tr * 128 + lr, col0 = tc * 128 + lc;
    const T* X = static_cast<const T*>(p.X) + row0 * p.ld + col0;
    Row8<T> x[8];
    if (p.vec && col0 + 8 <= p.cols && row0 + 8 <= p.rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i].load(X + i * p.ld);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i].load_some(X + i * p.ld, row0 + i < p.rows ? p.cols - col0 : 0);
    }
    if (ROWS) {
        const int block = (tc * 128 + lc) >> 5;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = x[i].get(e);
            uint32_t top = x[i].top();
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const bool real = row0 + i < p.rows && block < p.kb;
            const uint32_t byte = real ? scale_byte(top) : 127u;
            if ((lane & 3) == 0) sfr[((lr + i) & 31) * 16 + wr * 4 + (sub >> 2)] = static_cast<uint8_t>(byte);
            if (real)
                *reinterpret_cast<uint32_t*>(p.q + (static_cast<long long>(row0 + i) * p.kb + block) * 16 + (lane & 3) * 4) =
                    codes8(v, inv_scale(byte));
        }
    }
    if (COLS) {
        const bool rows_real = tr * 4 + wr < p.kbt;
        uint32_t tops[8];
        Row8<T>::tops(x, tops);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[i].get(e);
            uint32_t top = tops[e];
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 16));
            const uint32_t byte = rows_real && col0 + e < p.cols ? scale_byte(top) : 127u;
            if (lane < 8) sfc[((lc + e) & 31) * 16 + ((lc + e) >> 5) * 4 + wr] = static_cast<uint8_t>(byte);
            qc[(lc + e) * 17 + wr * 4 + (lane >> 3)] = codes8(v, inv_scale(byte));
        }
    }
    __syncthreads();
    if (ROWS && threadIdx.x < 128)
        p.sf[(static_cast<long long>(tr) * p.tiles_c + tc) * 128 + threadIdx.x] =
            reinterpret_cast<const uint32_t*>(sfr)[threadIdx.x];
    if (COLS) {
        if (threadIdx.x >= 128)
            p.sft[(static_cast<long long>(tc) * p.tiles_r + tr) * 128 + threadIdx.x - 128] =
                reinterpret_cast<const uint32_t*>(sfc)[threadIdx.x - 128];
        // four lanes a column, 16 bytes (one block) each
        const int cols = min(128, p.cols - tc * 128), block = tr * 4 + (threadIdx.x & 3);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int c = u * 64 + (threadIdx.x >> 2);
            const uint32_t* w = qc + c * 17 + (threadIdx.x & 3) * 4;
            if (c < cols && block < p.kbt)
                *reinterpret_cast<uint4*>(p.qt + (static_cast<long long>(tc * 128 + c) * p.kbt + block) * 16) =
                    make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// ---------------------------------------------------------------------------
// Values of an operand: a thread takes 8 columns.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float scale_value(uint32_t byte) {
    if (byte == 255u) return __uint_as_float(0x7FC00000u);
    return byte == 0u ? 0x1p-127f : __uint_as_float(byte << 23);
}

// Eight codes as fp32, by the hardware's conversion of two of them to fp16 (exact).
__device__ __forceinline__ void values8(uint32_t w, float f, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = a.x * f;
        v[2 * i + 1] = a.y * f;
    }
}

// A CTA takes 32 rows x 512 columns: a thread 8 columns of eight rows, whose loads
// are issued together.
constexpr int VALUE_ROWS = 8;

template <class T>
__global__ void __launch_bounds__(256) k_fp4_values(const uint8_t* q, const uint8_t* sf, int rows, int cols, int kb,
                                                    int tiles_c, T* out, long long ldo, int vec, int parts) {
    const int part = blockIdx.x % parts, group = blockIdx.x / parts;
    const int s = part * 64 + (threadIdx.x & 63), block = s >> 2, col = 8 * s;
    const int row0 = group * (4 * VALUE_ROWS) + (threadIdx.x >> 6);
    if (block >= kb) return;
    uint32_t w[VALUE_ROWS], sb[VALUE_ROWS];
#pragma unroll
    for (int i = 0; i < VALUE_ROWS; ++i) {
        const int row = row0 + 4 * i;
        w[i] = sb[i] = 0;
        if (row >= rows) continue;
        w[i] = *reinterpret_cast<const uint32_t*>(q + (static_cast<long long>(row) * kb + block) * 16 + (s & 3) * 4);
        sb[i] = sf[(static_cast<long long>(row >> 7) * tiles_c + (block >> 2)) * 512 + (row & 31) * 16 +
                   ((row & 127) >> 5) * 4 + (block & 3)];
    }
#pragma unroll
    for (int i = 0; i < VALUE_ROWS; ++i) {
        const int row = row0 + 4 * i;
        if (row >= rows) return;
        float v[8];
        values8(w[i], scale_value(sb[i]), v);
        T* o = out + row * ldo + col;
        if (vec && col + 8 <= cols) {
            if (sizeof(T) == 4) {
                __stcs(reinterpret_cast<float4*>(o), make_float4(v[0], v[1], v[2], v[3]));
                __stcs(reinterpret_cast<float4*>(o) + 1, make_float4(v[4], v[5], v[6], v[7]));
            } else {
                uint32_t h[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                    h[k] = *reinterpret_cast<const uint32_t*>(&b);
                }
                __stcs(reinterpret_cast<uint4*>(o), make_uint4(h[0], h[1], h[2], h[3]));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < cols) o[e] = static_cast<T>(v[e]);
        }
    }
}

template <class T>
cudaError_t quantize_as(const QuantParams& p, cudaStream_t s) {
    const unsigned int grid = static_cast<unsigned int>(p.tiles_r) * p.tiles_c;
    if (p.qt == nullptr) k_fp4_quantize<T, true, false><<<grid, 256, 0, s>>>(p);
    else if (p.q == nullptr) k_fp4_quantize<T, false, true><<<grid, 256, 0, s>>>(p);
    else k_fp4_quantize<T, true, true><<<grid, 256, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_fp4_quantize(const void* X, int dtype, int rows, int cols, int64_t ld, void* q, void* sf, void* qt,
                                void* sft, cudaStream_t s, int64_t* launches) {
    QuantParams p{};
    p.X = X;
    p.ld = ld;
    p.rows = rows;
    p.cols = cols;
    p.kb = fp4_blocks(cols);
    p.kbt = fp4_blocks(rows);
    p.tiles_c = fp4_tiles(cols);
    p.tiles_r = fp4_tiles(rows);
    p.vec = (reinterpret_cast<uintptr_t>(X) & 15) == 0 && ld % (dtype == MOARA_DTYPE_BF16 ? 8 : 4) == 0;
    p.q = static_cast<uint8_t*>(q);
    p.sf = static_cast<uint32_t*>(sf);
    p.qt = static_cast<uint8_t*>(qt);
    p.sft = static_cast<uint32_t*>(sft);
    ++*launches;
    return dtype == MOARA_DTYPE_BF16 ? quantize_as<__nv_bfloat16>(p, s) : quantize_as<float>(p, s);
}

cudaError_t launch_fp4_dequantize(const void* q, const void* sf, int rows, int cols, void* out, int dtype, int64_t ldo,
                                  cudaStream_t s, int64_t* launches) {
    const int kb = fp4_blocks(cols);
    const int parts = (4 * kb - 1) / 64 + 1;
    const unsigned int grid = static_cast<unsigned int>(parts) * ((rows - 1) / (4 * VALUE_ROWS) + 1);
    const bool bf = dtype == MOARA_DTYPE_BF16;
    const int vec = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ldo % (bf ? 8 : 4) == 0;
    const uint8_t* qq = static_cast<const uint8_t*>(q);
    const uint8_t* ss = static_cast<const uint8_t*>(sf);
    ++*launches;
    if (bf)
        k_fp4_values<__nv_bfloat16><<<grid, 256, 0, s>>>(qq, ss, rows, cols, kb, fp4_tiles(cols),
                                                         static_cast<__nv_bfloat16*>(out), ldo, vec, parts);
    else
        k_fp4_values<float><<<grid, 256, 0, s>>>(qq, ss, rows, cols, kb, fp4_tiles(cols), static_cast<float*>(out), ldo,
                                                 vec, parts);
    return cudaGetLastError();
}

}  // namespace moara
