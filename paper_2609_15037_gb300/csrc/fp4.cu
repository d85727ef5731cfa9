// MXFP4 operands: quantisation by rows and by columns from one read of the
// matrix, and the values of an operand.  DRAM-bound: per entry 4 or 2 bytes in
// and 17/32 of a byte out per orientation.
#include <cuda_bf16.h>

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

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// One CTA takes a 128 x 128 tile, which is one 512-byte scale tile of either
// orientation.  By rows, four lanes hold a 32-column block in registers as it is
// loaded; by columns, the tile goes through shared memory and a thread takes 32
// rows of one column.
template <class T, bool ROWS, bool COLS> __global__ void __launch_bounds__(256) k_fp4_quantize(const QuantParams p) {
    __shared__ __align__(16) uint8_t sfr[512];
    __shared__ __align__(16) uint8_t sfc[512];
    extern __shared__ __align__(16) float tile[];        // 128 x 128 (COLS)
    const int tr = blockIdx.x / p.tiles_c, tc = blockIdx.x % p.tiles_c;
    const int r0 = tr * 128, c0 = tc * 128;
    const int sub = threadIdx.x & 15;                     // 8 columns
    const int rw = threadIdx.x >> 4;                      // row within a pass of 16
    const int col = c0 + 8 * sub;
    const T* X = static_cast<const T*>(p.X);
    const bool wide = p.vec && col + 8 <= p.cols;
#pragma unroll 4
    for (int pass = 0; pass < 8; ++pass) {
        const int lr = pass * 16 + rw, row = r0 + lr;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
        if (row < p.rows) {
            const T* x = X + row * p.ld + col;
            if (wide) {
                load8(x, v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < p.cols) v[e] = static_cast<float>(x[e]);
            }
        }
        if (ROWS) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int block = (c0 >> 5) + (sub >> 2);
            const bool real = row < p.rows && block < p.kb;
            const uint32_t byte = real ? scale_byte(top) : 127u;
            if ((sub & 3) == 0) sfr[(lr & 31) * 16 + (lr >> 5) * 4 + (sub >> 2)] = static_cast<uint8_t>(byte);
            if (real)
                *reinterpret_cast<uint32_t*>(p.q + (static_cast<long long>(row) * p.kb + block) * 16 + (sub & 3) * 4) =
                    codes8(v, inv_scale(byte));
        }
        if (COLS) {
            float4* d = reinterpret_cast<float4*>(tile + lr * 128 + 8 * sub);
            d[0] = make_float4(v[0], v[1], v[2], v[3]);
            d[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
    __syncthreads();
    if (ROWS && threadIdx.x < 128)
        p.sf[(static_cast<long long>(tr) * p.tiles_c + tc) * 128 + threadIdx.x] =
            reinterpret_cast<const uint32_t*>(sfr)[threadIdx.x];
    if (COLS) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int lc = threadIdx.x & 127, blk = (threadIdx.x >> 7) + 2 * u;
            const int cc = c0 + lc, block = (r0 >> 5) + blk;
            float v[32];
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                v[e] = tile[(blk * 32 + e) * 128 + lc];
                top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
            }
            const bool real = cc < p.cols && block < p.kbt;
            const uint32_t byte = real ? scale_byte(top) : 127u;
            sfc[(lc & 31) * 16 + (lc >> 5) * 4 + blk] = static_cast<uint8_t>(byte);
            if (real) {
                const float f = inv_scale(byte);
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x[8] = {v[8 * k],     v[8 * k + 1], v[8 * k + 2], v[8 * k + 3],
                                        v[8 * k + 4], v[8 * k + 5], v[8 * k + 6], v[8 * k + 7]};
                    w[k] = codes8(x, f);
                }
                *reinterpret_cast<uint4*>(p.qt + (static_cast<long long>(cc) * p.kbt + block) * 16) =
                    make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        __syncthreads();
        if (threadIdx.x < 128)
            p.sft[(static_cast<long long>(tc) * p.tiles_r + tr) * 128 + threadIdx.x] =
                reinterpret_cast<const uint32_t*>(sfc)[threadIdx.x];
    }
}

// ---------------------------------------------------------------------------
// Values of an operand: a thread takes 8 columns.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float scale_value(uint32_t byte) {
    if (byte == 255u) return __uint_as_float(0x7FC00000u);
    return byte == 0u ? 0x1p-127f : __uint_as_float(byte << 23);
}

__device__ __forceinline__ float code_value(uint32_t c) {
    const uint32_t m = c & 7u;
    // magnitudes as fp32 bits: 0, 0.5, then exponent and one mantissa bit
    const float a = m < 2u ? 0.5f * static_cast<float>(m) : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1u) << 22);
    return c & 8u ? -a : a;
}

template <class T>
__global__ void __launch_bounds__(256) k_fp4_values(const uint8_t* q, const uint8_t* sf, int rows, int cols, int kb,
                                                    int tiles_c, T* out, long long ldo, int vec) {
    const long long per_row = 4LL * kb;
    const long long i = blockIdx.x * 256LL + threadIdx.x;
    if (i >= per_row * rows) return;
    const int row = static_cast<int>(i / per_row), s = static_cast<int>(i % per_row);
    const int block = s >> 2, col = 8 * s;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(q + (static_cast<long long>(row) * kb + block) * 16 + (s & 3) * 4);
    const float f = scale_value(
        sf[(static_cast<long long>(row >> 7) * tiles_c + (block >> 2)) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4 + (block & 3)]);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = code_value((w >> (4 * e)) & 15u) * f;
    T* o = out + row * ldo + col;
    if (vec && col + 8 <= cols) {
        if (sizeof(T) == 4) {
            reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                h[k] = *reinterpret_cast<const uint32_t*>(&b);
            }
            *reinterpret_cast<uint4*>(o) = make_uint4(h[0], h[1], h[2], h[3]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < cols) o[e] = static_cast<T>(v[e]);
    }
}

template <class T>
cudaError_t quantize_as(const QuantParams& p, cudaStream_t s) {
    const unsigned int grid = static_cast<unsigned int>(p.tiles_r) * p.tiles_c;
    constexpr int SMEM = 128 * 128 * 4;
    if (p.qt == nullptr) {
        k_fp4_quantize<T, true, false><<<grid, 256, 0, s>>>(p);
        return cudaGetLastError();
    }
    auto fn = p.q != nullptr ? k_fp4_quantize<T, true, true> : k_fp4_quantize<T, false, true>;
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    fn<<<grid, 256, SMEM, s>>>(p);
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
    const long long grid = (4LL * kb * rows + 255) / 256;
    const bool bf = dtype == MOARA_DTYPE_BF16;
    const int vec = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ldo % (bf ? 8 : 4) == 0;
    const uint8_t* qq = static_cast<const uint8_t*>(q);
    const uint8_t* ss = static_cast<const uint8_t*>(sf);
    ++*launches;
    if (bf)
        k_fp4_values<__nv_bfloat16><<<static_cast<unsigned int>(grid), 256, 0, s>>>(
            qq, ss, rows, cols, kb, fp4_tiles(cols), static_cast<__nv_bfloat16*>(out), ldo, vec);
    else
        k_fp4_values<float><<<static_cast<unsigned int>(grid), 256, 0, s>>>(qq, ss, rows, cols, kb, fp4_tiles(cols),
                                                                            static_cast<float*>(out), ldo, vec);
    return cudaGetLastError();
}

}  // namespace moara
