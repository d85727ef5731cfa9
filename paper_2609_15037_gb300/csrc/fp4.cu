// MXFP4 operands: quantisation by rows and by columns from one read of the
// matrix, and the values of an operand.  DRAM-bound: per entry 4 or 2 bytes in
// and 17/32 of a byte out per orientation.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fp4.cuh"
#include "launch.cuh"
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

// One CTA takes a 128 x 128 tile, which is one 512-byte scale tile of either
// orientation.  A lane holds 8 rows x 16 bytes of columns (8 of bf16, 4 of fp32) in
// registers and a warp 32 rows x 8 lanes of them, so that a row's block of 32 columns is
// four or eight lanes, a column's block of 32 rows the four lanes 8 apart, and a
// lane's codes of either are one word, or half of one.  The matrix passes through no
// shared memory (32 x 1 blocks of a 64 KB tile there took 67 us on 11008 x 4096 fp32, where
// this takes 38: 5.9 TB/s); only the columns' codes do, to leave in whole 64-byte
// lines.  Every lane working out every scale of its rows and columns took 45 us.
template <class T> struct Quant {
    static constexpr int N = 16 / sizeof(T);                         // columns of a lane
    static constexpr int ACROSS = 128 / (8 * N);                     // warps across a tile
    static constexpr int THREADS = 4 * ACROSS * 32;
    static constexpr int BLOCK = 32 / N;                             // lanes of a row's block
};

// The maxima of V values over L lanes STEP apart, each in one lane: lane j of them (j
// counted in steps) is left with values j * V / L .. in t[0 .. V / L - 1].  Half of the
// values change lanes in each round, so a lane works out V / L scales, not V.
template <int V, int L, int STEP> __device__ __forceinline__ void scatter_max(uint32_t (&t)[V], int lane) {
    int have = V;
#pragma unroll
    for (int o = L / 2; o > 0; o /= 2) {
        const bool upper = (lane & (o * STEP)) != 0;
        have /= 2;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if (i >= have) break;
            const uint32_t keep = upper ? t[i + have] : t[i], send = upper ? t[i] : t[i + have];
            t[i] = max(keep, __shfl_xor_sync(0xffffffffu, send, o * STEP));
        }
    }
}

template <class T, bool ROWS, bool COLS>
__global__ void __launch_bounds__(Quant<T>::THREADS, sizeof(T) == 4 ? 2 : ROWS && COLS ? 3 : 4) k_fp4_quantize(const QuantParams p) {
    constexpr int N = Quant<T>::N, BLOCK = Quant<T>::BLOCK, THREADS = Quant<T>::THREADS;
    __shared__ __align__(16) uint8_t sfr[512];
    __shared__ __align__(16) uint8_t sfc[512];
    __shared__ __align__(16) uint32_t qc[COLS ? 128 * 17 : 1];       // a column's 16 words of codes, and one of padding
    // in this order: a product behind it that begins early finds what earlier launches
    // wrote complete
    asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
    const int tr = blockIdx.x / p.tiles_c, tc = blockIdx.x % p.tiles_c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wr = warp / Quant<T>::ACROSS, sub = warp % Quant<T>::ACROSS * 8 + (lane & 7);     // row group, column group
    const int lr = wr * 32 + (lane >> 3) * 8, lc = sub * N;          // the lane's entries inside the tile
    const int row0 = tr * 128 + lr, col0 = tc * 128 + lc;
    const T* X = static_cast<const T*>(p.X) + row0 * p.ld + col0;
    Row<T, N> x[8];
    if (p.vec && col0 + N <= p.cols && row0 + 8 <= p.rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i].load(X + i * p.ld);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i].load_some(X + i * p.ld, row0 + i < p.rows ? p.cols - col0 : 0);
    }
    if (ROWS) {
        const int block = (tc * 128 + lc) >> 5;
        constexpr int OWN = 8 / BLOCK;                               // rows whose scale this lane works out
        uint32_t half = 0, tops[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) tops[i] = x[i].top();
        scatter_max<8, BLOCK, 1>(tops, lane);
        float factor[OWN];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int r = lane % BLOCK * OWN + i;
            const uint32_t byte = row0 + r < p.rows && block < p.kb ? scale_byte(tops[i]) : 127u;
            sfr[((lr + r) & 31) * 16 + wr * 4 + lc / 32] = static_cast<uint8_t>(byte);
            factor[i] = inv_scale(byte);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = x[i].get(e);
            const float f = __shfl_sync(0xffffffffu, factor[i % OWN], i / OWN, BLOCK);
            uint8_t* q = p.q + static_cast<long long>(row0 + i) * p.kb * 16 + block * 16;
            if constexpr (N == 8) {
                if (block < p.kb && row0 + i < p.rows) *reinterpret_cast<uint32_t*>(q + lane % 4 * 4) = codes8(v, f);
            } else if (i % 2 == 0) {
                half = codes4(v, f);
            } else {
                // two lanes hold a word of two rows: each takes one row's
                const uint32_t low = half & 0xFFFFu, high = codes4(v, f) & 0xFFFFu, odd = lane & 1;
                const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? low : high, 1);
                if (block < p.kb && row0 + i - 1 + static_cast<int>(odd) < p.rows)
                    *reinterpret_cast<uint32_t*>(q - (odd ? 0 : static_cast<long long>(p.kb) * 16) + lane % 8 / 2 * 4) =
                        odd ? other | high << 16 : low | other << 16;
            }
        }
    }
    if (COLS) {
        const bool rows_real = tr * 4 + wr < p.kbt;
        uint32_t tops[N];
        Row<T, N>::tops(x, tops);
        scatter_max<N, 4, 8>(tops, lane);
        constexpr int OWN = N / 4;                                   // columns whose scale this lane works out
        float factor[OWN];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int c = lc + (lane >> 3) * OWN + i;
            const uint32_t byte = rows_real && tc * 128 + c < p.cols ? scale_byte(tops[i]) : 127u;
            sfc[(c & 31) * 16 + (c >> 5) * 4 + wr] = static_cast<uint8_t>(byte);
            factor[i] = inv_scale(byte);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[i].get(e);
            const float f = __shfl_sync(0xffffffffu, factor[e % OWN], (lane & 7) | e / OWN * 8);
            qc[(lc + e) * 17 + wr * 4 + (lane >> 3)] = codes8(v, f);
        }
    }
    __syncthreads();
    if (ROWS && threadIdx.x < 128)
        p.sf[(static_cast<long long>(tr) * p.tiles_c + tc) * 128 + threadIdx.x] =
            reinterpret_cast<const uint32_t*>(sfr)[threadIdx.x];
    if (COLS) {
        if (threadIdx.x >= 128 && threadIdx.x < 256)
            p.sft[(static_cast<long long>(tc) * p.tiles_r + tr) * 128 + threadIdx.x - 128] =
                reinterpret_cast<const uint32_t*>(sfc)[threadIdx.x - 128];
        // four lanes a column, 16 bytes (one block) each
        const int cols = min(128, p.cols - tc * 128), block = tr * 4 + (threadIdx.x & 3);
#pragma unroll
        for (int u = 0; u < 512 / THREADS; ++u) {
            const int c = u * (THREADS / 4) + (threadIdx.x >> 2);
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

struct ValueParams {
    const uint8_t* q;
    const uint8_t* sf;
    int rows, cols, kb, tiles_c;
    int lanes;             // log2 of the threads along a row, up to as many as it needs
    int parts;             // CTAs along a row
    void* out;
    long long ldo;
};

__device__ __forceinline__ uint32_t scale_at(const ValueParams& p, int row, int block) {
    return p.sf[(static_cast<long long>(row >> 7) * p.tiles_c + (block >> 2)) * 512 + (row & 31) * 16 +
                ((row & 127) >> 5) * 4 + (block & 3)];
}

// Rows of `out` on 16-byte boundaries.  A thread takes 8 columns of four rows, whose
// loads are issued together; a CTA up to 512 columns, and more rows of a narrow matrix.
// 11008 x 4096 into bf16: 15.8 us, 7.2 TB/s.
constexpr int VALUE_ROWS = 4, VALUE_LANES = 64;

template <class T> __global__ void __launch_bounds__(256) k_fp4_values(const ValueParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int part = blockIdx.x % p.parts, group = blockIdx.x / p.parts, step = 256 >> p.lanes;
    const int s = (part << p.lanes) + (threadIdx.x & ((1 << p.lanes) - 1)), block = s >> 2, col = 8 * s;
    const int row0 = group * (step * VALUE_ROWS) + (threadIdx.x >> p.lanes);
    if (block >= p.kb) return;
    uint32_t w[VALUE_ROWS], sb[VALUE_ROWS];
#pragma unroll
    for (int i = 0; i < VALUE_ROWS; ++i) {
        const int row = row0 + step * i;
        w[i] = sb[i] = 0;
        if (row >= p.rows) continue;
        w[i] = *reinterpret_cast<const uint32_t*>(p.q + (static_cast<long long>(row) * p.kb + block) * 16 + (s & 3) * 4);
        sb[i] = scale_at(p, row, block);
    }
#pragma unroll
    for (int i = 0; i < VALUE_ROWS; ++i) {
        const int row = row0 + step * i;
        if (row >= p.rows) return;
        float v[8];
        values8(w[i], scale_value(sb[i]), v);
        T* o = static_cast<T*>(p.out) + row * p.ldo + col;
        if (col + 8 <= p.cols) {
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
                if (col + e < p.cols) o[e] = static_cast<T>(v[e]);
        }
    }
}

// Rows on any boundary.  A thread works out 8 columns of four rows; a row's words are
// stored one to a lane, through shared memory, so that a store is contiguous.  In a row
// of bf16 that begins between two words a thread takes its columns one further on: the
// first code of its neighbour is its eighth.  11007 x 4097 into bf16 took 127 us with the
// columns of a thread stored one by one, 74 with two columns to a thread, and takes 45.
template <class T> __global__ void __launch_bounds__(256) k_fp4_values_any(const ValueParams p) {
    constexpr int WORDS = 2 * sizeof(T), SHIFT = sizeof(T) == 2 ? 2 : 3;          // of a thread's columns
    __shared__ __align__(16) uint32_t staged[256 * WORDS];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lanes = 1 << p.lanes, at_once = 32 >> p.lanes, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = blockIdx.x % p.parts, group = blockIdx.x / p.parts;
    const int s = part * lanes + (lane & (lanes - 1)), block = s >> 2;
    const int row0 = (group * 8 + warp) * at_once * VALUE_ROWS;
    uint8_t* const out = static_cast<uint8_t*>(p.out);
    const long long pitch = p.ldo * static_cast<long long>(sizeof(T));
    auto odd_row = [&](int row) {
        return sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(out + row * pitch) & 2) != 0;
    };
    uint32_t w[VALUE_ROWS], next[VALUE_ROWS], s0[VALUE_ROWS], s1[VALUE_ROWS];
#pragma unroll
    for (int i = 0; i < VALUE_ROWS; ++i) {
        const int row = row0 + i * at_once + (lane >> p.lanes);
        w[i] = next[i] = s0[i] = s1[i] = 0;
        if (row >= p.rows || block >= p.kb) continue;
        const uint8_t* q = p.q + (static_cast<long long>(row) * p.kb + block) * 16 + (s & 3) * 4;
        w[i] = *reinterpret_cast<const uint32_t*>(q);
        s0[i] = scale_at(p, row, block);
        if (sizeof(T) == 2 && s + 1 < 4 * p.kb) {
            next[i] = q[4];
            s1[i] = (s & 3) == 3 ? scale_at(p, row, block + 1) : s0[i];
        }
    }
    uint32_t* const mine = staged + warp * (32 * WORDS);
#pragma unroll
    for (int i = 0; i < VALUE_ROWS; ++i) {
        const int row = row0 + i * at_once + (lane >> p.lanes);
        const bool odd = row < p.rows && odd_row(row);
        float v[9];
        {
            float x[8];
            values8(w[i], scale_value(s0[i]), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = x[e];
        }
        if (sizeof(T) == 2) {
            float x[8];
            values8(next[i], scale_value(s1[i]), x);
            v[8] = x[0];
            if (odd && s == 0) *reinterpret_cast<T*>(out + row * pitch) = static_cast<T>(v[0]);
        }
        __syncwarp();
        uint32_t h[8];
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            if (sizeof(T) == 4) {
                h[k] = __float_as_uint(v[k]);
            } else {
                const __nv_bfloat162 y = __floats2bfloat162_rn(odd ? v[2 * k + 1] : v[2 * k], odd ? v[2 * k + 2] : v[2 * k + 1]);
                h[k] = *reinterpret_cast<const uint32_t*>(&y);
            }
        }
#pragma unroll
        for (int k = 0; k < WORDS; k += 4)
            *reinterpret_cast<uint4*>(mine + lane * WORDS + k) = make_uint4(h[k], h[k + 1], h[k + 2], h[k + 3]);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            const int x = k * 32 + lane, r = row0 + i * at_once + (x >> (p.lanes + SHIFT));
            const int word = x & ((lanes << SHIFT) - 1);
            if (r >= p.rows) break;
            uint8_t* row_at = out + r * pitch;
            const int shift = odd_row(r) ? 1 : 0;
            const int col = part * lanes * 8 + word * (4 / static_cast<int>(sizeof(T))) + shift;
            if (col + static_cast<int>(4 / sizeof(T)) <= p.cols)
                *reinterpret_cast<uint32_t*>(row_at + static_cast<long long>(col) * sizeof(T)) = mine[x];
            else if (sizeof(T) == 2 && col < p.cols)
                *reinterpret_cast<uint16_t*>(row_at + static_cast<long long>(col) * 2) = static_cast<uint16_t>(mine[x]);
        }
    }
}

template <class T>
cudaError_t quantize_as(const QuantParams& p, cudaStream_t s) {
    const unsigned int grid = static_cast<unsigned int>(p.tiles_r) * p.tiles_c;
    const auto fn = p.qt == nullptr  ? k_fp4_quantize<T, true, false>
                    : p.q == nullptr ? k_fp4_quantize<T, false, true>
                                     : k_fp4_quantize<T, true, true>;
    return launch(fn, dim3(grid), dim3(Quant<T>::THREADS), 0, s, 1, p);
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
    ValueParams p{};
    p.q = static_cast<const uint8_t*>(q);
    p.sf = static_cast<const uint8_t*>(sf);
    p.rows = rows;
    p.cols = cols;
    p.kb = fp4_blocks(cols);
    p.tiles_c = fp4_tiles(cols);
    p.out = out;
    p.ldo = ldo;
    const bool bf = dtype == MOARA_DTYPE_BF16;
    const bool vec = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ldo % (bf ? 8 : 4) == 0;
    const int units = 4 * p.kb;
    while ((1 << p.lanes) < units && (1 << p.lanes) < (vec ? VALUE_LANES : 32)) ++p.lanes;
    p.parts = ((units - 1) >> p.lanes) + 1;
    const int per = (256 >> p.lanes) * VALUE_ROWS;
    const unsigned int grid = static_cast<unsigned int>(p.parts) * ((rows - 1) / per + 1);
    auto fn = vec ? (bf ? k_fp4_values<__nv_bfloat16> : k_fp4_values<float>)
                  : (bf ? k_fp4_values_any<__nv_bfloat16> : k_fp4_values_any<float>);
    ++*launches;
    // begins early, but lets nothing begin beside itself: CTAs that wait would take its own
    // CTAs' places (both orientations of a 509 x 2049 matrix 19.2 us instead of 16.6)
    return launch(fn, dim3(grid), dim3(256), 0, s, 1, p);
}

}  // namespace moara
