// MXFP4 operands: quantisation by rows and by columns from one read of the
// matrix, and the values of an operand.  DRAM-bound: per entry 4 or 2 bytes in
// and 17/32 of a byte out per orientation.
#include <cuda_bf16.h>

#include <type_traits>

#include "fp4.cuh"
#include "launch.cuh"
#include "layers.h"
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
    const float* rstd;     // NORM: of the rows
    const float* gain;     // of the columns
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

// With NORM the entries are those of a norm's output, x rstd gain in fp32, which is never
// stored: the norm's kernel leaves h, which is still in L2, and rstd.
template <class T, bool ROWS, bool COLS, bool NORM>
__global__ void __launch_bounds__(Quant<T>::THREADS, sizeof(T) == 4 || NORM ? 2 : ROWS && COLS ? 3 : 4) k_fp4_quantize(const QuantParams p) {
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
    Row<T, N> from[8];
    const bool whole = col0 + N <= p.cols && row0 + 8 <= p.rows;
    // rows on other boundaries: by lines of 8 bytes, while they lie inside the matrix.  Eight
    // rows further a row begins on the same byte of its line.
    constexpr uintptr_t LINE = 7;
    const uintptr_t begin = reinterpret_cast<uintptr_t>(p.X);
    const uintptr_t end = reinterpret_cast<uintptr_t>(static_cast<const T*>(p.X) + (p.rows - 1) * p.ld + p.cols);
    if (whole && p.vec) {
#pragma unroll
        for (int i = 0; i < 8; ++i) from[i].load(X + i * p.ld);
    } else if (whole && (reinterpret_cast<uintptr_t>(X) & ~LINE) >= begin &&
               (reinterpret_cast<uintptr_t>(X + 7 * p.ld) & ~LINE) + 24 <= end) {
#pragma unroll
        for (int i = 0; i < 8; ++i) from[i].load_any(X + i * p.ld, static_cast<int>((begin + i * p.ld * sizeof(T)) & LINE));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) from[i].load_some(X + i * p.ld, row0 + i < p.rows ? p.cols - col0 : 0);
    }
    using Value = typename std::conditional<NORM, Row<float, N>, Row<T, N>>::type;
    Value x[8];
    if constexpr (NORM) {
        float g[N];
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = col0 + e < p.cols ? p.gain[col0 + e] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = row0 + i < p.rows ? p.rstd[row0 + i] : 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e)
                x[i].w[e] = row0 + i < p.rows && col0 + e < p.cols ? __float_as_uint(from[i].get(e) * s * g[e]) : 0u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = from[i];
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
        Value::tops(x, tops);
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
// Values of an operand.  Every value is a bf16 number (a code of two bits of exponent and
// one of mantissa times a power of two from 2^-127 on), so the products are taken two at
// a time in bf16, exactly, whatever the output's type.
// ---------------------------------------------------------------------------
// Bytes of the pair {a, b} by the nibbles of sel; a nibble's highest bit asks for the
// byte's highest bit eight times.
__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t sel) {
    uint32_t y;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(y) : "r"(a), "r"(b), "r"(sel));
    return y;
}

// Eight codes as bf16: 0, 1/2, 1, 3/2, 2, 3, 4, 6 from a table of each byte, then the signs.
__device__ __forceinline__ void values8(uint32_t w, uint32_t (&h)[4]) {
    const uint32_t sizes = w & 0x77777777u, even = w << 4;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t sel = sizes >> (16 * i), sign = permute(even, w, i == 0 ? 0xD9C8u : 0xFBEAu);
        const uint32_t low = permute(0xC0800000u, 0xC0804000u, sel);
        const uint32_t high = permute(0x3F3F3F00u, 0x40404040u, sel) | (sign & 0x80808080u);
        h[2 * i] = permute(low, high, 0x5140u);
        h[2 * i + 1] = permute(low, high, 0x7362u);
    }
}

// A scale twice as bf16: 2^-127 and NaN are the exponents' ends with the same bit beside them.
__device__ __forceinline__ uint32_t scale_value(uint32_t byte) {
    const uint32_t y = byte << 7 | (((byte + 1) & 0xFEu) == 0 ? 0x40u : 0u);
    return permute(y, y, 0x1010u);
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}

struct ValueParams {
    const uint8_t* q;
    const uint8_t* sf;
    int rows, cols, kb, tiles_c;
    int units;             // threads that a row needs, at most
    int lanes;             // log2 of the threads along a row, up to as many as it needs
    int parts;             // CTAs along a row
    void* out;
    long long ldo;
};

// A thread takes 16 bytes of the output (8 columns of bf16, 4 of fp32) of four adjacent
// rows, whose loads are issued together and whose scales lie 16 bytes apart; a CTA up to 64
// threads of a row, and more rows of a narrow matrix.  11008 x 4096 into bf16: 13.5 us, 8.5
// TB/s with what L2 keeps; conversions to fp32, products and packing there took 15.8, 95
// instructions for 16 bytes instead of 65.
// ANY: rows of `out` on any boundary.  A thread's 16 bytes are a line of the output all the
// same: their codes are the last of the thread's in front and the first of its own.  4978 x 5370
// into bf16: 14.3 us (4992 x 5376: 8.3); rows' words one to a lane through shared memory 25.7.
constexpr int VALUE_ROWS = 4, VALUE_LANES = 64;

template <class T, bool ANY> __global__ void __launch_bounds__(256) k_fp4_values(const ValueParams p) {
    constexpr int N = 16 / sizeof(T), PER = 32 / N;                  // columns of a thread, threads of a block
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int part = blockIdx.x % p.parts, group = blockIdx.x / p.parts, step = 256 >> p.lanes;
    const int s = (part << p.lanes) + (threadIdx.x & ((1 << p.lanes) - 1));
    const int row0 = (group * step + (threadIdx.x >> p.lanes)) * VALUE_ROWS, rows = p.rows - row0;
    if (s >= p.units || rows <= 0) return;
    const long long pitch = static_cast<long long>(p.kb) * 16;
    const uint8_t* const q0 = p.q + row0 * pitch;
    const uint8_t* const sf0 =
        p.sf + static_cast<long long>(row0 >> 7) * p.tiles_c * 512 + (row0 & 31) * 16 + ((row0 & 127) >> 5) * 4;
    // codes (in the low bits) and scales of the columns from N * unit on
    auto fetch = [&](int unit, uint32_t (&w)[VALUE_ROWS], uint32_t (&byte)[VALUE_ROWS]) {
        const int block = unit / PER;
        const uint8_t* q = q0 + static_cast<long long>(unit) * (N / 2);
        const uint8_t* sf = sf0 + static_cast<long long>(block >> 2) * 512 + (block & 3);
#pragma unroll
        for (int i = 0; i < VALUE_ROWS; ++i) {
            w[i] = byte[i] = 0;
            if (i >= rows || unit < 0 || block >= p.kb) continue;
            w[i] = N == 8 ? *reinterpret_cast<const uint32_t*>(q) : *reinterpret_cast<const uint16_t*>(q);
            byte[i] = sf[16 * i];
            q += pitch;
        }
    };
    uint32_t w[VALUE_ROWS], sb[VALUE_ROWS], before[VALUE_ROWS], sbefore[VALUE_ROWS];
    fetch(s, w, sb);
    if (ANY) fetch(s - 1, before, sbefore);
    T* o = static_cast<T*>(p.out) + row0 * p.ldo + N * static_cast<long long>(s);
#pragma unroll
    for (int i = 0; i < VALUE_ROWS; ++i, o += p.ldo) {
        if (i >= rows) return;
        // entries of the row's first line that are not the row's
        const int n = ANY ? static_cast<int>(reinterpret_cast<uintptr_t>(o) & 15) / static_cast<int>(sizeof(T)) : 0;
        const uint32_t f = scale_value(sb[i]);
        uint32_t h[4];
        if (ANY) {
            values8(N == 8 ? __funnelshift_l(before[i], w[i], 4 * n) : (w[i] << 16 | before[i]) >> (16 - 4 * n), h);
            const uint32_t pf = scale_value(sbefore[i]);
            // of each column's scale, which two bytes of {f, pf}
            uint32_t sel[4];
            sel[0] = 0x10101010u | __funnelshift_lc(0x44444444u, 0u, 8 * n);
            sel[2] = 0x10101010u | __funnelshift_lc(0x44444444u, 0u, max(8 * n - 32, 0));
            sel[1] = sel[0] >> 16;
            sel[3] = sel[2] >> 16;
#pragma unroll
            for (int k = 0; k < N / 2; ++k) h[k] = mul_bf16x2(h[k], permute(f, pf, sel[k]));
        } else {
            values8(w[i], h);
#pragma unroll
            for (int k = 0; k < N / 2; ++k) h[k] = mul_bf16x2(h[k], f);
        }
        if (N == 4) {
            h[3] = h[1] & 0xFFFF0000u;
            h[2] = h[1] << 16;
            h[1] = h[0] & 0xFFFF0000u;
            h[0] = h[0] << 16;
        }
        const int col = N * s - n;
        T* to = o - n;
        if (col >= 0 && col + N <= p.cols) {
            __stcs(reinterpret_cast<uint4*>(to), make_uint4(h[0], h[1], h[2], h[3]));
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (col + e < 0 || col + e >= p.cols) continue;
                if constexpr (N == 4) reinterpret_cast<uint32_t*>(to)[e] = h[e];
                else reinterpret_cast<uint16_t*>(to)[e] = static_cast<uint16_t>(h[e / 2] >> (16 * (e & 1)));
            }
        }
    }
}

template <class T, bool NORM>
cudaError_t quantize_as(const QuantParams& p, cudaStream_t s) {
    const unsigned int grid = static_cast<unsigned int>(p.tiles_r) * p.tiles_c;
    const auto fn = p.qt == nullptr  ? k_fp4_quantize<T, true, false, NORM>
                    : p.q == nullptr ? k_fp4_quantize<T, false, true, NORM>
                                     : k_fp4_quantize<T, true, true, NORM>;
    return launch(fn, dim3(grid), dim3(Quant<T>::THREADS), 0, s, 1, p);
}

QuantParams quant_params(const void* X, int dtype, int rows, int cols, int64_t ld, void* q, void* sf, void* qt, void* sft) {
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
    return p;
}

}  // namespace

cudaError_t launch_fp4_quantize(const void* X, int dtype, int rows, int cols, int64_t ld, void* q, void* sf, void* qt,
                                void* sft, cudaStream_t s, int64_t* launches) {
    const QuantParams p = quant_params(X, dtype, rows, cols, ld, q, sf, qt, sft);
    ++*launches;
    return dtype == MOARA_DTYPE_BF16 ? quantize_as<__nv_bfloat16, false>(p, s) : quantize_as<float, false>(p, s);
}

cudaError_t launch_norm_quantize(const void* h, int dtype, int rows, int cols, int64_t ld, const float* rstd,
                                 const float* gain, void* q, void* sf, void* qt, void* sft, cudaStream_t s,
                                 int64_t* launches) {
    QuantParams p = quant_params(h, dtype, rows, cols, ld, q, sf, qt, sft);
    p.rstd = rstd;
    p.gain = gain;
    ++*launches;
    return dtype == MOARA_DTYPE_BF16 ? quantize_as<__nv_bfloat16, true>(p, s) : quantize_as<float, true>(p, s);
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
    p.units = (cols - 1) / (bf ? 8 : 4) + (vec ? 1 : 2);
    while ((1 << p.lanes) < p.units && (1 << p.lanes) < VALUE_LANES) ++p.lanes;
    p.parts = ((p.units - 1) >> p.lanes) + 1;
    const int per = (256 >> p.lanes) * VALUE_ROWS;
    const unsigned int grid = static_cast<unsigned int>(p.parts) * ((rows - 1) / per + 1);
    auto fn = vec ? (bf ? k_fp4_values<__nv_bfloat16, false> : k_fp4_values<float, false>)
                  : (bf ? k_fp4_values<__nv_bfloat16, true> : k_fp4_values<float, true>);
    ++*launches;
    // begins early, but lets nothing begin beside itself: CTAs that wait would take its own
    // CTAs' places (both orientations of a 509 x 2049 matrix 19.2 us instead of 16.6)
    return launch(fn, dim3(grid), dim3(256), 0, s, 1, p);
}

}  // namespace moara
