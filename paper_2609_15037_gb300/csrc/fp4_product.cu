// MXFP4 products D = A B^T on the block-scaled tensor-core path.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "fp4.cuh"
#include "fp4_settle.h"
#include "launch.cuh"
#include "ops.h"
#include "tc_ptx.cuh"
#include "waits.cuh"

namespace moara {
namespace {

// A stage holds 256 entries of K of both operands (128 bytes a row, one row of the
// 128-byte swizzle) and their scales, two 512-byte tiles per 128 rows.
constexpr int BK = 256;
constexpr int OPERAND = 128 * BK / 2;              // 16 KB: 128 rows of either operand
constexpr int SF_BYTES = 1024;                     // the scales of 128 rows

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// ---------------------------------------------------------------------------
// Products with few tiles.  The weight's rows are the MMA's 128 rows, up to 128 rows
// of A (tokens) its columns, so that a single token costs columns and not rows;
// a cluster of up to eight CTAs shares K, and each adds the others' sums for its
// share of the tokens through shared memory.  With the weight in L2, bound by latency (launch, one trip
// to memory, the sums) up to some hundred tokens, then by the operands' way from L2:
// with N = K = 4096 one token takes 4.6 us, 48 tokens 6.2, 128 8.2, 256 8.8 (a weight from
// DRAM: 5.2, and 8.2 against 6.1 with N = 11008, where its bytes are 3.5).  (A warp per two rows of
// the weight without tensor cores takes 4.7 us for a token there and 7.2 against 6.1 with
// N = 11008: the conversions bound it.)
// With QUANT, A comes as it is (at most 8 rows) and the four epilogue warps
// quantise a stage's rows into shared memory, so that a token's product is one
// launch (4.6 us); every CTA of a K range does that again, which pays for few rows: 8 take
// 5.9 us and some 6.4 with a launch of its own for the quantisation, 16 take 8.1 and 6.4.
// ---------------------------------------------------------------------------
constexpr int F_THREADS = 6 * 32;                  // TMA, MMA, four epilogue warps
constexpr int F_STAGES = 4;                        // at most
constexpr int F_TMEM = 256, F_TMEM_SF = 128, F_TMEM_STAGE = 16;
constexpr int F_QUANT = 8;                         // most rows that are quantised on the way
static_assert(F_TMEM_SF + F_STAGES * F_TMEM_STAGE <= F_TMEM, "tensor memory");

struct FewParams {
    CUtensorMap wmap, xmap;
    const uint8_t* wsf;
    const uint8_t* xsf;
    const void* X;         // QUANT
    long long ldx;
    int xvec;              // rows of X may be read 16 bytes at a time
    void* D;
    long long ldd;
    int M, N, K;           // rows of A, rows of B, entries
    int tiles_n;
    int ct;                // scale tiles along K
    int nt;                // tokens of a tile, a multiple of 16
    int stages;
    int split;             // CTAs of a cluster
    int early;             // the launch in front wrote A only: B may be read before it has ended
    int bf16;
    int vec;               // four entries of a row of D may be written at once
    int ctl;               // offset of the barriers in shared memory
    int* status;
    long long wait_limit;  // clock cycles of a bounded wait before it gives up
};

struct FewCtl {
    uint64_t full[F_STAGES], empty[F_STAGES];
    uint64_t accf, drain;
    uint32_t tmem;
    int abort;
    int filled[5];         // stages that the producer and each quantising warp filled
};

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(a));
    return v;
}

// Eight entries of row `row` from column `col` on, zero outside.
template <class T>
__device__ __forceinline__ void load_x(const FewParams& p, int row, int col, Row<T, 8>& x) {
    const T* src = static_cast<const T*>(p.X) + row * p.ldx + col;
    if (p.xvec && col + 8 <= p.K) x.load(src);
    else x.load_some(src, p.K - col);
}

// MANY: a CTA's share of the tokens is added up and stored four tokens at a time.
template <bool QUANT, class T, bool MANY>
__global__ void __launch_bounds__(F_THREADS) k_fp4_few(const __grid_constant__ FewParams p) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    FewCtl* ctl = reinterpret_cast<FewCtl*>(smem + p.ctl);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % p.split, tile = blockIdx.x / p.split;
    const int n0 = tile % p.tiles_n * 128, m0 = tile / p.tiles_n * 128;
    const int steps = (p.K + BK - 1) / BK;
    const int k0 = static_cast<int>(static_cast<long long>(steps) * rank / p.split);
    const int k1 = static_cast<int>(static_cast<long long>(steps) * (rank + 1) / p.split);
    const int x_bytes = p.nt * (BK / 2), stage_bytes = OPERAND + x_bytes + 2 * SF_BYTES;
    volatile int* abort_flag = &ctl->abort;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            ptx::mbar_init(ptx::smem_u32(&ctl->full[s]), QUANT ? 5 : 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->empty[s]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&ctl->accf), 1);
        ptx::mbar_init(ptx::smem_u32(&ctl->drain), 1);
        ctl->abort = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_u32(&ctl->tmem), F_TMEM);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    asm volatile("griddepcontrol.launch_dependents;");
    if (!p.early) asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp == 0) {
        if (lane == 0) {
            // this CTA's copies of step k: the weight's, and the tokens'
            auto load_w = [&](int k, int stage) {
                const uint32_t fb = ptx::smem_u32(&ctl->full[stage]), w = ptx::smem_u32(smem + stage * stage_bytes);
                const uint32_t sf = min(2, p.ct - 2 * k) * 512u;
                ptx::mbar_arrive_expect_tx(fb, OPERAND + sf + (QUANT ? 0 : x_bytes + sf));
                ptx::tma_load_2d(w, &p.wmap, fb, k * (BK / 2), n0);
                ptx::bulk_load(w + OPERAND + x_bytes, p.wsf + (static_cast<long long>(n0 >> 7) * p.ct + 2 * k) * 512, sf, fb);
            };
            auto load_t = [&](int k, int stage) {
                if (QUANT) return;
                const uint32_t fb = ptx::smem_u32(&ctl->full[stage]), w = ptx::smem_u32(smem + stage * stage_bytes);
                const uint32_t sf = min(2, p.ct - 2 * k) * 512u;
                ptx::tma_load_2d(w + OPERAND, &p.xmap, fb, k * (BK / 2), m0);
                ptx::bulk_load(w + OPERAND + x_bytes + SF_BYTES,
                               p.xsf + (static_cast<long long>(m0 >> 7) * p.ct + 2 * k) * 512, sf, fb);
            };
            const int ahead = min(p.stages, k1 - k0);
            for (int i = 0; i < ahead; ++i) load_w(k0 + i, i);
            if (p.early) asm volatile("griddepcontrol.wait;" ::: "memory");
            for (int i = 0; i < ahead; ++i) load_t(k0 + i, i);
            int stage = 0, k = k0 + ahead;
            uint32_t phase = 0;
            for (; k < k1; ++k) {
                if (!ptx::mbar_wait(ptx::smem_u32(&ctl->empty[stage]), phase, abort_flag, p.status,
                                    MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit))
                    break;
                load_w(k, stage);
                load_t(k, stage);
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
            ctl->filled[4] = k - k0;
        }
    } else if (warp == 1) {
        const bool leader = ptx::elect_one();
        const uint32_t base = ptx::smem_u32(smem);
        int stage = 0;
        uint32_t phase = 0;
        for (int k = k0; k < k1; ++k) {
            if (!ptx::mbar_wait_warp(ptx::smem_u32(&ctl->full[stage]), phase, abort_flag, p.status,
                                     MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit))
                break;
            ptx::tc_fence_after();
            if (leader) {
                const uint32_t w = base + stage * stage_bytes, sw = w + OPERAND + x_bytes;
                const uint32_t tw = tmem + F_TMEM_SF + stage * F_TMEM_STAGE, tx = tw + 8;
                const uint64_t dsw = ptx::smem_desc_plain(sw, 128), dsx = ptx::smem_desc_plain(sw + SF_BYTES, 128);
                const uint64_t dw = ptx::smem_desc_sw128(w, 16, 1024), dx = ptx::smem_desc_sw128(w + OPERAND, 16, 1024);
                const int mmas = min(4, (p.K - k * BK + 63) / 64);
                const uint32_t idesc = ptx::idesc_mxf4(128, 0, 0) | static_cast<uint32_t>(p.nt >> 3) << 17;
                const uint32_t half = ptx::idesc_mxf4(0, 0, 1) ^ ptx::idesc_mxf4(0, 0, 0);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (2 * h >= mmas) break;
                    ptx::tmem_cp_scales(tw + 4 * h, dsw + 32 * h);
                    ptx::tmem_cp_scales(tx + 4 * h, dsx + 32 * h);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < mmas)
                        ptx::mma_mxf4(tmem, dw + 2 * i, dx + 2 * i, i & 1 ? idesc | half : idesc, tw + 4 * (i >> 1),
                                      tx + 4 * (i >> 1), (k - k0) | i);
                ptx::mma_commit(ptx::smem_u32(&ctl->empty[stage]));
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        if (leader) {
            ptx::mma_commit(ptx::smem_u32(&ctl->accf));
            ptx::mma_commit(ptx::smem_u32(&ctl->drain));
        }
        __syncwarp();
        wait_drain(ptx::smem_u32(&ctl->drain), 0);
    } else {
        const int quad = warp & 3;
        if (QUANT) {
            // a warp takes every fourth row: lane l has columns 8l .. +7 of the stage,
            // four lanes a block
            constexpr int PER = F_QUANT / 4;
            Row<T, 8> x[PER];
            auto fetch = [&](int k) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int row = quad + 4 * i;
                    if (row < p.M) load_x<T>(p, row, k * BK + 8 * lane, x[i]);
                }
            };
            fetch(k0);
            int stage = 0, k = k0;
            uint32_t phase = 0;
            for (; k < k1; ++k) {
                if (!ptx::mbar_wait_warp(ptx::smem_u32(&ctl->empty[stage]), phase ^ 1, abort_flag, p.status,
                                         MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit))
                    break;
                uint8_t* rows = smem + stage * stage_bytes + OPERAND;
                uint8_t* sf = rows + x_bytes + SF_BYTES;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int row = quad + 4 * i;
                    if (row >= p.M) break;                          // warp-uniform
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = x[i].get(e);
                    uint32_t top = x[i].top();
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const uint32_t byte = scale_byte(top);
                    // the 128-byte swizzle: 16-byte chunk ^ row % 8
                    *reinterpret_cast<uint32_t*>(rows + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4) =
                        codes8(v, inv_scale(byte));
                    if ((lane & 3) == 0) sf[(lane >> 4) * 512 + row * 16 + ((lane >> 2) & 3)] = static_cast<uint8_t>(byte);
                }
                if (k + 1 < k1) fetch(k + 1);
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->full[stage]));
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
            if (lane == 0) ctl->filled[quad] = k - k0;
        }
        if (ptx::mbar_wait_warp(ptx::smem_u32(&ctl->accf), 0, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit)) {
            // sums [token][128 rows of the weight] over the stages, which are all consumed
            ptx::tc_fence_after();
            float* part = reinterpret_cast<float*>(smem) + quad * 32 + lane;
            const int tokens = min(p.nt, p.M - m0);
            for (int c = 0; c < tokens; c += 16) {
                float v[16];
                __syncwarp();
                ptx::tmem_ld16(tmem + (static_cast<uint32_t>(quad * 32) << 16) + c, v);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (c + e < tokens) part[(c + e) * 128] = v[e];
            }
        }
    }
    // Tensor memory is given back before this CTA waits for others of its cluster: those may
    // themselves be waiting for some on an SM that holds as many CTAs as it has
    // tensor memory for.
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, F_TMEM);
    }
    // a wait that ran out: no copy stays in flight (otherwise the MMAs have waited for all)
    if (threadIdx.x == 0 && *abort_flag)
        settle_few<QUANT ? 4 : 0>(
            ctl->filled[4], ctl->filled, p.stages, [&](int s) { ptx::mbar_arrive(ptx::smem_u32(&ctl->full[s])); },
            [&](int s, uint32_t parity) { wait_drain(ptx::smem_u32(&ctl->full[s]), parity); });
    __syncwarp();
    ptx::cluster_sync();                                            // every CTA's sums are in its shared memory
    // whether a CTA of the cluster gave up: its sums are none, and nothing is stored
    const uint32_t gave_up =
        lane < p.split ? ptx::ld_cluster_u32(ptx::mapa(ptx::smem_u32(&ctl->abort), static_cast<uint32_t>(lane))) : 0u;
    {
        const int tokens = min(p.nt, p.M - m0), share = (tokens + p.split - 1) / p.split;
        const int t1 = min(tokens, (rank + 1) * share), col = n0 + 4 * lane;
        const uint32_t own = ptx::smem_u32(smem) + 16 * lane;
        constexpr int WARPS = F_THREADS / 32;
        auto put = [&](int t, const float4& sum) {
            const long long at = (m0 + t) * p.ldd + col;
            const float v[4] = {sum.x, sum.y, sum.z, sum.w};
            if (p.vec && col + 4 <= p.N) {
                if (p.bf16)
                    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.D) + at) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
                else
                    *reinterpret_cast<float4*>(static_cast<float*>(p.D) + at) = sum;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (col + e >= p.N) continue;
                    if (p.bf16) static_cast<__nv_bfloat16*>(p.D)[at + e] = __float2bfloat16_rn(v[e]);
                    else static_cast<float*>(p.D)[at + e] = v[e];
                }
            }
        };
        // what is read together: a token from each of up to eight CTAs, or four of many tokens
        // from one or two (128 x 8192 x 600: 7.7 us, token by token 9.6); in one kernel the two
        // take a single token 0.1 us longer
        if constexpr (MANY) {
            const uint32_t a = ptx::mapa(own, 0), b = ptx::mapa(own, p.split - 1);
            for (int t0 = rank * share + warp; t0 < t1; t0 += 4 * WARPS) {
                float4 x[4], y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = min(t0 + i * WARPS, t1 - 1);
                    x[i] = ld_cluster_f4(a + t * 512);
                    if (p.split == 2) y[i] = ld_cluster_f4(b + t * 512);
                }
                if (__any_sync(0xffffffffu, gave_up != 0)) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (t0 + i * WARPS >= t1) break;
                    if (p.split == 2) {
                        x[i].x += y[i].x; x[i].y += y[i].y; x[i].z += y[i].z; x[i].w += y[i].w;
                    }
                    put(t0 + i * WARPS, x[i]);
                }
            }
        } else {
            uint32_t from[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) from[r] = ptx::mapa(own, r < p.split ? r : 0);
            for (int t = rank * share + warp; t < t1; t += WARPS) {
                float4 part[8];
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < p.split) part[r] = ld_cluster_f4(from[r] + t * 512);
                if (__any_sync(0xffffffffu, gave_up != 0)) break;
                float4 sum = part[0];
#pragma unroll
                for (int r = 1; r < 8; ++r) {
                    if (r >= p.split) break;
                    sum.x += part[r].x; sum.y += part[r].y; sum.z += part[r].z; sum.w += part[r].w;
                }
                put(t, sum);
            }
        }
    }
    __syncwarp();
    ptx::cluster_sync();                                            // no CTA leaves while another reads its sums
}

// ---------------------------------------------------------------------------
// Large products: 2-CTA pairs, tile 256 x 256.  Each CTA loads its 128 rows of A and
// half of B's rows per stage and the scales of its rows of A and of all of B's;
// the even CTA issues.  The accumulator is not doubled (256 columns, beside which
// the scales of every stage live): eight warps take it whole into registers,
// which costs some hundred cycles between two tiles, and store it beside the next
// tile's MMAs, through 2 KB of shared memory each: rows of 64 bytes whatever their
// alignment.
//
// 16384 x 11008 x 4096 into bf16: 257 us, 5.7 PFLOP/s (three times the bf16 rate), at
// 2.0 GHz and 1376 of 1400 W; 8192^3 166 us, 6.6 PFLOP/s; 4096^3 28.4 us, 256 tiles in
// four rounds of 76 pairs.  A stage of 256 entries takes 670 clocks, its four MMAs
// 512 of them; what they wait for is not known (at 128 bytes a clock its 35 KB would be written
// to and read from shared memory in 560, but the tensor pipe's reads are counted at 27% of
// their peak).  The drain of a tile costs 0.4 us, the stores of D beside the MMAs another 0.5 of
// its 6.9; 0.6 have no account.
// ---------------------------------------------------------------------------
constexpr int P_BM = 256, P_BN = 256;
constexpr int EPI_WARPS = 8;
constexpr int P_THREADS = (2 + EPI_WARPS) * 32;
// tensor memory: the accumulator, then each stage's scales (A: 2 x 4 columns, B: 2 x 8)
constexpr int P_TMEM_STAGE = 24;
constexpr int P_STAGE = 2 * OPERAND + 3 * SF_BYTES;
constexpr int P_STAGES = 6;
constexpr int P_OUT = 32 * 64;                                     // a warp's staging of D: 32 rows of 64 bytes
constexpr int P_CTL = 256;
constexpr int P_SMEM = P_STAGES * P_STAGE + EPI_WARPS * P_OUT + P_CTL;
static_assert(P_STAGE % 1024 == 0 && P_SMEM <= 227 * 1024, "stages stay on the swizzle's 1024-byte lines");
static_assert(P_BN + P_STAGES * P_TMEM_STAGE <= 512, "tensor memory");

struct PairParams {
    CUtensorMap amap, bmap, samap, sbmap;
    void* D;
    long long ldd;
    int M, N, K;
    int tiles_m, tiles_n;
    int bf16;
    int vec;               // rows of D begin on 16-byte lines
    int* status;
    long long wait_limit;  // clock cycles of a bounded wait before it gives up
};

struct PairCtl {
    uint64_t full[P_STAGES], empty[P_STAGES];
    uint64_t accf, acce, drain;
    uint32_t tmem;
    int abort;
    uint32_t steps;        // stages that this CTA's producer filled
};
static_assert(sizeof(PairCtl) <= P_CTL, "the barriers fit behind the staging of D");

// Tiles in groups of eight row tiles, so that the operands of the tiles in flight stay
// in L2.
__device__ __forceinline__ void tile_of(const PairParams& p, int t, int& m0, int& n0) {
    constexpr int G = 8;
    const int per = G * p.tiles_n, g = t / per, first = g * G;
    const int rows = min(G, p.tiles_m - first), r = t - g * per;
    m0 = (first + r % rows) * P_BM;
    n0 = (r / rows) * P_BN;
}

// Bytes from an address to the next 16-byte line.
__device__ __forceinline__ int to_line(const uint8_t* at) {
    return static_cast<int>(-reinterpret_cast<uintptr_t>(at) & 15);
}

// 64 bytes of 32 rows from a warp's staging to D, 16 bytes a lane.  left: bytes of the
// rows that exist.  ANY: each row was staged from its first whole line on.
template <int ES, bool ANY>
__device__ __forceinline__ void store_rows(const uint8_t* stage, uint8_t* d, long long pitch, int rows, int left, int lane) {
    const int b = lane % 4 * 16;
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        const int r = i + lane / 4;
        if (r >= rows) continue;
        const uint8_t* x = stage + r * 64 + (((b >> 4) ^ ((r >> 1) & 3)) << 4);
        uint8_t* to = d + r * pitch + b;
        const int skip = ANY ? to_line(to) : 0;
        to += skip;
        if (b + 16 + skip <= left) {
            __stcs(reinterpret_cast<uint4*>(to), *reinterpret_cast<const uint4*>(x));   // D does not displace the operands in L2
        } else {
            const int end = left - (b + skip), eight = end & 8, four = end & 4;     // less than a line, or nothing
            if (end <= 0) continue;
            if (eight) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(x);
            if (four) *reinterpret_cast<uint32_t*>(to + eight) = *reinterpret_cast<const uint32_t*>(x + eight);
            if (ES == 2 && (end & 2))
                *reinterpret_cast<uint16_t*>(to + eight + four) = *reinterpret_cast<const uint16_t*>(x + eight + four);
        }
    }
}

// 256 bytes (64 words of lane = row) of a warp's 32 rows of D from row, col on.  Rows on
// other boundaries than 16 bytes leave as whole lines too, after their words were moved up
// in the registers: 7195 x 8923 x 246 into bf16 51.5 us, into fp32 91; stored by words or
// halves where they lie, 96 and 122 (N = 8928, whose rows are aligned: 37 and 60).
template <int ES>
__device__ __forceinline__ void store_words(const PairParams& p, uint8_t* stage, int row, int col, uint32_t (&w)[64], int lane) {
    constexpr int COLS = 64 / ES;                                   // of a 64-byte chunk
    const int rows = p.M - row;
    const long long pitch = p.ldd * ES;
    uint8_t* d = static_cast<uint8_t*>(p.D) + row * pitch + static_cast<long long>(col) * ES;
    if (!p.vec) {
        // what a row has in front of its first line, and the rest from there on
        uint8_t* first = d + lane * pitch;
        const int skip = to_line(first), have = lane < rows ? min(p.N - col, 4 * COLS) * ES : 0;
        const int half = skip & 2, four = skip & 4, eight = skip & 8;
        const bool all = skip <= have;
        if (!all) {                                                 // the last columns of D
#pragma unroll
            for (int e = 0; e < 16 / ES; ++e) {
                if (e * ES >= have) continue;
                if (ES == 2) *reinterpret_cast<uint16_t*>(first + 2 * e) = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
                else *reinterpret_cast<uint32_t*>(first + 4 * e) = w[e];
            }
        }
        if (ES == 2) {
            if (all && half) *reinterpret_cast<uint16_t*>(first) = static_cast<uint16_t>(w[0]);
#pragma unroll
            for (int e = 0; e < 64; ++e) w[e] = __funnelshift_r(w[e], e < 63 ? w[e + 1] : 0u, half * 8);
        }
        if (all && four) *reinterpret_cast<uint32_t*>(first + half) = w[0];
#pragma unroll
        for (int e = 0; e < 63; ++e) w[e] = four ? w[e + 1] : w[e];
        if (all && eight) *reinterpret_cast<uint2*>(first + half + four) = make_uint2(w[0], w[1]);
#pragma unroll
        for (int e = 0; e < 62; ++e) w[e] = eight ? w[e + 2] : w[e];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if (col + c * COLS >= p.N || rows <= 0) break;              // warp-uniform
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int x = 16 * c + 4 * j;
            *reinterpret_cast<uint4*>(stage + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[x], w[x + 1], w[x + 2], w[x + 3]);
        }
        __syncwarp();
        // up to the end of the rows, or of these 256 bytes
        const int left = (min(p.N - col, 4 * COLS) - c * COLS) * ES;
        uint8_t* to = d + 64 * c;
        if (p.vec) store_rows<ES, false>(stage, to, pitch, rows, left, lane);
        else store_rows<ES, true>(stage, to, pitch, rows, left, lane);
    }
}

__global__ void __launch_bounds__(P_THREADS, 1) k_fp4_pair(const __grid_constant__ PairParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];             // there is no room to align it here
    uint8_t* staging = smem + P_STAGES * P_STAGE;
    PairCtl* ctl = reinterpret_cast<PairCtl*>(staging + EPI_WARPS * P_OUT);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int crank = static_cast<int>(ptx::cluster_ctarank());
    volatile int* abort_flag = &ctl->abort;
    if ((ptx::smem_u32(smem) & 1023u) != 0) {                       // the same in every CTA
        if (threadIdx.x == 0) atomicCAS(p.status, 0, MOARA_ERR_ALIGN);
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < P_STAGES; ++s) {
            ptx::mbar_init(ptx::smem_u32(&ctl->full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->empty[s]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&ctl->accf), 1);
        ptx::mbar_init(ptx::smem_u32(&ctl->acce), 2 * EPI_WARPS);      // both CTAs' warps, on the even CTA
        ptx::mbar_init(ptx::smem_u32(&ctl->drain), 1);
        ctl->abort = 0;
        ctl->steps = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc2(ptx::smem_u32(&ctl->tmem), 512);
        ptx::tmem_relinquish2();
    }
    ptx::tc_fence_before();
    __syncwarp();
    ptx::cluster_sync();            // barriers of both CTAs initialised before any remote signal
    ptx::tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    pdl_begin();
    const int tiles = p.tiles_m * p.tiles_n;
    const int first = blockIdx.x >> 1, stride = gridDim.x >> 1;
    const int steps = (p.K + BK - 1) / BK;

    // this CTA's copies of step k of a tile into a stage
    auto fill = [&](int m0, int n0, int k, int stage) {
        const uint32_t own = ptx::smem_u32(&ctl->full[stage]), fb = ptx::mapa(own, 0);
        if (crank == 0) ptx::mbar_arrive_expect_tx(own, 2 * P_STAGE);
        const uint32_t a = ptx::smem_u32(smem + stage * P_STAGE);
        const uint32_t b = a + OPERAND, sa = b + OPERAND, sb = sa + SF_BYTES;
        ptx::tma_load_2d_pair(a, &p.amap, fb, k * (BK / 2), m0 + 128 * crank);
        ptx::tma_load_2d_pair(b, &p.bmap, fb, k * (BK / 2), n0 + 128 * crank);
        ptx::tma_load_2d_pair(sa, &p.samap, fb, k * 256, (m0 >> 7) + crank);
        ptx::tma_load_2d_pair(sb, &p.sbmap, fb, k * 256, n0 >> 7);
    };

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, filled = 0;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += stride) {
                int m0, n0;
                tile_of(p, t, m0, n0);
                for (int k = 0; k < steps; ++k) {
                    if (!ptx::mbar_wait(ptx::smem_u32(&ctl->empty[stage]), phase ^ 1, abort_flag, p.status,
                                        MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit)) {
                        ok = false;
                        break;
                    }
                    fill(m0, n0, k, stage);
                    ++filled;
                    if (++stage == P_STAGES) { stage = 0; phase ^= 1; }
                }
            }
            ctl->steps = filled;
        }
    } else if (warp == 1) {
        if (crank == 0) {
            // The whole warp runs the loop, so that addresses stay in uniform registers; one
            // lane issues.  A stage's scales are copied before the MMAs of the stage in
            // front are issued: beside them, not between the two.
            const bool leader = ptx::elect_one();
            const int mine = (tiles - first + stride - 1) / stride;
            const int total = mine * steps;
            const uint32_t base = ptx::smem_u32(smem), full = ptx::smem_u32(&ctl->full[0]);
            const uint32_t empty = ptx::smem_u32(&ctl->empty[0]);
            const int tail = (p.K - (steps - 1) * BK + 63) / 64;          // MMAs of a tile's last stage
            auto scales = [&](int stage, uint32_t phase) {
                if (!ptx::mbar_wait_warp(full + 8 * stage, phase, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit))
                    return false;
                ptx::tc_fence_after();
                if (leader) {
                    const uint32_t sa = base + stage * P_STAGE + 2 * OPERAND, sb = sa + SF_BYTES;
                    const uint32_t ta = tmem + P_BN + stage * P_TMEM_STAGE, tb = ta + 8;
                    const uint64_t da = ptx::smem_desc_plain(sa, 128), db = ptx::smem_desc_plain(sb, 128);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        ptx::tmem_cp_scales2(ta + 4 * h, da + 32 * h);
                        ptx::tmem_cp_scales2(tb + 8 * h, db + 32 * h);
                        ptx::tmem_cp_scales2(tb + 8 * h + 4, db + 64 + 32 * h);
                    }
                }
                __syncwarp();
                return true;
            };
            int stage = 0, k = 0;
            uint32_t phase = 0, acc = 0;
            bool ok = scales(0, 0);
            for (int g = 0; g < total && ok; ++g) {
                const int next = stage + 1 == P_STAGES ? 0 : stage + 1;
                if (g + 1 < total && !scales(next, next == 0 ? phase ^ 1 : phase)) break;
                if (k == 0) {
                    ok = ptx::mbar_wait_cluster_warp(ptx::smem_u32(&ctl->acce), acc ^ 1, abort_flag, p.status,
                                                     MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    acc ^= 1;
                }
                const bool last = k + 1 == steps;
                if (leader) {
                    const uint32_t a = base + stage * P_STAGE;
                    const uint32_t ta = tmem + P_BN + stage * P_TMEM_STAGE, tb = ta + 8;
                    const uint64_t da = ptx::smem_desc_sw128(a, 16, 1024);
                    const uint64_t db = ptx::smem_desc_sw128(a + OPERAND, 16, 1024);
                    const int mmas = last ? tail : 4;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < mmas)
                            ptx::mma2_mxf4(tmem, da + 2 * i, db + 2 * i, ptx::idesc_mxf4(P_BM, P_BN, i & 1),
                                           ta + 4 * (i >> 1), tb + 8 * (i >> 1), (k | i) != 0);
                    ptx::mma2_commit_mc(empty + 8 * stage, 0x3);
                    if (last) ptx::mma2_commit_mc(ptx::smem_u32(&ctl->accf), 0x3);
                }
                __syncwarp();
                k = last ? 0 : k + 1;
                stage = next;
                if (next == 0) phase ^= 1;
            }
            if (leader) ptx::mma2_commit_mc(ptx::smem_u32(&ctl->drain), 0x1);
            __syncwarp();
            wait_drain(ptx::smem_u32(&ctl->drain), 0);
        }
    } else {
        // lane quadrant warp % 4, column half (warp - 2) / 4
        const int quad = warp & 3, half = (warp - 2) >> 2;
        uint8_t* out = staging + (warp - 2) * P_OUT;
        const uint32_t release = ptx::mapa(ptx::smem_u32(&ctl->acce), 0);
        uint32_t acc = 0;
        for (int t = first; t < tiles; t += stride, acc ^= 1) {
            int m0, n0;
            tile_of(p, t, m0, n0);
            if (!ptx::mbar_wait_warp(ptx::smem_u32(&ctl->accf), acc, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT,
                                     p.wait_limit))
                break;
            ptx::tc_fence_after();
            const uint32_t from = tmem + (static_cast<uint32_t>(quad * 32) << 16) + half * 128;
            const int row = m0 + crank * 128 + quad * 32, col = n0 + half * 128;
            uint32_t w[64];
            if (p.bf16) {
                // both halves are rounded into 64 words before anything is stored
                uint32_t v[64];
                ptx::tmem_ld64(from, v);
#pragma unroll
                for (int e = 0; e < 32; ++e) w[e] = pack2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
                ptx::tmem_ld64(from + 64, v);
#pragma unroll
                for (int e = 0; e < 32; ++e) w[32 + e] = pack2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
            } else {
                ptx::tmem_ld64(from, w);
                store_words<4>(p, out, row, col, w, lane);
                __syncwarp();
                ptx::tmem_ld64(from + 64, w);
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_remote(release);
            if (p.bf16) store_words<2>(p, out, row, col, w, lane);
            else store_words<4>(p, out, row, col + 64, w, lane);
        }
    }
    ptx::tc_fence_before();
    __syncwarp();
    pair_abort(ctl, crank);
    __syncwarp();
    ptx::cluster_sync();            // no CTA leaves while its peer may still signal or fill it
    if (*abort_flag) {              // the same in both CTAs
        // the copies of any step do: every stage takes as many bytes
        if (threadIdx.x == 0) pair_settle<P_STAGES>(ctl, crank, [&](int, int stage) { fill(0, 0, 0, stage); });
        __syncwarp();
        ptx::cluster_sync();
    }
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc2(tmem, 512);
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encoder() {
    static const EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}

bool encode(CUtensorMap* map, const void* q, int rows, int cols, int box_rows) {
    EncodeTiledFn fn = encoder();
    if (fn == nullptr) return false;
    const cuuint64_t pitch = static_cast<cuuint64_t>(fp4_blocks(cols)) * 16;
    const cuuint64_t dims[2] = {pitch, static_cast<cuuint64_t>(rows)}, strides[1] = {pitch};
    const cuuint32_t box[2] = {BK / 2, static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(q), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Scales as words: 1024 bytes (two tiles along K) of `box_rows` row tiles.
bool encode_scales(CUtensorMap* map, const void* sf, int rows, int cols, int box_rows) {
    EncodeTiledFn fn = encoder();
    if (fn == nullptr) return false;
    const cuuint64_t pitch = static_cast<cuuint64_t>(fp4_tiles(cols)) * 512;
    const cuuint64_t dims[2] = {pitch / 4, static_cast<cuuint64_t>(fp4_tiles(rows))}, strides[1] = {pitch};
    const cuuint32_t box[2] = {256, static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(sf), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Lets a kernel take all shared memory of an SM: once per device, 0.4 us of a call
// otherwise.  One instantiation per kernel.
template <int ID, class... P> cudaError_t allow_shared(void (*fn)(P...)) {
    static std::atomic<uint64_t> done{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess || (device < 64 && (done.load() >> device & 1))) return e;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e == cudaSuccess && device < 64) done.fetch_or(1ull << device);
    return e;
}

cudaError_t launch_pair(const Fp4Product& a, int* status, cudaStream_t s) {
    PairParams p{};
    if (!encode(&p.amap, a.aq, a.M, a.K, 128) || !encode(&p.bmap, a.bq, a.N, a.K, 128) ||
        !encode_scales(&p.samap, a.asf, a.M, a.K, 1) || !encode_scales(&p.sbmap, a.bsf, a.N, a.K, 2))
        return cudaErrorInvalidValue;
    p.D = a.D;
    p.ldd = a.ldd;
    p.M = a.M;
    p.N = a.N;
    p.K = a.K;
    p.tiles_m = (a.M - 1) / P_BM + 1;
    p.tiles_n = (a.N - 1) / P_BN + 1;
    p.bf16 = a.dtype == MOARA_DTYPE_BF16;
    const uintptr_t d = reinterpret_cast<uintptr_t>(a.D), pitch = static_cast<uintptr_t>(a.ldd) * (p.bf16 ? 2 : 4);
    p.vec = (d | pitch) % 16 == 0;
    p.status = status;
    p.wait_limit = a.wait_limit;
    const cudaError_t e = allow_shared<1>(k_fp4_pair);
    if (e != cudaSuccess) return e;
    const long long tiles = static_cast<long long>(p.tiles_m) * p.tiles_n;
    return launch(k_fp4_pair, dim3(2 * static_cast<unsigned int>(std::min<long long>(tiles, 76))), dim3(P_THREADS), P_SMEM,
                  s, 2, p);
}

// X: A as it is (quantised on the way), or null.
template <bool QUANT, class T>
cudaError_t launch_few(const Fp4Product& a, bool early, int* status, cudaStream_t s) {
    FewParams p{};
    p.nt = std::min(128, (a.M + 15) / 16 * 16);
    if (!encode(&p.wmap, a.bq, a.N, a.K, 128)) return cudaErrorInvalidValue;
    if (!QUANT && !encode(&p.xmap, a.aq, a.M, a.K, p.nt)) return cudaErrorInvalidValue;
    p.wsf = static_cast<const uint8_t*>(a.bsf);
    p.xsf = static_cast<const uint8_t*>(a.asf);
    p.X = a.X;
    p.ldx = a.ldx;
    p.xvec = (reinterpret_cast<uintptr_t>(a.X) & 15) == 0 && a.ldx * static_cast<int64_t>(sizeof(T)) % 16 == 0;
    p.D = a.D;
    p.ldd = a.ldd;
    p.M = a.M;
    p.N = a.N;
    p.K = a.K;
    p.tiles_n = (a.N - 1) / 128 + 1;
    p.ct = fp4_tiles(a.K);
    p.bf16 = a.dtype == MOARA_DTYPE_BF16;
    const uintptr_t size = p.bf16 ? 2 : 4;
    p.vec = (reinterpret_cast<uintptr_t>(a.D) | static_cast<uintptr_t>(a.ldd) * size) % (4 * size) == 0;
    p.early = early;
    p.status = status;
    p.wait_limit = a.wait_limit;
    const int steps = (a.K - 1) / BK + 1;
    const long long tiles = static_cast<long long>(p.tiles_n) * ((a.M - 1) / 128 + 1);
    // K over more CTAs while they are at most 5/4 of the SMs: with N = K = 4096 a token
    // takes 4.9 us in clusters of four (128 CTAs) and 7.2 in clusters of eight (256), with N
    // = 11008 6.6 in clusters of two (172) and 7.9 without.  Beyond half of the SMs the sums of
    // more than 32 tokens only repay a long K: 128 tokens, N = 2048, K = 2048 take 6.2 us in
    // clusters of four (64 CTAs) and 8.7 in clusters of eight; N = 4864, K = 2048 7.5 in
    // clusters of two (76) and 8.6 of four, but K = 11008 12.9 and 12.0
    p.split = 1;
    const auto pays = [&](int split) {
        const long long ctas = tiles * split;
        return split <= steps && (ctas <= 76 || (ctas <= 190 && (p.nt <= 32 || split * split <= steps)));
    };
    while (p.split < 8 && pays(2 * p.split)) p.split *= 2;
    p.stages = std::min(p.nt > 64 ? F_STAGES - 1 : F_STAGES, (steps - 1) / p.split + 1);    // two CTAs fit an SM
    const int stage = OPERAND + p.nt * (BK / 2) + 2 * SF_BYTES;
    p.ctl = (std::max(p.stages * stage, p.nt * 512) + 15) / 16 * 16;
    const int smem = 1024 + p.ctl + static_cast<int>(sizeof(FewCtl));
    const int share = (std::min(p.nt, a.M) - 1) / p.split + 1;
    const bool many = !QUANT && p.split <= 2 && share > 2 * (F_THREADS / 32);
    const auto fn = many ? k_fp4_few<QUANT, T, !QUANT> : k_fp4_few<QUANT, T, false>;
    const cudaError_t e = many ? allow_shared<8>(fn) : allow_shared<QUANT ? sizeof(T) : 0>(fn);
    if (e != cudaSuccess) return e;
    // begins beside the end of the launch in front where it is short or leaves room: a token
    // through 4096 x 4096 4.4 instead of 4.9 us in a row of them.  Otherwise two of its CTAs
    // share an SM while others idle (128 x 4096 x 4096: 8.8 us instead of 8.0)
    const bool overlap = early || p.nt <= 32 || tiles * p.split <= 76;
    return launch_if(overlap, fn, dim3(static_cast<unsigned int>(tiles * p.split)), dim3(F_THREADS), smem,
                     s, p.split, p);
}

// Pairs where their tiles occupy a quarter of the GPU and more, and a sixth where K is
// short; the other form, which shares K, below that.  20 tiles (512 x 2560 x 4096): 9.4 us against
// 10.3; 16 (512 x 2048): 9.4 against 8.6, but with K = 2048 7.0 against 7.7; 12 (512 x 1536 x 2048) 7.0
// against 7.5.
bool large(const Fp4Product& a) {
    const long long tiles = static_cast<long long>((a.M - 1) / P_BM + 1) * ((a.N - 1) / P_BN + 1);
    return tiles >= (a.K <= 2048 ? 12 : 19) && a.M > 128;
}

}  // namespace

bool fp4_quantizes(int M) { return M <= F_QUANT; }

cudaError_t launch_fp4_product(const Fp4Product& a, bool early, int* status, cudaStream_t s, int64_t* launches) {
    ++*launches;
    if (a.X != nullptr)
        return a.x_dtype == MOARA_DTYPE_BF16 ? launch_few<true, __nv_bfloat16>(a, false, status, s)
                                             : launch_few<true, float>(a, false, status, s);
    return large(a) ? launch_pair(a, status, s) : launch_few<false, float>(a, early, status, s);
}

}  // namespace moara
