// MXFP4 products D = A B^T on the block-scaled tensor-core path.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "ops.h"
#include "tc_ptx.cuh"

namespace moara {
namespace {

// A stage holds 256 entries of K of both operands (128 bytes a row, one row of the
// 128-byte swizzle) and their scales, two 512-byte tiles per 128 rows.
constexpr int BM = 128, BN = 256, BK = 256;
constexpr int A_BYTES = BM * BK / 2, B_BYTES = BN * BK / 2;
constexpr int SFA_BYTES = 1024, SFB_BYTES = 2048;
constexpr int STAGE_BYTES = A_BYTES + B_BYTES + SFA_BYTES + SFB_BYTES;
constexpr int STAGES = 4;
constexpr int EPI_WARPS = 8;
constexpr int THREADS = (2 + EPI_WARPS) * 32;
constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + 256;
// tensor memory: the accumulator, then each stage's scales (A: 2 x 4 columns,
// B: 2 x 8)
constexpr int TMEM_SF = BN, TMEM_STAGE = 24;
static_assert(TMEM_SF + STAGES * TMEM_STAGE <= 512, "tensor memory");
static_assert(STAGE_BYTES % 1024 == 0 && SMEM <= 227 * 1024, "stages stay on the swizzle's 1024-byte lines");
constexpr long long kWait = 1LL << 32;

struct ProductParams {
    CUtensorMap amap, bmap;
    const uint8_t* asf;
    const uint8_t* bsf;
    void* D;
    long long ldd;
    int M, N, K;
    int tiles_m, tiles_n;
    int ct;                // scale tiles along K
    int bf16;
    int vec;               // rows of D are 16-byte aligned
    int* status;
};

struct Ctl {
    uint64_t full[STAGES], empty[STAGES];
    uint64_t accf, acce, drain;
    uint32_t tmem;
    int abort;
};

__device__ __forceinline__ bool drained(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!ptx::mbar_try_wait(bar, parity))
        if (clock64() - t0 > kWait) return false;
    return true;
}

// Tiles in groups of G row tiles, so that the operands of the tiles in flight stay
// in L2.
template <int TM, int TN, int G, class P> __device__ __forceinline__ void grouped_tile(const P& p, int t, int& m0, int& n0) {
    const int per = G * p.tiles_n, g = t / per, first = g * G;
    const int rows = min(G, p.tiles_m - first), r = t - g * per;
    m0 = (first + r % rows) * TM;
    n0 = (r / rows) * TN;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void store16(const ProductParams& p, int row, int col, const float (&v)[16]) {
    const long long at = row * p.ldd + col;
    if (p.vec && col + 16 <= p.N) {
        if (p.bf16) {
            uint4* o = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.D) + at);
            o[0] = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
            o[1] = make_uint4(pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]), pack2(v[14], v[15]));
        } else {
            float4* o = reinterpret_cast<float4*>(static_cast<float*>(p.D) + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        if (col + e >= p.N) continue;
        if (p.bf16) static_cast<__nv_bfloat16*>(p.D)[at + e] = __float2bfloat16_rn(v[e]);
        else static_cast<float*>(p.D)[at + e] = v[e];
    }
}

// Warp 0 loads, warp 1 issues copies of scales and MMAs, eight warps drain.
__global__ void __launch_bounds__(THREADS, 1) k_fp4_product(const __grid_constant__ ProductParams p) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    Ctl* ctl = reinterpret_cast<Ctl*>(smem + STAGES * STAGE_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &ctl->abort;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            ptx::mbar_init(ptx::smem_u32(&ctl->full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->empty[s]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&ctl->accf), 1);
        ptx::mbar_init(ptx::smem_u32(&ctl->acce), EPI_WARPS);
        ptx::mbar_init(ptx::smem_u32(&ctl->drain), 1);
        ctl->abort = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_u32(&ctl->tmem), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    const int tiles = p.tiles_m * p.tiles_n;
    const int steps = (p.K + BK - 1) / BK;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, issued = 0, last = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
                int m0, n0;
                grouped_tile<BM, BN, 16>(p, t, m0, n0);
                const int nt = n0 + 128 < p.N ? 2 : 1;             // scale tiles along N
                for (int k = 0; k < steps; ++k) {
                    if (!ptx::mbar_wait(ptx::smem_u32(&ctl->empty[stage]), phase ^ 1, abort_flag, p.status,
                                        MOARA_ERR_DEVICE_TIMEOUT, kWait)) {
                        ok = false;
                        break;
                    }
                    const uint32_t fb = ptx::smem_u32(&ctl->full[stage]);
                    const uint32_t a = ptx::smem_u32(smem + stage * STAGE_BYTES);
                    const uint32_t b = a + A_BYTES, sa = b + B_BYTES, sb = sa + SFA_BYTES;
                    const int at = 2 * k;                           // first scale tile along K
                    const uint32_t sfb = min(2, p.ct - at) * 512u;
                    ptx::mbar_arrive_expect_tx(fb, A_BYTES + B_BYTES + sfb * (1 + nt));
                    ptx::tma_load_2d(a, &p.amap, fb, k * (BK / 2), m0);
                    ptx::tma_load_2d(b, &p.bmap, fb, k * (BK / 2), n0);
                    ptx::bulk_load(sa, p.asf + (static_cast<long long>(m0 >> 7) * p.ct + at) * 512, sfb, fb);
                    for (int j = 0; j < nt; ++j)
                        ptx::bulk_load(sb + j * 1024, p.bsf + (static_cast<long long>((n0 >> 7) + j) * p.ct + at) * 512,
                                       sfb, fb);
                    issued |= 1u << stage;
                    last = (last & ~(1u << stage)) | (phase << stage);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
            for (int s = 0; s < STAGES; ++s)
                if (issued & (1u << s)) drained(ptx::smem_u32(&ctl->full[s]), (last >> s) & 1);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, acc = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, acc ^= 1) {
                int m0, n0;
                grouped_tile<BM, BN, 16>(p, t, m0, n0);
                const int nt = n0 + 128 < p.N ? 2 : 1;
                ok = ptx::mbar_wait(ptx::smem_u32(&ctl->acce), acc ^ 1, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT,
                                    kWait);
                if (!ok) break;
                ptx::tc_fence_after();
                for (int k = 0; k < steps; ++k) {
                    if (!ptx::mbar_wait(ptx::smem_u32(&ctl->full[stage]), phase, abort_flag, p.status,
                                        MOARA_ERR_DEVICE_TIMEOUT, kWait)) {
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after();
                    const uint32_t a = ptx::smem_u32(smem + stage * STAGE_BYTES);
                    const uint32_t b = a + A_BYTES, sa = b + B_BYTES, sb = sa + SFA_BYTES;
                    const uint32_t ta = tmem + TMEM_SF + stage * TMEM_STAGE, tb = ta + 8;
                    const int mmas = min(4, (p.K - k * BK + 63) / 64);
                    for (int h = 0; h < (mmas + 1) / 2; ++h) {
                        ptx::tmem_cp_scales(ta + 4 * h, ptx::smem_desc_plain(sa + 512 * h, 128));
                        for (int j = 0; j < nt; ++j)
                            ptx::tmem_cp_scales(tb + 8 * h + 4 * j, ptx::smem_desc_plain(sb + 1024 * j + 512 * h, 128));
                    }
                    for (int i = 0; i < mmas; ++i)
                        ptx::mma_mxf4(tmem, ptx::smem_desc_sw128(a + 32 * i, 16, 1024),
                                      ptx::smem_desc_sw128(b + 32 * i, 16, 1024), ptx::idesc_mxf4(BM, 128 * nt, i & 1),
                                      ta + 4 * (i >> 1), tb + 8 * (i >> 1), (k | i) != 0);
                    ptx::mma_commit(ptx::smem_u32(&ctl->empty[stage]));
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
                ptx::mma_commit(ptx::smem_u32(&ctl->accf));
            }
            ptx::mma_commit(ptx::smem_u32(&ctl->drain));
            drained(ptx::smem_u32(&ctl->drain), 0);
        }
    } else {
        // lane quadrant warp % 4, column half (warp - 2) / 4
        const int quad = warp & 3, half = (warp - 2) >> 2;
        uint32_t acc = 0;
        for (int t = blockIdx.x; t < tiles; t += gridDim.x, acc ^= 1) {
            int m0, n0;
            grouped_tile<BM, BN, 16>(p, t, m0, n0);
            const bool got = ptx::mbar_wait(ptx::smem_u32(&ctl->accf), acc, abort_flag, p.status,
                                            MOARA_ERR_DEVICE_TIMEOUT, kWait);
            if (!__all_sync(0xffffffffu, got)) break;
            ptx::tc_fence_after();
            const int row = m0 + quad * 32 + lane;
            for (int c = 0; c < 8; ++c) {
                const int col = n0 + half * 128 + c * 16;
                if (col >= p.N) break;                              // warp-uniform
                float v[16];
                __syncwarp();
                ptx::tmem_ld16(tmem + (static_cast<uint32_t>(quad * 32) << 16) + half * 128 + c * 16, v);
                if (row < p.M) store16(p, row, col, v);
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->acce));
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

// ---------------------------------------------------------------------------
// Large products: 2-CTA pairs, tile 256 x 256.  Each CTA loads its 128 rows of A and
// half of B's rows per stage and the scales of its rows of A and of all of B's;
// the even CTA issues.  The accumulator is not doubled (256 columns, beside which
// the scales of every stage live): eight warps take it whole into registers,
// which costs some hundred cycles between two tiles, and store it beside the next
// tile's MMAs.
// ---------------------------------------------------------------------------
constexpr int P_BM = 256, P_BN = 256;
constexpr int P_OPERAND = 128 * BK / 2;                            // 16 KB: 128 rows of A or B
constexpr int P_STAGE = 2 * P_OPERAND + SFA_BYTES + SFB_BYTES;
constexpr int P_STAGES = 6;
constexpr int P_SMEM = 1024 + P_STAGES * P_STAGE + 256;
static_assert(P_STAGE % 1024 == 0 && P_SMEM <= 227 * 1024, "stages stay on the swizzle's 1024-byte lines");
static_assert(P_BN + P_STAGES * TMEM_STAGE <= 512, "tensor memory");

struct PairParams {
    CUtensorMap amap, bmap, samap, sbmap;
    void* D;
    long long ldd;
    int M, N, K;
    int tiles_m, tiles_n;
    int bf16;
    int vec;               // bytes to which rows of D are aligned: 32, 16 or 0
    int* status;
};

struct PairCtl {
    uint64_t full[P_STAGES], empty[P_STAGES];
    uint64_t accf, acce, drain;
    uint32_t tmem;
    int abort;
};

// 128 columns of one row of D.
__device__ __forceinline__ void store128(const PairParams& p, int row, int col, const uint32_t (&v)[128]) {
    const long long at = row * p.ldd + col;
    if (p.bf16) {
        __nv_bfloat16* d = static_cast<__nv_bfloat16*>(p.D) + at;
#pragma unroll
        for (int c = 0; c < 128; c += 16) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = pack2(__uint_as_float(v[c + 2 * e]), __uint_as_float(v[c + 2 * e + 1]));
            if (p.vec == 32 && col + c + 16 <= p.N) {
                ptx::st_global_256(d + c, w);
            } else if (p.vec == 16 && col + c + 16 <= p.N) {
                reinterpret_cast<uint4*>(d + c)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4*>(d + c)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (col + c + e < p.N) d[c + e] = __float2bfloat16_rn(__uint_as_float(v[c + e]));
            }
        }
    } else {
        float* d = static_cast<float*>(p.D) + at;
#pragma unroll
        for (int c = 0; c < 128; c += 8) {
            const uint32_t w[8] = {v[c], v[c + 1], v[c + 2], v[c + 3], v[c + 4], v[c + 5], v[c + 6], v[c + 7]};
            if (p.vec == 32 && col + c + 8 <= p.N) {
                ptx::st_global_256(d + c, w);
            } else if (p.vec == 16 && col + c + 8 <= p.N) {
                reinterpret_cast<uint4*>(d + c)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4*>(d + c)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + c + e < p.N) d[c + e] = __uint_as_float(w[e]);
            }
        }
    }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) k_fp4_pair(const __grid_constant__ PairParams p) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    PairCtl* ctl = reinterpret_cast<PairCtl*>(smem + P_STAGES * P_STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int crank = static_cast<int>(ptx::cluster_ctarank());
    volatile int* abort_flag = &ctl->abort;
    if (threadIdx.x == 0) {
        for (int s = 0; s < P_STAGES; ++s) {
            ptx::mbar_init(ptx::smem_u32(&ctl->full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->empty[s]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&ctl->accf), 1);
        ptx::mbar_init(ptx::smem_u32(&ctl->acce), 2 * EPI_WARPS);      // both CTAs' warps, on the even CTA
        ptx::mbar_init(ptx::smem_u32(&ctl->drain), 1);
        ctl->abort = 0;
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
    const int tiles = p.tiles_m * p.tiles_n;
    const int first = blockIdx.x >> 1, stride = gridDim.x >> 1;
    const int steps = (p.K + BK - 1) / BK;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += stride) {
                int m0, n0;
                grouped_tile<P_BM, P_BN, 8>(p, t, m0, n0);
                for (int k = 0; k < steps; ++k) {
                    if (!ptx::mbar_wait(ptx::smem_u32(&ctl->empty[stage]), phase ^ 1, abort_flag, p.status,
                                        MOARA_ERR_DEVICE_TIMEOUT, kWait)) {
                        ok = false;
                        break;
                    }
                    const uint32_t own = ptx::smem_u32(&ctl->full[stage]), fb = ptx::mapa(own, 0);
                    if (crank == 0) ptx::mbar_arrive_expect_tx(own, 2 * P_STAGE);
                    const uint32_t a = ptx::smem_u32(smem + stage * P_STAGE);
                    const uint32_t b = a + P_OPERAND, sa = b + P_OPERAND, sb = sa + SFA_BYTES;
                    ptx::tma_load_2d_pair(a, &p.amap, fb, k * (BK / 2), m0 + 128 * crank);
                    ptx::tma_load_2d_pair(b, &p.bmap, fb, k * (BK / 2), n0 + 128 * crank);
                    ptx::tma_load_2d_pair(sa, &p.samap, fb, k * 256, (m0 >> 7) + crank);
                    ptx::tma_load_2d_pair(sb, &p.sbmap, fb, k * 256, n0 >> 7);
                    if (++stage == P_STAGES) { stage = 0; phase ^= 1; }
                }
            }
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
                if (!ptx::mbar_wait(full + 8 * stage, phase, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT, kWait))
                    return false;
                ptx::tc_fence_after();
                if (leader) {
                    const uint32_t sa = base + stage * P_STAGE + 2 * P_OPERAND, sb = sa + SFA_BYTES;
                    const uint32_t ta = tmem + P_BN + stage * TMEM_STAGE, tb = ta + 8;
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
                    ok = ptx::mbar_wait_cluster(ptx::smem_u32(&ctl->acce), acc ^ 1, abort_flag, p.status,
                                                MOARA_ERR_DEVICE_TIMEOUT, kWait);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    acc ^= 1;
                }
                const bool last = k + 1 == steps;
                if (leader) {
                    const uint32_t a = base + stage * P_STAGE;
                    const uint32_t ta = tmem + P_BN + stage * TMEM_STAGE, tb = ta + 8;
                    const uint64_t da = ptx::smem_desc_sw128(a, 16, 1024);
                    const uint64_t db = ptx::smem_desc_sw128(a + P_OPERAND, 16, 1024);
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
            drained(ptx::smem_u32(&ctl->drain), 0);
        }
    } else {
        // lane quadrant warp % 4, column half (warp - 2) / 4
        const int quad = warp & 3, half = (warp - 2) >> 2;
        const uint32_t release = ptx::mapa(ptx::smem_u32(&ctl->acce), 0);
        uint32_t acc = 0;
        for (int t = first; t < tiles; t += stride, acc ^= 1) {
            int m0, n0;
            grouped_tile<P_BM, P_BN, 8>(p, t, m0, n0);
            const bool got = ptx::mbar_wait(ptx::smem_u32(&ctl->accf), acc, abort_flag, p.status,
                                            MOARA_ERR_DEVICE_TIMEOUT, kWait);
            if (!__all_sync(0xffffffffu, got)) break;
            ptx::tc_fence_after();
            uint32_t v[128];
            ptx::tmem_ld128(tmem + (static_cast<uint32_t>(quad * 32) << 16) + half * 128, v);
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_remote(release);
            const int row = m0 + crank * 128 + quad * 32 + lane;
            if (row < p.M) store128(p, row, n0 + half * 128, v);
        }
    }
    ptx::tc_fence_before();
    __syncwarp();
    ptx::cluster_sync();            // no CTA leaves while its peer may still signal or fill it
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
    p.vec = (d | pitch) % 32 == 0 ? 32 : (d | pitch) % 16 == 0 ? 16 : 0;
    p.status = status;
    const cudaError_t e = cudaFuncSetAttribute(k_fp4_pair, cudaFuncAttributeMaxDynamicSharedMemorySize, P_SMEM);
    if (e != cudaSuccess) return e;
    const long long tiles = static_cast<long long>(p.tiles_m) * p.tiles_n;
    k_fp4_pair<<<2 * static_cast<unsigned int>(std::min<long long>(tiles, 76)), THREADS, P_SMEM, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

size_t fp4_product_workspace(int, int, int) { return 0; }

cudaError_t launch_fp4_product(const Fp4Product& a, int* status, cudaStream_t s, int64_t* launches) {
    if (a.M > 128) {
        ++*launches;
        return launch_pair(a, status, s);
    }
    ProductParams p{};
    if (!encode(&p.amap, a.aq, a.M, a.K, BM) || !encode(&p.bmap, a.bq, a.N, a.K, BN)) return cudaErrorInvalidValue;
    p.asf = static_cast<const uint8_t*>(a.asf);
    p.bsf = static_cast<const uint8_t*>(a.bsf);
    p.D = a.D;
    p.ldd = a.ldd;
    p.M = a.M;
    p.N = a.N;
    p.K = a.K;
    p.tiles_m = (a.M - 1) / BM + 1;
    p.tiles_n = (a.N - 1) / BN + 1;
    p.ct = fp4_tiles(a.K);
    p.bf16 = a.dtype == MOARA_DTYPE_BF16;
    p.vec = (reinterpret_cast<uintptr_t>(a.D) & 15) == 0 && a.ldd % (p.bf16 ? 8 : 4) == 0;
    p.status = status;
    const cudaError_t e = cudaFuncSetAttribute(k_fp4_product, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    const long long tiles = static_cast<long long>(p.tiles_m) * p.tiles_n;
    k_fp4_product<<<static_cast<unsigned int>(std::min<long long>(tiles, 152)), THREADS, SMEM, s>>>(p);
    ++*launches;
    return cudaGetLastError();
}

}  // namespace moara
