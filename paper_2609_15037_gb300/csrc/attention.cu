// Causal attention over packed sequences with grouped heads, bf16 on the tensor cores.
//   S = scale q k^T (keys up to the query's own place in its sequence), P = softmax S,
//   O = P V, lse = log sum exp S
// and its gradients from dO, with delta = rowsum(dO O):
//   P = exp(S - lse), dV = P^T dO, dS = P (dO V^T - delta), dQ = scale dS K, dK = scale dS^T Q
// Bound by the tensor cores (4 D and 10 D operations a visible pair of query and key).  S
// and dS are fp32 sums in tensor memory and never leave the SM; P and dS are rounded to bf16
// for the products that take them, the form in which the tensor cores read them: an error
// of 2^-8 of each term at most, which the sums over keys or queries average (outputs 1.7e-3 of their
// norm from the exact ones, of which their own rounding is 1.66e-3; gradients 2.2e-3 to 2.7e-3).
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <climits>

#include "f32x2.cuh"
#include "launch.cuh"
#include "layers.h"
#include "tc_ptx.cuh"
#include "waits.cuh"

namespace moara {
namespace {

using bf16 = __nv_bfloat16;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int ROWS = 128;                       // of a tile of queries or keys
constexpr int PANEL = ROWS * 128;               // 64 columns of a tile: 128 rows of one line of the swizzle

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Descriptors of a tile, as an operand by rows and as the one whose rows are summed over, and
// that of a tile some bytes further on (they count in 16 bytes).  A product issues in fewer clocks where its
// descriptors are one number and constants (16384 tokens: 2% longer with each worked out).
__device__ __forceinline__ uint64_t by_rows(uint32_t tile) { return ptx::smem_desc_sw128(tile, 16, 1024); }
__device__ __forceinline__ uint64_t to_sum(uint32_t tile) { return ptx::smem_desc_sw128(tile, PANEL, 1024); }
__device__ __forceinline__ uint64_t beside(uint64_t d, int bytes) { return d + static_cast<uint64_t>(bytes / 16); }

// D = A B^T over DP columns, both tiles in shared memory by rows (K-major): 128 x 128.
template <int DP> __device__ __forceinline__ void mma_rows(uint32_t d, uint64_t da, uint64_t db) {
    constexpr uint32_t idesc = ptx::idesc_bf16(128, ROWS, 0, 0);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const int at = k / 4 * PANEL + k % 4 * 32;
        ptx::mma_f16(d, beside(da, at), beside(db, at), idesc, k > 0);
    }
}

// The same tile as the operand whose rows are summed over: D (128 x DP) (+)= A B with A in
// tensor memory, RUN entries of K in columns a .. a + RUN / 2 - 1, RUN more from a + PITCH on
// and so on; of the first 16 `steps` rows of B those from 16 FROM up to 16 TO.
template <int DP, int RUN, int PITCH, int FROM = 0, int TO = ROWS / 16>
__device__ __forceinline__ void mma_sum(uint32_t d, uint32_t a, uint64_t db, int steps, bool add) {
    constexpr uint32_t idesc = ptx::idesc_bf16(128, DP, 0, 1);
    const auto one = [&](int k, uint32_t acc) {
        ptx::mma_f16_ta(d, a + k * 16 / RUN * PITCH + k * 16 % RUN / 2, beside(db, k * 2048), idesc, acc);
    };
    // a test for each would take as long as a product; where the first is issued outside of the branch a
    // forward step of two halves takes 3% longer, where it is inside one of the gradients 1.5%
    if (FROM == 0 && TO == ROWS / 16) {
        one(0, add);
        if (steps >= TO) {
#pragma unroll
            for (int k = 1; k < TO; ++k) one(k, 1);
        } else {
            for (int k = 1; k < steps; ++k) one(k, 1);
        }
    } else if (steps >= TO) {
        one(FROM, add);
#pragma unroll
        for (int k = FROM + 1; k < TO; ++k) one(k, 1);
    } else {
        for (int k = FROM; k < steps; ++k) one(k, add || k > FROM);
    }
}

// Rows from `rows` to the next multiple of 16 of a tile become zero, by a warp that
// issues the products next: what lies there is another sequence's (or nothing), and a
// factor of zero does not silence its infinities and NaN.
template <int DP> __device__ __forceinline__ void clear_rows(uint8_t* tile, int rows, int lane) {
    const int n = ((rows + 15) / 16 * 16 - rows) * 8;              // 16-byte pieces of a panel
    for (int i = lane; i < n * (DP / 64); i += 32)
        *reinterpret_cast<uint4*>(tile + i / n * PANEL + rows * 128 + i % n * 16) = make_uint4(0, 0, 0, 0);
    ptx::fence_proxy_async_smem();
    __syncwarp();
}

// ---------------------------------------------------------------------------
// Which tile of which head entry n of a list of `heads` times its tiles is: sequence after sequence,
// some heads at a time, the last tile of each first.  Tiles that run side by side are of few
// heads, whose tensors the GPU's L2 holds (with a tile of all heads before the next one, the 128 heads
// of four sequences of 4096 tokens come from DRAM again and again: 1662 us for their gradients, so 1428), and of the heads that come
// last the shortest tiles come last.
// ---------------------------------------------------------------------------
struct Place {
    AttentionTile sequence;
    int tile, head;                              // tile: counted from the last
    __device__ __forceinline__ Place(const AttentionTile* list, int n, int heads, int rows) {
        sequence = list[n / heads];
        const int tiles = (sequence.length - 1) / rows + 1, most = max(1, min(heads, kBeside / tiles));
        int r = n - sequence.first * heads;
        const int group = r / (most * tiles), have = min(most, heads - group * most);
        r -= group * most * tiles;
        tile = r / have;
        head = group * most + r % have;
    }
    static constexpr int kBeside = 304;          // tiles of the heads that are taken together, two an SM
};

// ---------------------------------------------------------------------------
// Outputs.  A CTA takes 256 queries of a head, two tiles of 128, and goes through the
// keys in tiles of 128 from the sequence's first on.  While the four warps of one tile
// turn its S into P, the tensor cores work for the other: S (128 columns of tensor memory),
// over which P is written, and O (DP columns) each.  A row belongs to a thread.  A row's
// maximum is followed lazily: O is only rescaled once S exceeds the reference by 2^8, so
// that rows rarely wait for their O.  (The method is a published one: a running maximum, Milakov and Gimelshein 2018;
// over tiles of keys, Dao et al. 2022; two tiles of queries in turn, Shah et al. 2024.)  Q, K and V of the next pair of tiles come while this one's last steps
// run, its first S while O is stored: the tensor cores stand still between pairs for its first P alone.
// 16384 tokens, 28 heads on 4 of 128: 1174 to 1202 us, 1.60 to 1.64 PFLOP/s (0.85 of the cuBLAS burst rate, 0.93 of the
// sustained one).
// ---------------------------------------------------------------------------
template <int DP> struct Forward {
    static constexpr int TILE = DP / 64 * PANEL;
    static constexpr int SLOTS = DP == 128 ? 4 : 8;                // tiles of K and V in turn
    static constexpr int STAGE = 8 * 2048;                         // of the warps that store O
    static constexpr int CTL = 384;
    static constexpr int SMEM = (2 + SLOTS) * TILE + STAGE + CTL;
    static constexpr int THREADS = 10 * 32;                        // two tiles' warps, copies, products
};

struct ForwardParams {
    CUtensorMap q, k, v;
    bf16* out;
    bf16* rest;
    float* lse;
    const AttentionTile* pairs;
    int tokens, heads, group, dim;
    float scale, scale2;                         // of natural exponentials, and of powers of two
    int* status;
    long long wait_limit;
};

// 32 rows of a warp (one a lane) of CHUNKS 16-byte pieces from registers to rows of the output
// `pitch` bytes apart; `rows` of them exist, and `bytes` of each.  CHUNKS lanes exchange pieces
// until each has the same one of all their rows, so that a row's leave beside one another.
template <int CHUNKS>
__device__ __forceinline__ void store_rows(uint4 (&w)[CHUNKS], uint8_t* to, long long pitch, int rows, int bytes, int lane) {
#pragma unroll
    for (int s = CHUNKS / 2; s > 0; s /= 2) {
        const bool upper = (lane & s) != 0;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            if (i & s) continue;
            uint4 send = upper ? w[i] : w[i + s];
            send.x = __shfl_xor_sync(0xffffffffu, send.x, s);
            send.y = __shfl_xor_sync(0xffffffffu, send.y, s);
            send.z = __shfl_xor_sync(0xffffffffu, send.z, s);
            send.w = __shfl_xor_sync(0xffffffffu, send.w, s);
            if (upper) w[i] = send;
            else w[i + s] = send;
        }
    }
    const int c = lane % CHUNKS, r0 = lane - c;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
        if (r0 + i < rows && c * 16 < bytes) *reinterpret_cast<uint4*>(to + (r0 + i) * pitch + c * 16) = w[i];
}

// The same through shared memory of the warp's own, 32 CHUNKS 16 bytes: where registers are few, and
// the memory is free.
template <int CHUNKS>
__device__ __forceinline__ void store_rows(uint8_t* stage, const uint4 (&w)[CHUNKS], uint8_t* to, long long pitch, int rows, int bytes,
                                           int lane) {
    constexpr int MASK = CHUNKS < 8 ? CHUNKS - 1 : 7, PER = 32 / CHUNKS;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
        *reinterpret_cast<uint4*>(stage + (lane * CHUNKS + (c ^ (lane * CHUNKS / 8 & MASK))) * 16) = w[c];
    __syncwarp();
    const int c = lane % CHUNKS;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int r = i * PER + lane / CHUNKS;
        const uint4 v = *reinterpret_cast<const uint4*>(stage + (r * CHUNKS + (c ^ (r * CHUNKS / 8 & MASK))) * 16);
        if (r < rows && c * 16 < bytes) *reinterpret_cast<uint4*>(to + r * pitch + c * 16) = v;
    }
    __syncwarp();
}

// Waits of the warp that issues products.  Several at once: each costs some 100 clocks, and
// the queue of products holds about 200 clocks of them.
struct Waits {
    volatile int* abort;
    int* status;
    long long limit;
    __device__ __forceinline__ bool one(uint32_t bar, uint32_t parity) const {
        return ptx::mbar_wait_warp(bar, parity, abort, status, MOARA_ERR_DEVICE_TIMEOUT, limit);
    }
    __device__ __forceinline__ bool two(uint32_t a, uint32_t pa, uint32_t b, uint32_t pb) const {
        const bool x = ptx::mbar_try_wait(a, pa), y = ptx::mbar_try_wait(b, pb);
        return __all_sync(0xffffffffu, x && y) || (one(a, pa) && one(b, pb));
    }
    __device__ __forceinline__ bool three(uint32_t a, uint32_t pa, uint32_t b, uint32_t pb, uint32_t c, uint32_t pc) const {
        const bool x = ptx::mbar_try_wait(a, pa), y = ptx::mbar_try_wait(b, pb), z = ptx::mbar_try_wait(c, pc);
        return __all_sync(0xffffffffu, x && y && z) || (one(a, pa) && one(b, pb) && one(c, pc));
    }
};

// Two tiles of 128 queries of a head.
struct alignas(16) Pair {
    int begin, length, head;
    int q0;                                      // the first of the two, -1: no more of them
    __device__ __forceinline__ bool second() const { return (q0 + 1) * ROWS < length; }
    __device__ __forceinline__ int tiles() const { return q0 + 1 + second(); }     // of keys; tile i of the two sees q0 + 1 + i
};

__device__ __forceinline__ Pair pair_at(const ForwardParams& p, int n) {
    const Place x(p.pairs, n, p.heads, 2 * ROWS);
    return Pair{x.sequence.begin, x.sequence.length, x.head, 2 * ((x.sequence.length - 1) / (2 * ROWS) - x.tile)};
}

// Asks for a CTA of the grid that has not begun, in whose place this one goes on: the answer
// comes to shared memory beside the work.  Not again behind a refusal.
__device__ __forceinline__ void request(uint4* to, uint64_t& bar) {
    const uint32_t b = ptx::smem_u32(&bar);
    ptx::fence_proxy_async_smem();               // the last answer has been read
    ptx::mbar_arrive_expect_tx(b, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                     ptx::smem_u32(to)),
                 "r"(b)
                 : "memory");
}

// The index of that CTA, or -1.
__device__ __forceinline__ int answer(const uint4* from) {
    int n;
    asm volatile(
        "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t"
        "ld.shared.b128 r, [%1];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "mov.b32 %0, -1;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n\t}"
        : "=r"(n)
        : "r"(ptx::smem_u32(from))
        : "memory");
    return n;
}

template <int SLOTS> struct ForwardCtl {
    alignas(16) uint4 answer;                    // to the request for another CTA's tiles
    Pair pairs[2];                               // this CTA's, in turn
    struct {
        uint64_t sfull, pfull[2], ofull;
    } of[2];                                     // the two tiles of queries
    uint64_t qfull[2], qempty[2], full[SLOTS], empty[SLOTS], drain, answered, listed[2], taken[2];
    uint32_t tmem;
    int abort;
    uint32_t filled;                             // phases of the ring's last copies
    int filled_q[2];                             // copies of queries
};

// ONE: a CTA has one pair; otherwise it goes on with those of CTAs that have not begun, its next copies
// beside its last steps.
template <int DP, bool ONE>
__global__ void __launch_bounds__(Forward<DP>::THREADS, 1) k_attention(const __grid_constant__ ForwardParams p) {
    using F = Forward<DP>;
    using Ctl = ForwardCtl<F::SLOTS>;
    static_assert(sizeof(Ctl) <= F::CTL, "the barriers fit");
    extern __shared__ __align__(1024) uint8_t smem[];              // aligned here its addresses would be in registers
    uint8_t* ring = smem + 2 * F::TILE;
    uint8_t* stages = ring + F::SLOTS * F::TILE;
    Ctl* ctl = reinterpret_cast<Ctl*>(stages + F::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &ctl->abort;
    if ((ptx::smem_u32(smem) & 1023u) != 0) {                       // the same in every CTA
        if (threadIdx.x == 0) atomicCAS(p.status, 0, MOARA_ERR_ALIGN);
        return;
    }
    auto fill = [&](uint8_t* to, const CUtensorMap* map, uint64_t& bar, int h, int row) {
        const uint32_t b = ptx::smem_u32(&bar);
        ptx::mbar_arrive_expect_tx(b, F::TILE);
        for (int c = 0; c < DP / 64; ++c) ptx::tma_load_3d(ptx::smem_u32(to) + c * PANEL, map, b, c * 64, h, row);
    };
    if (threadIdx.x == 8 * 32) {
        // the thread that copies starts what the first products need beside the others' set-up
        for (int i = 0; i < 2; ++i) {
            for (uint64_t* x : {&ctl->qfull[i], &ctl->qempty[i], &ctl->of[i].sfull, &ctl->of[i].ofull, &ctl->listed[i]})
                ptx::mbar_init(ptx::smem_u32(x), 1);
            for (int h = 0; h < 2; ++h) ptx::mbar_init(ptx::smem_u32(&ctl->of[i].pfull[h]), 4);
            ptx::mbar_init(ptx::smem_u32(&ctl->taken[i]), 9);
        }
        for (int i = 0; i < F::SLOTS; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl->full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->empty[i]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&ctl->drain), 1);
        ptx::mbar_init(ptx::smem_u32(&ctl->answered), 1);
        ctl->abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
        pdl_begin();
        const Pair x = pair_at(p, blockIdx.x);
        ctl->pairs[0] = x;
        fill(smem, &p.q, ctl->qfull[0], x.head, x.begin + x.q0 * ROWS);
        fill(ring, &p.k, ctl->full[0], x.head / p.group, x.begin);
        if (x.second()) fill(smem + F::TILE, &p.q, ctl->qfull[1], x.head, x.begin + (x.q0 + 1) * ROWS);
        fill(ring + F::TILE, &p.v, ctl->full[1], x.head / p.group, x.begin);
    }
    if (warp == 9) {
        ptx::tmem_alloc(ptx::smem_u32(&ctl->tmem), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    pdl_begin();
    auto wait = [&](uint64_t& bar, uint32_t parity) {
        return ptx::mbar_wait_warp(ptx::smem_u32(&bar), parity, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit);
    };

    // the CTA's pair of a round, to every warp but the one that copies, until the warp has done with it
    auto pair_of = [&](int round, bool& ok) {
        if (round > 0) ok = wait(ctl->listed[round & 1], (round - 1) >> 1 & 1);
        return ok ? ctl->pairs[round & 1] : Pair{0, 0, 0, -1};
    };
    auto done_with = [&](int round) {
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->taken[round & 1]));
    };

    if (warp == 8) {
        if (lane == 0) {
            auto until = [&](uint64_t& bar, int phase) {
                return ptx::mbar_wait(ptx::smem_u32(&bar), phase & 1, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit);
            };
            uint32_t phases = ~0u;                                  // of the ring's slots
            int nq[2] = {};                                         // copies of queries
            bool ok = true;
            Pair x = ctl->pairs[0];
            for (int round = 0; ok && x.q0 >= 0; ++round) {
                const int kv = x.head / p.group, copies = 2 * x.tiles();
                auto copy_q = [&](int i) {
                    ok = nq[i] == 0 || until(ctl->qempty[i], nq[i] - 1);
                    if (!ok) return;
                    if (round > 0) fill(smem + i * F::TILE, &p.q, ctl->qfull[i], x.head, x.begin + (x.q0 + i) * ROWS);
                    ++nq[i];
                };
                auto copy = [&](int j) {
                    const int slot = j % F::SLOTS;
                    if (round > 0 || j > 1) {                       // those are begun above
                        // of a slot that has not been filled: the phase before its first
                        ok = until(ctl->empty[slot], phases >> slot);
                        if (!ok) return;
                        fill(ring + slot * F::TILE, j & 1 ? &p.v : &p.k, ctl->full[slot], kv, x.begin + j / 2 * ROWS);
                    }
                    phases ^= 1u << slot;
                };
                bool asked = false;
                copy_q(0);
                for (int j = 0; ok && j < copies; ++j) {
                    // a CTA's tiles that has not begun, once this one's last step is near
                    if (!ONE && j == copies - 2) {
                        request(&ctl->answer, ctl->answered);
                        asked = true;
                    }
                    copy(j);
                    if (ok && j == 0 && x.second()) copy_q(1);
                }
                if (ONE) break;
                if (!ok || !until(ctl->answered, round)) {
                    if (asked) wait_drain(ptx::smem_u32(&ctl->answered), round & 1);
                    break;
                }
                const int next = answer(&ctl->answer);
                if (next >= 0) x = pair_at(p, next);
                else x.q0 = -1;
                const int slot = (round + 1) & 1;
                ok = round == 0 || until(ctl->taken[slot], (round - 1) >> 1);
                if (!ok) break;
                ctl->pairs[slot] = x;
                ptx::mbar_arrive(ptx::smem_u32(&ctl->listed[slot]));
            }
            ctl->filled = phases;
            for (int i = 0; i < 2; ++i) ctl->filled_q[i] = nq[i];
        }
    } else if (warp == 9) {
        const bool leader = ptx::elect_one();
        const uint32_t base = ptx::smem_u32(smem), slots = ptx::smem_u32(ring);
        const Waits waits{abort_flag, p.status, p.wait_limit};
        const uint32_t full = ptx::smem_u32(&ctl->full[0]), pfull = ptx::smem_u32(&ctl->of[0].pfull[0]);
        uint32_t step[2] = {}, tile[2] = {};                        // of each of the two tiles, so far
        uint32_t phases = 0;                                        // of the ring's slots, with whose first a pair begins
        bool ok = true;
        for (int round = 0; !ONE || round < 1; ++round) {
            const Pair x = pair_of(round, ok);
            if (x.q0 < 0) break;
            const bool second = x.second();
            const int tiles = x.tiles();
            done_with(round);
            {
                // S over the last pair's P, whose product is in front; its O stays until this pair's P is there
                const uint32_t qfull = ptx::smem_u32(&ctl->qfull[0]);
                auto score = [&](int i) {
                    ptx::tc_fence_after();
                    if (leader) {
                        mma_rows<DP>(tmem + i * ROWS, by_rows(base + i * F::TILE), by_rows(slots));
                        ptx::mma_commit(ptx::smem_u32(&ctl->of[i].sfull));
                        if (i == 0 && x.q0 == 0) ptx::mma_commit(ptx::smem_u32(&ctl->qempty[0]));
                    }
                    __syncwarp();
                };
                if (!(ok = waits.two(qfull, tile[0]++ & 1, full, phases & 1))) break;
                score(0);
                if (second) {
                    if (!(ok = waits.one(qfull + 8, tile[1]++ & 1))) break;
                    score(1);
                }
                phases ^= 1;
                if (leader) ptx::mma_commit(ptx::smem_u32(&ctl->empty[0]));
                __syncwarp();
            }
            for (int j = 0; j < tiles && ok; ++j) {
                const int vs = (2 * j + 1) % F::SLOTS, ks = (2 * j + 2) % F::SLOTS;
                const bool more = j + 1 < tiles;
                const int left = x.length - j * ROWS;                // keys from this tile on
                const int steps = left >= ROWS ? ROWS / 16 : (left + 15) / 16;
                const uint32_t v = slots + vs * F::TILE, k = slots + ks * F::TILE;
                const uint32_t vp = phases >> vs & 1, kp = phases >> ks & 1;
                const bool one = j <= x.q0;                              // the first tile of queries sees these keys
                const uint32_t first = pfull + (one ? 0 : 32), parity = (one ? step[0] : step[1]) & 1;  // whose P comes first
                ok = more ? waits.three(full + 8 * vs, vp, full + 8 * ks, kp, first, parity)
                          : waits.two(full + 8 * vs, vp, first, parity);
                if (!ok) break;
                phases ^= 1u << vs | (more ? 1u << ks : 0);
                if (left < ROWS && left % 16 != 0) clear_rows<DP>(ring + vs * F::TILE, left, lane);
                if (one) {
                    ptx::tc_fence_after();
                    // P comes in halves, so that its product begins before all of it is there
                    if (leader) mma_sum<DP, ROWS, 0, 0, 4>(tmem + 256, tmem, to_sum(v), steps, j > 0);
                    __syncwarp();
                    if (!(ok = waits.one(pfull + 8, step[0] & 1))) break;
                    ptx::tc_fence_after();
                    if (leader) {
                        mma_sum<DP, ROWS, 0, 4, 8>(tmem + 256, tmem, to_sum(v), steps, true);
                        if (j == x.q0) {
                            ptx::mma_commit(ptx::smem_u32(&ctl->of[0].ofull));
                        } else {
                            // S over the P that the product in front of it has read by then
                            mma_rows<DP>(tmem, by_rows(base), by_rows(k));
                            ptx::mma_commit(ptx::smem_u32(&ctl->of[0].sfull));
                            if (j + 1 == x.q0) ptx::mma_commit(ptx::smem_u32(&ctl->qempty[0]));
                        }
                    }
                    __syncwarp();
                    ++step[0];
                    if (second && !(ok = waits.one(pfull + 32, step[1] & 1))) break;
                }
                if (second) {
                    ptx::tc_fence_after();
                    if (leader) mma_sum<DP, ROWS, 0, 0, 4>(tmem + 256 + DP, tmem + ROWS, to_sum(v), steps, j > 0);
                    __syncwarp();
                    if (!(ok = waits.one(pfull + 40, step[1] & 1))) break;
                    ptx::tc_fence_after();
                    if (leader) {
                        mma_sum<DP, ROWS, 0, 4, 8>(tmem + 256 + DP, tmem + ROWS, to_sum(v), steps, true);
                        if (!more) {
                            ptx::mma_commit(ptx::smem_u32(&ctl->of[1].ofull));
                        } else {
                            mma_rows<DP>(tmem + ROWS, by_rows(base + F::TILE), by_rows(k));
                            ptx::mma_commit(ptx::smem_u32(&ctl->of[1].sfull));
                            if (j + 2 == tiles) ptx::mma_commit(ptx::smem_u32(&ctl->qempty[1]));
                        }
                    }
                    __syncwarp();
                    ++step[1];
                }
                if (leader) {
                    ptx::mma_commit(ptx::smem_u32(&ctl->empty[vs]));
                    if (more) ptx::mma_commit(ptx::smem_u32(&ctl->empty[ks]));
                }
                __syncwarp();
            }
            if (!ok) break;
        }
        if (leader) ptx::mma_commit(ptx::smem_u32(&ctl->drain));
        __syncwarp();
        wait_drain(ptx::smem_u32(&ctl->drain), 0);
    } else {
        const int i = warp >> 2, quad = warp & 3, r = quad * 32 + lane;     // tile, lane quadrant, row
        const uint32_t st = tmem + (static_cast<uint32_t>(quad * 32) << 16) + i * ROWS;
        const uint32_t ot = st + 256 + i * (DP - ROWS);
        // registers are few.  Bit 0: phase of S, bit 1: of O, bit 2: whether this pair has begun, the others: pairs so far
        uint32_t at = 0;
        bool ok = true;
        for (; !ONE || at < 8; at = (at & ~4u) + 8) {
            int left;                                               // steps
            {
                const Pair x = pair_of(at >> 3, ok);
                if (x.q0 < 0) break;
                left = i == 0 ? x.q0 + 1 : x.second() ? x.tiles() : 0;
            }
            if (left == 0) {
                done_with(at >> 3);
                continue;
            }
            float ref = 0.0f, sum = 0.0f;                           // in units of S
            for (; left > 0; --left, at = (at | 4) ^ 1) {
                ok = wait(ctl->of[i].sfull, at & 1);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t s[2][64];
                ptx::tmem_ld64(st, s[0]);
                ptx::tmem_ld64(st + 64, s[1]);
                if (left == 1) {                                        // the diagonal
#pragma unroll
                    for (int c = 0; c < ROWS; ++c)
                        if (c > r) s[c / 64][c % 64] = 0xFF800000u;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < ROWS; c += 2)
                    top[c / 2 % 4] = max3(top[c / 2 % 4], __uint_as_float(s[c / 64][c % 64]), __uint_as_float(s[c / 64][c % 64 + 1]));
                float high = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                // nothing but minus infinity: a reference that the first finite score replaces
                if (high == -INFINITY) high = -1e30f;
                if ((at & 4) == 0) {
                    ref = high;
                } else if (__any_sync(0xffffffffu, (high - ref) * p.scale2 > 8.0f)) {
                    // S of this tile is there, so the products in front of it have added to O
                    const float to = fmaxf(high, ref), f = ex2((ref - to) * p.scale2);
                    ref = to;
                    sum *= f;
#pragma unroll
                    for (int c = 0; c < DP; c += 32) {
                        uint32_t o[32];
                        ptx::tmem_ld32(ot + c, o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        ptx::tmem_st32(ot + c, o);
                    }
                }
                const uint64_t by = both(p.scale2), shift = both(-ref * p.scale2);
                uint64_t part[2] = {};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t w[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        float a, b;
                        split(fma2(f32x2(__uint_as_float(s[h][2 * c]), __uint_as_float(s[h][2 * c + 1])), by, shift), a, b);
                        a = ex2(a);
                        b = ex2(b);
                        part[c & 1] = add2(part[c & 1], f32x2(a, b));
                        w[c] = pack2(a, b);
                    }
                    ptx::tmem_st32(st + 32 * h, w);
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->of[i].pfull[h]));
                }
                float a, b;
                split(add2(part[0], part[1]), a, b);
                sum += a + b;
            }
            if (ok) ok = wait(ctl->of[i].ofull, at >> 1 & 1);
            at ^= 2;
            if (ok) {
                ptx::tc_fence_after();
                const Pair pair = ctl->pairs[at >> 3 & 1];
                const int head = pair.head, row = (pair.q0 + i) * ROWS + r;     // in the sequence
                const float inv = 1.0f / sum;
                const long long token = pair.begin + row;
                if (row < pair.length) p.lse[static_cast<long long>(head) * p.tokens + token] = fmaf(ref, p.scale, logf(sum));
                const long long pitch = static_cast<long long>(p.heads) * p.dim * 2, first = ((token - lane) * p.heads + head) * p.dim;
                const int rows = pair.length - (row - lane);
#pragma unroll
                for (int c = 0; c < DP; c += 32) {
                    uint32_t o[32];
                    ptx::tmem_ld32(ot + c, o);
                    uint4 w[4], l[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t a[4], b[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float y = __uint_as_float(o[8 * e + 2 * x]) * inv, z = __uint_as_float(o[8 * e + 2 * x + 1]) * inv;
                            a[x] = pack2(y, z);
                            b[x] = pack2(y - __uint_as_float(a[x] << 16), z - __uint_as_float(a[x] & 0xFFFF0000u));
                        }
                        w[e] = make_uint4(a[0], a[1], a[2], a[3]);
                        l[e] = make_uint4(b[0], b[1], b[2], b[3]);
                    }
                    const int bytes = (p.dim - c) * 2;
                    uint8_t* const stage = stages + warp * (F::STAGE / 8);
                    store_rows(stage, w, reinterpret_cast<uint8_t*>(p.out + first + c), pitch, rows, bytes, lane);
                    if (p.rest != nullptr) store_rows(stage, l, reinterpret_cast<uint8_t*>(p.rest + first + c), pitch, rows, bytes, lane);
                }
            }
            done_with(at >> 3);
            if (!ok) break;
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) {      // a wait that ran out: no copy stays in flight
        for (int i = 0; i < 2; ++i)
            if (ctl->filled_q[i] > 0) wait_drain(ptx::smem_u32(&ctl->qfull[i]), (ctl->filled_q[i] - 1) & 1);
        for (int n = 0; n < F::SLOTS; ++n) wait_drain(ptx::smem_u32(&ctl->full[n]), ctl->filled >> n & 1);
    }
    if (warp == 9) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------
// Gradients.  Two kinds of tiles, so that every sum has one owner and one order (five products a
// pair of tiles become seven; adding dQ up where dK and dV are would need atomics, whose order
// changes the result).  KEYS: 128 keys of a head of k and v, against the queries that see them, of
// every head that shares it; with S^T = K Q^T, P^T and dS^T stay in tensor memory and
// dV += P^T dO, dK += dS^T Q take them from there.  Otherwise 128 queries of a head against their
// keys: dQ += dS K.
//
// Sixteen warps turn S into P and dP = dO V^T into dS (32 columns of a row a thread), one
// issues products, one copies.  A CTA takes tile after tile from a counter, each
// warp goes from one to the next on its own, and the next tile's first copies and products run
// beside this one's last sums and stores.  The operand that
// is used twice in a step (first in S, last in a sum) has three slots, the other two.  Where the
// longest tiles would outlast the rest, a cluster shares a tile's steps, and its CTAs add one
// another's sums, in order, through shared memory.
// ---------------------------------------------------------------------------
template <int DP> struct Backward {
    static constexpr int TILE = DP / 64 * PANEL;
    static constexpr int SA = 3, SB = 2;
    static constexpr int STATS = 2 * 2 * ROWS * 4;                 // lse and delta of two steps
    static constexpr int CTL = 512;
    static constexpr int SMEM = (2 + SA + SB) * TILE + STATS + CTL;
    static constexpr int WARPS = 16;                               // that turn S into dS
    static constexpr int THREADS = (WARPS + 2) * 32;
    static_assert(SMEM <= 227 * 1024, "shared memory");
};

struct BackwardParams {
    CUtensorMap q, k, v, dout;
    const float* lse;
    const float* delta;
    bf16* dq;
    bf16* dk;
    bf16* dv;
    const AttentionTile* tiles;
    unsigned int* counter;                       // of the tiles that have been taken, beyond one a CTA
    int n_tiles;
    int tokens, heads, kv_heads, group, dim;
    int split;                                   // CTAs of a cluster, which share a tile's steps
    float scale;
    int* status;
    long long wait_limit;
};

// dpfull and dsfull are those of even and of odd steps.  In tiles of queries dP of the next step is issued
// before this step's is waited for, and dS of the next may be there before this step's is: of a single barrier
// two phases could pass a waiting warp by, whose parity is the old one again.
struct BackwardCtl {
    uint64_t fixed, afull[3], aempty[3], bfull[2], bempty[2], sfull, pfull, dpfull[2], dsfull[2], stats[2], done, read, drain, listed[2], taken[2];
    uint32_t tmem;
    int abort;
    int filled[3];
    int tiles[2];                                // the CTA's next tiles, of which the warps learn here
};

// Tile n: those of the keys first, of which a group of heads makes the longest.  Its steps are every `split`-th of (head, tile) in order.  KEYS: tiles of queries from the keys' own
// to the sequence's last, for each head of the group; otherwise tiles of keys up to the queries' own.
struct Work {
    AttentionTile sequence;
    int tile, owner, kv;                         // of the sequence, the head that it is of, its head of k and v
    bool keys;
    int at, head, count;                         // of the next step; steps
    int first, last, stride, all;
    __device__ __forceinline__ bool get(const BackwardParams& p, int n) {
        const int rank = blockIdx.x % p.split, of_keys = p.n_tiles * p.kv_heads;
        if (n >= of_keys + p.n_tiles * p.heads) return false;
        keys = n < of_keys;
        if (!keys) n -= of_keys;
        const Place x(p.tiles, n, keys ? p.kv_heads : p.heads, ROWS);
        sequence = x.sequence;
        owner = x.head;
        kv = keys ? owner : owner / p.group;
        last = (sequence.length - 1) / ROWS;
        tile = keys ? x.tile : last - x.tile;
        first = keys ? tile : 0;
        stride = p.split;
        all = keys ? (last - first + 1) * p.group : tile + 1;
        count = all > rank ? (all - rank - 1) / p.split + 1 : 0;
        at = first + rank;
        head = keys ? kv * p.group : kv;
        wrap();
        return true;
    }
    __device__ __forceinline__ void wrap() {
        while (at > last) {
            at -= last - first + 1;
            ++head;
        }
    }
    __device__ __forceinline__ void next() {
        at += stride;
        wrap();
    }
    // rows of the step's tile that exist
    __device__ __forceinline__ int rows() const { return at == last ? sequence.length - last * ROWS : ROWS; }
    // first token of the tile
    __device__ __forceinline__ int token() const { return sequence.begin + tile * ROWS; }
};

// Where a CTA of a cluster leaves four columns of a row of its first or second sum.
template <int DP> __device__ __forceinline__ uint32_t sum_at(int which, int row, int c) {
    return (which * ROWS + row) * DP * 4 + (c ^ (row & 7)) * 16;
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
    return v;
}

// Columns of tensor memory.  KEYS: S, dP, dV, dK; otherwise S, dP of even and odd steps, dQ.
constexpr uint32_t COL_S = 0, COL_DP = 128, COL_SUM_B = 256, COL_SUM_A = 384;
template <bool KEYS> __device__ __forceinline__ uint32_t dp_column(int j) {
    return KEYS ? COL_DP : COL_DP + static_cast<uint32_t>(j & 1) * 128;
}

template <int DP> struct Shared {
    uint8_t* smem;
    uint8_t* ring_a;
    uint8_t* ring_b;
    float* stats;
    BackwardCtl* ctl;
    __device__ __forceinline__ explicit Shared(uint8_t* base) {
        using F = Backward<DP>;
        smem = base;
        ring_a = smem + 2 * F::TILE;
        ring_b = ring_a + F::SA * F::TILE;
        stats = reinterpret_cast<float*>(ring_b + F::SB * F::TILE);
        ctl = reinterpret_cast<BackwardCtl*>(ring_b + F::SB * F::TILE + F::STATS);
    }
};

// What the warp that issues products carries from tile to tile.
struct Products {
    uint32_t tmem;
    int sa = 0, sb = 0;                          // slots of both rings, whose phases end with theirs
    uint32_t pa = 0, pb = 0, step = 0, tile = 0;
};

template <int DP, bool KEYS>
__device__ __forceinline__ bool multiply(const Shared<DP>& x, const Waits& waits, Products& st, Work& work, bool leader, int lane) {
    using F = Backward<DP>;
    BackwardCtl* const ctl = x.ctl;
    const uint32_t fixed = ptx::smem_u32(x.smem), ra = ptx::smem_u32(x.ring_a), rb = ptx::smem_u32(x.ring_b);
    const uint32_t afull = ptx::smem_u32(&ctl->afull[0]), bfull = ptx::smem_u32(&ctl->bfull[0]);
    const uint32_t aempty = ptx::smem_u32(&ctl->aempty[0]), bempty = ptx::smem_u32(&ctl->bempty[0]);
    const uint32_t pfull = ptx::smem_u32(&ctl->pfull), sfull = ptx::smem_u32(&ctl->sfull);
    const uint32_t dsfull = ptx::smem_u32(&ctl->dsfull[0]), dpfull = ptx::smem_u32(&ctl->dpfull[0]);
    const uint32_t tmem = st.tmem;
    const int steps = work.count;
    // rows of the tile that a sum runs over
    int rows = work.rows();
    auto clean_a = [&] {
        if (rows % 16 != 0) clear_rows<DP>(x.ring_a + st.sa * F::TILE, rows, lane);
    };
    auto clean_b = [&] {
        if (KEYS && rows % 16 != 0) clear_rows<DP>(x.ring_b + st.sb * F::TILE, rows, lane);
    };
    if (steps == 0) return true;
    if (!waits.three(ptx::smem_u32(&ctl->fixed), st.tile & 1, afull + 8 * st.sa, st.pa, bfull + 8 * st.sb, st.pb)) return false;
    clean_a();
    clean_b();
    ptx::tc_fence_after();
    if (leader) {
        mma_rows<DP>(tmem + COL_S, by_rows(fixed), by_rows(ra + st.sa * F::TILE));
        ptx::mma_commit(sfull);
        mma_rows<DP>(tmem + COL_DP, by_rows(fixed + F::TILE), by_rows(rb + st.sb * F::TILE));
        ptx::mma_commit(dpfull + 8 * (st.step & 1));
        if (!KEYS) ptx::mma_commit(bempty + 8 * st.sb);
    }
    __syncwarp();
    // the last tile's sums have been read from the columns that this one's go to
    if (st.tile > 0 && !waits.one(ptx::smem_u32(&ctl->read), (st.tile - 1) & 1)) return false;
    for (int j = 0; j < steps; ++j, ++st.step) {
        const bool more = j + 1 < steps;
        const uint32_t parity = st.step & 1, ds_parity = st.step >> 1 & 1;
        const uint32_t ds = dsfull + 8 * parity, dp_next = dpfull + 8 * (parity ^ 1);
        const int oa = st.sa, ob = st.sb, sums = (rows + 15) / 16;
        const uint32_t a = ra + oa * F::TILE, b = rb + ob * F::TILE;
        work.next();
        rows = work.rows();
        if (++st.sa == F::SA) { st.sa = 0; st.pa ^= 1; }
        if (++st.sb == F::SB) { st.sb = 0; st.pb ^= 1; }
        const uint32_t a1 = ra + st.sa * F::TILE, b1 = rb + st.sb * F::TILE;
        if (KEYS) {
            if (!(more ? waits.two(pfull, parity, afull + 8 * st.sa, st.pa) : waits.one(pfull, parity))) return false;
            if (more) clean_a();
            ptx::tc_fence_after();
            if (leader) {
                mma_sum<DP, 32, 32>(tmem + COL_SUM_B, tmem + COL_S, to_sum(b), sums, j > 0);
                ptx::mma_commit(bempty + 8 * ob);
                if (more) {                                         // over the P that the product in front of it has read by then
                    mma_rows<DP>(tmem + COL_S, by_rows(fixed), by_rows(a1));
                    ptx::mma_commit(sfull);
                }
            }
            __syncwarp();
            if (!(more ? waits.two(ds, ds_parity, bfull + 8 * st.sb, st.pb) : waits.one(ds, ds_parity))) return false;
            if (more) clean_b();
        } else {
            if (more) {
                if (!waits.three(pfull, parity, afull + 8 * st.sa, st.pa, bfull + 8 * st.sb, st.pb)) return false;
                clean_a();
                ptx::tc_fence_after();
                if (leader) {
                    mma_rows<DP>(tmem + COL_S, by_rows(fixed), by_rows(a1));
                    ptx::mma_commit(sfull);
                    mma_rows<DP>(tmem + dp_column<KEYS>(j + 1), by_rows(fixed + F::TILE), by_rows(b1));
                    ptx::mma_commit(dp_next);
                    ptx::mma_commit(bempty + 8 * st.sb);
                }
                __syncwarp();
            }
            if (!(more ? waits.one(ds, ds_parity) : waits.two(pfull, parity, ds, ds_parity))) return false;
        }
        ptx::tc_fence_after();
        if (leader) {
            mma_sum<DP, 32, 32>(tmem + COL_SUM_A, tmem + dp_column<KEYS>(j), to_sum(a), sums, j > 0);
            ptx::mma_commit(aempty + 8 * oa);
            if (KEYS && more) {
                mma_rows<DP>(tmem + COL_DP, by_rows(fixed + F::TILE), by_rows(b1));
                ptx::mma_commit(dp_next);
            }
            if (!more) ptx::mma_commit(ptx::smem_u32(&ctl->done));
        }
        __syncwarp();
    }
    ++st.tile;
    return true;
}

// What a warp that turns S into dS carries from tile to tile.
struct Slopes {
    uint32_t tmem;
    uint32_t step = 0, of_keys = 0, tile = 0;    // steps, those of tiles of keys, tiles
};

template <int DP, bool KEYS>
__device__ __forceinline__ bool turn(const BackwardParams& p, const Shared<DP>& x, const Waits& waits, Slopes& st, Work& work, int warp,
                                     int lane) {
    using F = Backward<DP>;
    constexpr int WARPS = F::WARPS;
    BackwardCtl* const ctl = x.ctl;
    auto wait = [&](uint64_t& bar, uint32_t parity) { return waits.one(ptx::smem_u32(&bar), parity); };
    const int part = warp >> 2, quad = warp & 3, r = quad * 32 + lane, c0 = part * 32;
    const uint32_t lanes = st.tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const int tile = work.tile, begin = work.sequence.begin, length = work.sequence.length;
    const int row = tile * ROWS + r;                                // in the sequence
    const long long token = begin + row;
    const uint64_t scale = both(p.scale * kLog2e);
    const int owners = KEYS ? p.kv_heads : p.heads, steps = work.count;
    if (steps == 0) return true;
    uint64_t lse = 0, delta = 0;                                    // negative, of the row
    if (!KEYS && row < length) {
        lse = both(-p.lse[static_cast<long long>(work.owner) * p.tokens + token] * kLog2e);
        delta = both(-p.delta[static_cast<long long>(work.owner) * p.tokens + token]);
    }
    // KEYS: negative lse (first 128 threads) or delta (the next) of a query of a step
    auto stat = [&] {
        const int q = work.at * ROWS + r;
        if (q >= length || part >= 2) return 0.0f;
        const long long from = static_cast<long long>(work.head) * p.tokens + begin + q;
        return part == 0 ? -p.lse[from] * kLog2e : -p.delta[from];
    };
    float ahead = KEYS ? stat() : 0.0f;
    for (int j = 0; j < steps; ++j, ++st.step) {
        const uint32_t slot = st.of_keys & 1, parity = st.step & 1;
        const ulonglong2* sl = reinterpret_cast<const ulonglong2*>(x.stats + slot * 2 * ROWS + c0);
        const ulonglong2* sd = sl + ROWS / 4;
        const int at = work.at, rows = work.rows();
        work.next();
        if (KEYS) {
            if (part < 2) x.stats[slot * 2 * ROWS + part * ROWS + r] = ahead;
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->stats[slot]));
            if (j + 1 < steps) ahead = stat();
            // all warps' (a barrier whose wait is bounded); they have left the step before by then
            if (!wait(ctl->stats[slot], (st.of_keys >> 1) & 1)) return false;
            ++st.of_keys;
        }
        // which columns of this thread count: from `from` on (KEYS) up to `to`
        int from = 0, to = 32;
        if (KEYS) {
            if (at == tile) from = r - c0;
            to = rows - c0;
        } else if (at == tile) {
            to = r + 1 - c0;
        }
        const bool all = __all_sync(0xffffffffu, from <= 0 && to >= 32);
        auto put = [&](uint32_t column, float (&v)[32], uint64_t& bar) {
            if (!all) {
#pragma unroll
                for (int c = 0; c < 32; ++c) v[c] = c >= from && c < to ? v[c] : 0.0f;
            }
            uint32_t w[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) w[c] = pack2(v[2 * c], v[2 * c + 1]);
            ptx::tmem_st16(lanes + column + c0, w);
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&bar));
        };
        if (!wait(ctl->sfull, parity)) return false;
        ptx::tc_fence_after();
        uint32_t s[32];
        ptx::tmem_ld32(lanes + COL_S + c0, s);
        if (!KEYS) {
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->pfull));
        }
        float v[32];
#pragma unroll
        for (int c = 0; c < 32; c += 4) {
            const ulonglong2 l = KEYS ? sl[c / 4] : make_ulonglong2(lse, lse);
#pragma unroll
            for (int e = c; e < c + 4; e += 2) {
                split(fma2(f32x2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), scale, e == c ? l.x : l.y), v[e], v[e + 1]);
                v[e] = ex2(v[e]);
                v[e + 1] = ex2(v[e + 1]);
            }
        }
        if (KEYS) put(COL_S, v, ctl->pfull);
        if (!wait(ctl->dpfull[parity], st.step >> 1 & 1)) return false;
        ptx::tc_fence_after();
        ptx::tmem_ld32(lanes + dp_column<KEYS>(j) + c0, s);
#pragma unroll
        for (int c = 0; c < 32; c += 4) {
            const ulonglong2 d = KEYS ? sd[c / 4] : make_ulonglong2(delta, delta);
#pragma unroll
            for (int e = c; e < c + 4; e += 2)
                split(mul2(f32x2(v[e], v[e + 1]), add2(f32x2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), e == c ? d.x : d.y)),
                      v[e], v[e + 1]);
        }
        put(dp_column<KEYS>(j), v, ctl->dsfull[parity]);            // what does not count may be infinite or NaN
    }
    if (!wait(ctl->done, st.tile & 1)) return false;
    ++st.tile;
    ptx::tc_fence_after();
    // KEYS: the first half of the threads has dV, the second dK; otherwise all have dQ
    constexpr int PARTS = KEYS ? WARPS / 8 : WARPS / 4, WIDTH = DP / PARTS;
    const bool first = KEYS && part < PARTS;
    const uint32_t src = lanes + (first ? COL_SUM_B : COL_SUM_A);
    const float factor = first ? 1.0f : p.scale;
    const int o0 = part % PARTS * WIDTH;
    uint4 w[WIDTH / 8];
#pragma unroll
    for (int c = 0; c < WIDTH; c += 16) {
        float o[16];
        ptx::tmem_ld16(src + o0 + c, o);
        if (p.split > 1) {                                          // the tiles are no longer read
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<float4*>(x.smem + sum_at<DP>(first, r, (o0 + c) / 4 + e)) =
                    make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
            w[c / 8 + e] = make_uint4(pack2(o[8 * e] * factor, o[8 * e + 1] * factor), pack2(o[8 * e + 2] * factor, o[8 * e + 3] * factor),
                                      pack2(o[8 * e + 4] * factor, o[8 * e + 5] * factor),
                                      pack2(o[8 * e + 6] * factor, o[8 * e + 7] * factor));
    }
    ptx::tc_fence_before();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->read));
    if (p.split > 1) return true;
    bf16* const out = (KEYS ? first ? p.dv : p.dk : p.dq) + ((token - lane) * owners + work.owner) * p.dim + o0;
    store_rows(w, reinterpret_cast<uint8_t*>(out), static_cast<long long>(owners) * p.dim * 2, length - (row - lane),
               (p.dim - o0) * 2, lane);
    return true;
}

template <int DP> __global__ void __launch_bounds__(Backward<DP>::THREADS, 1) k_attention_grad(const __grid_constant__ BackwardParams p) {
    using F = Backward<DP>;
    constexpr int WARPS = F::WARPS;
    static_assert(sizeof(BackwardCtl) <= F::CTL, "the barriers fit");
    extern __shared__ __align__(1024) uint8_t smem[];              // there is no room to align it here
    const Shared<DP> x(smem);
    BackwardCtl* const ctl = x.ctl;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &ctl->abort;
    if ((ptx::smem_u32(smem) & 1023u) != 0) {                       // the same in every CTA
        if (threadIdx.x == 0) atomicCAS(p.status, 0, MOARA_ERR_ALIGN);
        return;
    }
    // copies of a tile of 128 tokens, of the next step, and of what a tile keeps
    auto copy = [&](uint8_t* to, const CUtensorMap* map, uint64_t& bar, int h, int row) {
        for (int c = 0; c < DP / 64; ++c)
            ptx::tma_load_3d(ptx::smem_u32(to) + c * PANEL, map, ptx::smem_u32(&bar), c * 64, h, row);
    };
    auto copy_a = [&](const Work& w, int slot) {
        ptx::mbar_arrive_expect_tx(ptx::smem_u32(&ctl->afull[slot]), F::TILE);
        copy(x.ring_a + slot * F::TILE, w.keys ? &p.q : &p.k, ctl->afull[slot], w.head, w.sequence.begin + w.at * ROWS);
    };
    auto copy_b = [&](const Work& w, int slot) {
        ptx::mbar_arrive_expect_tx(ptx::smem_u32(&ctl->bfull[slot]), F::TILE);
        copy(x.ring_b + slot * F::TILE, w.keys ? &p.dout : &p.v, ctl->bfull[slot], w.head, w.sequence.begin + w.at * ROWS);
    };
    auto copy_fixed = [&](const Work& w) {
        ptx::mbar_arrive_expect_tx(ptx::smem_u32(&ctl->fixed), 2 * F::TILE);
        copy(x.smem, w.keys ? &p.k : &p.q, ctl->fixed, w.owner, w.token());
        copy(x.smem + F::TILE, w.keys ? &p.v : &p.dout, ctl->fixed, w.owner, w.token());
    };
    if (threadIdx.x == WARPS * 32) {
        // the thread that copies starts what the first step needs beside the others' set-up
        for (uint64_t* b : {&ctl->fixed, &ctl->sfull, &ctl->dpfull[0], &ctl->dpfull[1], &ctl->done, &ctl->drain})
            ptx::mbar_init(ptx::smem_u32(b), 1);
        for (uint64_t* b : {&ctl->pfull, &ctl->dsfull[0], &ctl->dsfull[1], &ctl->stats[0], &ctl->stats[1], &ctl->read})
            ptx::mbar_init(ptx::smem_u32(b), WARPS);
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl->listed[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->taken[i]), WARPS + 1);
        }
        for (int i = 0; i < F::SA; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl->afull[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->aempty[i]), 1);
        }
        for (int i = 0; i < F::SB; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl->bfull[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl->bempty[i]), 1);
        }
        ctl->abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
        pdl_begin();
        ctl->tiles[0] = blockIdx.x / p.split;
        ptx::mbar_arrive(ptx::smem_u32(&ctl->listed[0]));
        Work work;
        if (work.get(p, blockIdx.x / p.split) && work.count > 0) {
            copy_fixed(work);
            copy_a(work, 0);
            copy_b(work, 0);
        }
    }
    if (warp == WARPS + 1) {
        ptx::tmem_alloc(ptx::smem_u32(&ctl->tmem), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    pdl_begin();
    const Waits waits{abort_flag, p.status, p.wait_limit};
    // the CTA's tile of a round, to every warp but the one that copies
    auto tile_of = [&](int round, Work& work, bool& ok) {
        const int slot = round & 1;
        ok = waits.one(ptx::smem_u32(&ctl->listed[slot]), (round >> 1) & 1);
        if (!ok) return false;
        const int n = ctl->tiles[slot];
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl->taken[slot]));
        return work.get(p, n);
    };

    if (warp == WARPS) {
        if (lane == 0) {
            int na = 0, nb = 0, tiles = 0;
            auto room = [&](uint64_t& bar, int n, int slots) {
                return n < slots || ptx::mbar_wait(ptx::smem_u32(&bar), (n / slots - 1) & 1, abort_flag, p.status,
                                                   MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit);
            };
            Work work;
            bool ok = true;
            int n = blockIdx.x / p.split;
            for (int round = 0; ok && work.get(p, n); ++round) {
                if (round == 0 && work.count > 0) {                 // begun above
                    na = nb = tiles = 1;
                    work.next();
                }
                for (int j = round == 0; j < work.count; ++j, work.next()) {
                    ok = room(ctl->aempty[na % F::SA], na, F::SA);
                    if (!ok) break;
                    copy_a(work, na++ % F::SA);
                    ok = room(ctl->bempty[nb % F::SB], nb, F::SB);
                    if (!ok) break;
                    copy_b(work, nb++ % F::SB);
                    if (j > 0) continue;
                    // the last tile's products are done
                    ok = ptx::mbar_wait(ptx::smem_u32(&ctl->done), (tiles - 1) & 1, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT,
                                        p.wait_limit);
                    if (!ok) break;
                    copy_fixed(work);
                    ++tiles;
                }
                if (!ok) break;
                // the next tile; a cluster has one
                n = p.split > 1 ? INT_MAX : static_cast<int>(gridDim.x + atomicAdd(p.counter, 1u));
                const int slot = (round + 1) & 1;
                ok = round == 0 || ptx::mbar_wait(ptx::smem_u32(&ctl->taken[slot]), ((round - 1) >> 1) & 1, abort_flag, p.status,
                                                  MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit);
                if (!ok) break;
                ctl->tiles[slot] = n;
                ptx::mbar_arrive(ptx::smem_u32(&ctl->listed[slot]));
            }
            ctl->filled[0] = na;
            ctl->filled[1] = nb;
            ctl->filled[2] = tiles;
        }
    } else if (warp == WARPS + 1) {
        // The whole warp runs the loop, one lane issues (a lane alone takes 1650 clocks for sixteen
        // products, whose time is 1030); what a product needs but P and dS is there ahead of them.
        const bool leader = ptx::elect_one();
        Products st;
        st.tmem = tmem;
        Work work;
        bool ok = true;
        for (int round = 0; ok && tile_of(round, work, ok); ++round)
            ok = work.keys ? multiply<DP, true>(x, waits, st, work, leader, lane) : multiply<DP, false>(x, waits, st, work, leader, lane);
        if (leader) ptx::mma_commit(ptx::smem_u32(&ctl->drain));
        __syncwarp();
        wait_drain(ptx::smem_u32(&ctl->drain), 0);
    } else {
        Slopes st;
        st.tmem = tmem;
        Work work;
        bool ok = true;
        for (int round = 0; ok && tile_of(round, work, ok); ++round)
            ok = work.keys ? turn<DP, true>(p, x, waits, st, work, warp, lane) : turn<DP, false>(p, x, waits, st, work, warp, lane);
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) {      // a wait that ran out: no copy stays in flight
        if (ctl->filled[2] > 0) wait_drain(ptx::smem_u32(&ctl->fixed), (ctl->filled[2] - 1) & 1);
        for (int n = max(0, ctl->filled[0] - F::SA); n < ctl->filled[0]; ++n)
            wait_drain(ptx::smem_u32(&ctl->afull[n % F::SA]), (n / F::SA) & 1);
        for (int n = max(0, ctl->filled[1] - F::SB); n < ctl->filled[1]; ++n)
            wait_drain(ptx::smem_u32(&ctl->bfull[n % F::SB]), (n / F::SB) & 1);
    }
    if (warp == WARPS + 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
    __syncthreads();
    if (p.split == 1) return;
    // a cluster has one tile
    ptx::cluster_sync();                         // every CTA's sums are in its shared memory
    const bool gave_up =
        lane < p.split && ptx::ld_cluster_u32(ptx::mapa(ptx::smem_u32(&ctl->abort), static_cast<uint32_t>(lane))) != 0;
    Work work;
    if (work.get(p, blockIdx.x / p.split) && !__any_sync(0xffffffffu, gave_up)) {
        // a share of the rows each; ranks behind the last step have none
        const int ranks = min(p.split, work.all), rank = blockIdx.x % p.split, owners = work.keys ? p.kv_heads : p.heads;
        const int share = ROWS / p.split, chunks = DP / 8;
        for (int n = threadIdx.x; n < (work.keys ? 2 : 1) * share * chunks; n += blockDim.x) {
            const int c = n % chunks, row = rank * share + n / chunks % share, which = n / (chunks * share);
            float o[8] = {};
            for (int k = 0; k < ranks; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float4 v = ld_cluster_f4(ptx::mapa(ptx::smem_u32(smem + sum_at<DP>(which, row, 2 * c + e)), k));
                    o[4 * e] += v.x; o[4 * e + 1] += v.y; o[4 * e + 2] += v.z; o[4 * e + 3] += v.w;
                }
            if (work.tile * ROWS + row >= work.sequence.length || 8 * c >= p.dim) continue;
            const float factor = which != 0 ? 1.0f : p.scale;
            bf16* out = (which != 0 ? p.dv : work.keys ? p.dk : p.dq) +
                        (static_cast<long long>(work.token() + row) * owners + work.owner) * p.dim + 8 * c;
            *reinterpret_cast<uint4*>(out) = make_uint4(pack2(o[0] * factor, o[1] * factor), pack2(o[2] * factor, o[3] * factor),
                                                        pack2(o[4] * factor, o[5] * factor), pack2(o[6] * factor, o[7] * factor));
        }
    }
    __syncwarp();
    ptx::cluster_sync();                         // no CTA leaves while another reads its sums
}

struct DeltaParams {
    const bf16* dout;
    const bf16* out;
    const bf16* rest;
    float* delta;
    unsigned int* counter;                       // of the next launch, set to zero
    long long row, head;                         // pitches of dO
    int tokens, heads, dim;
};

// delta = rowsum(dO O), with what the rounding of O dropped where it was kept: an error of
// delta is the same for all keys of a row, and where keys share a direction dQ's error would
// grow with their number (1024 keys: 0.45% of dQ's norm with O alone, 0.25% so).  16 lanes a
// row, heads of a token beside one another.
__global__ void __launch_bounds__(256) k_attention_delta(const DeltaParams p) {
    pdl_begin();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.counter = 0;
    const long long n = static_cast<long long>(blockIdx.x) * 16 + (threadIdx.x >> 4);
    const int c = (threadIdx.x & 15) * 8;
    const long long token = n / p.heads;
    const int head = static_cast<int>(n % p.heads);
    float sum = 0.0f;
    if (token < p.tokens && c < p.dim) {
        const long long at = n * p.dim + c;
        const uint4 a = *reinterpret_cast<const uint4*>(p.dout + token * p.row + head * p.head + c);
        const uint4 b = *reinterpret_cast<const uint4*>(p.out + at);
        const uint4 l = p.rest == nullptr ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(p.rest + at);
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w}, z[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16) + __uint_as_float(z[e] << 16), sum);
            sum = fmaf(__uint_as_float(x[e] & 0xFFFF0000u),
                       __uint_as_float(y[e] & 0xFFFF0000u) + __uint_as_float(z[e] & 0xFFFF0000u), sum);
        }
    }
#pragma unroll
    for (int o = 8; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (token < p.tokens && (threadIdx.x & 15) == 0) p.delta[static_cast<long long>(head) * p.tokens + token] = sum;
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

// 128 tokens of a head, 64 entries at a time; entries behind the head's last and tokens
// behind the tensor's last are zeros.
bool encode(CUtensorMap* map, const void* x, int tokens, int heads, int dim, int64_t row, int64_t head) {
    EncodeTiledFn fn = encoder();
    if (fn == nullptr) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(head) * 2, static_cast<cuuint64_t>(row) * 2};
    const cuuint32_t box[3] = {64, 1, ROWS}, estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(x), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Lets a kernel take `bytes` of shared memory: once per device.
template <int ID, class... P> cudaError_t allow_shared(void (*fn)(P...), int bytes) {
    static std::atomic<uint64_t> done{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess || (device < 64 && (done.load() >> device & 1))) return e;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && device < 64) done.fetch_or(1ull << device);
    return e;
}

// A pair a CTA where all of them run at once, or where a pair's steps are many: the loop around them
// costs each some 150 clocks, and what it hides is a pair's first copies and last stores (16384
// tokens, 28 heads of 128: 5% longer with the loop; 32 x 512, 16 heads of 128: 77 and 67; the same at 16 steps a
// pair, of heads of 64 at 32).
template <int DP> cudaError_t forward_as(const ForwardParams& p, int ctas, long long steps, cudaStream_t s) {
    const bool one = ctas <= 152 || steps * DP > 2048LL * ctas;
    const auto fn = one ? k_attention<DP, true> : k_attention<DP, false>;
    const cudaError_t e = one ? allow_shared<DP>(fn, Forward<DP>::SMEM) : allow_shared<DP + 1>(fn, Forward<DP>::SMEM);
    if (e != cudaSuccess) return e;
    return launch(fn, dim3(ctas), dim3(Forward<DP>::THREADS), Forward<DP>::SMEM, s, 1, p);
}

template <int DP> cudaError_t backward_as(const BackwardParams& p, cudaStream_t s) {
    const cudaError_t e = allow_shared<DP>(k_attention_grad<DP>, Backward<DP>::SMEM);
    if (e != cudaSuccess) return e;
    // a CTA an SM, or a cluster a tile
    const unsigned int tiles = static_cast<unsigned int>(p.n_tiles) * (p.kv_heads + p.heads);
    const unsigned int ctas = p.split > 1 ? tiles * p.split : std::min(tiles, 152u);
    return launch(k_attention_grad<DP>, dim3(ctas), dim3(Backward<DP>::THREADS), Backward<DP>::SMEM, s, p.split, p);
}

}  // namespace

cudaError_t launch_attention(const Attention& a, cudaStream_t s, int64_t* launches) {
    ForwardParams p{};
    if (!encode(&p.q, a.q, a.tokens, a.heads, a.dim, a.q_row, a.q_head) ||
        !encode(&p.k, a.k, a.tokens, a.kv_heads, a.dim, a.k_row, a.k_head) ||
        !encode(&p.v, a.v, a.tokens, a.kv_heads, a.dim, a.v_row, a.v_head))
        return cudaErrorInvalidValue;
    p.out = static_cast<bf16*>(a.out);
    p.rest = static_cast<bf16*>(a.rest);
    p.lse = a.lse;
    p.pairs = a.pairs;
    p.tokens = a.tokens;
    p.heads = a.heads;
    p.group = a.heads / a.kv_heads;
    p.dim = a.dim;
    p.scale = a.scale;
    p.scale2 = a.scale * kLog2e;
    p.status = a.status;
    p.wait_limit = a.wait_limit;
    ++*launches;
    const int ctas = a.n_pairs * a.heads;
    const long long steps = a.work / 2 * a.heads;                  // two tiles of queries share a step
    return a.dim <= 64 ? forward_as<64>(p, ctas, steps, s) : forward_as<128>(p, ctas, steps, s);
}

cudaError_t launch_attention_backward(const AttentionGrad& a, cudaStream_t s, int64_t* launches) {
    BackwardParams p{};
    if (!encode(&p.q, a.q, a.tokens, a.heads, a.dim, a.q_row, a.q_head) ||
        !encode(&p.k, a.k, a.tokens, a.kv_heads, a.dim, a.k_row, a.k_head) ||
        !encode(&p.v, a.v, a.tokens, a.kv_heads, a.dim, a.v_row, a.v_head) ||
        !encode(&p.dout, a.dout, a.tokens, a.heads, a.dim, a.do_row, a.do_head))
        return cudaErrorInvalidValue;
    const DeltaParams d{static_cast<const bf16*>(a.dout), static_cast<const bf16*>(a.out), static_cast<const bf16*>(a.rest),
                        a.delta, reinterpret_cast<unsigned int*>(a.delta + static_cast<long long>(a.tokens) * a.heads),
                        a.do_row, a.do_head, a.tokens, a.heads, a.dim};
    const long long rows = static_cast<long long>(a.tokens) * a.heads;
    p.counter = d.counter;
    ++*launches;
    cudaError_t e = launch(k_attention_delta, dim3(static_cast<unsigned int>((rows - 1) / 16 + 1)), dim3(256), 0, s, 1, d);
    if (e != cudaSuccess) return e;
    p.lse = a.lse;
    p.delta = a.delta;
    p.dq = static_cast<bf16*>(a.dq);
    p.dk = static_cast<bf16*>(a.dk);
    p.dv = static_cast<bf16*>(a.dv);
    p.tiles = a.tiles;
    p.n_tiles = a.n_tiles;
    p.tokens = a.tokens;
    p.heads = a.heads;
    p.kv_heads = a.kv_heads;
    p.group = a.heads / a.kv_heads;
    p.dim = a.dim;
    p.scale = a.scale;
    p.status = a.status;
    p.wait_limit = a.wait_limit;
    // clusters share a tile while the longest would outlast an SM's share of all steps, and has
    // more than eight
    const long long longest = static_cast<long long>(a.longest) * p.group, most = std::max<long long>(8, 2 * a.work * a.heads / 152);
    p.split = 1;
    while (p.split < 8 && longest > most * p.split) p.split *= 2;
    ++*launches;
    return a.dim <= 64 ? backward_as<64>(p, s) : backward_as<128>(p, s);
}

}  // namespace moara
