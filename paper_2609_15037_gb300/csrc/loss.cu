// Clipped policy loss of a batch of tokens from their logits, with its gradient.
//   lp = z_a - log sum_j exp z_j, rho = exp(lp - old), x = ref - lp
//   loss = -min(rho A, clamp(rho, low, high) A) + kl (exp x - x - 1)
//   dz_j = g (1[j = a] - exp(z_j) / sum),   g = w (kl (1 - exp x) - [not clipped] rho A)
// DRAM-bound: the logits are read once and their gradient written once.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cstddef>

#include "f32x2.cuh"
#include "launch.cuh"
#include "layers.h"
#include "tc_ptx.cuh"
#include "waits.cuh"

namespace moara {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718f, kLn2Rest = -1.90465421e-9f;      // ln 2 in two fp32 numbers

struct LossParams {
    const void* z;
    void* dz;
    const int64_t* target;
    const float* old_logp;
    const float* ref_logp;
    const float* adv;
    const float* weight;
    float* logp;
    float2* terms;
    long long ldz, lddz;
    int rows, vocab, part, split;
    float low, high, kl, mean;     // mean: weight of a token where none are given
    int* status;
    long long wait_limit;
};

// exp(x) - x - 1 without the cancellation of small x: there its Taylor series, whose
// terms behind x^9 are below 2^-24 of the first for |x| <= 1/2.
__device__ __forceinline__ float exp_beyond_linear(float x) {
    if (fabsf(x) > 0.5f) return expm1f(x) - x;
    float s = 1.0f / 362880;
    s = fmaf(s, x, 1.0f / 40320);
    s = fmaf(s, x, 1.0f / 5040);
    s = fmaf(s, x, 1.0f / 720);
    s = fmaf(s, x, 1.0f / 120);
    s = fmaf(s, x, 1.0f / 24);
    s = fmaf(s, x, 1.0f / 6);
    s = fmaf(s, x, 0.5f);
    return s * x * x;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A sum held in two fp32 numbers: what an addition rounds off goes to the second.
struct Sum {
    float hi = 0.0f, lo = 0.0f;
    __device__ __forceinline__ void add(float x) {
        const float s = hi + x, b = s - hi;
        lo += (hi - (s - b)) + (x - b);
        hi = s;
    }
    // - x ln 2
    __device__ __forceinline__ void subtract_ln2(float x) {
        const float y = x * kLn2;
        add(-y);
        lo -= fmaf(x, kLn2, -y) + x * kLn2Rest;
    }
    // beside an infinite sum there is NaN
    __device__ __forceinline__ float value() const { return fabsf(hi) < INFINITY ? hi + lo : hi; }
    __device__ __forceinline__ float minus(float x) const {
        Sum s = *this;
        s.add(-x);
        return s.value();
    }
};

// 16 bytes of a row as fp32, their largest (NaN left out: it returns in the sum), and
// exponentials relative to a reference logit: powers of two of (z - ref) log2 e, which no size of the
// logits takes out of fp32's range but where the exponential is zero.  bf16 logits leave out what the two
// operations round off, an error far below the gradient's rounding; fp32 logits take what the product
// rounds off as a factor (1 + its natural power).
template <class T> struct Line;

template <> struct Line<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float top(const uint4& w) {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    static __device__ __forceinline__ float exponential(float z, float ref) {
        const float t = z - ref, x = t * kLog2e, y = ex2(x);
        // of minus infinity the rest is NaN: its exponential is 0 whatever it is
        const float rest = x == -INFINITY ? 0.0f : fmaf(t, kLog2e, -x);
        return fmaf(y, rest * 0.69314718f, y);
    }
    static __device__ __forceinline__ void exponentials(const uint4& w, float ref, float (&e)[4]) {
        e[0] = exponential(__uint_as_float(w.x), ref);
        e[1] = exponential(__uint_as_float(w.y), ref);
        e[2] = exponential(__uint_as_float(w.z), ref);
        e[3] = exponential(__uint_as_float(w.w), ref);
    }
    static __device__ __forceinline__ float apart(float x) { return expf(x); }      // of a difference of references
    static __device__ __forceinline__ uint4 pack(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    static __device__ __forceinline__ float rounded(float x) { return x; }
};

template <> struct Line<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t y;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
        return y;
    }
    static __device__ __forceinline__ float top(const uint4& w) {
        const uint32_t t = max2(max2(w.x, w.y), max2(w.z, w.w));
        return fmaxf(__uint_as_float(t << 16), __uint_as_float(t & 0xFFFF0000u));
    }
    static __device__ __forceinline__ float exponential(float z, float ref) { return ex2((z - ref) * kLog2e); }
    static __device__ __forceinline__ void exponentials(const uint4& w, float ref, float (&e)[8]) {
        const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            split(mul2(add2(widen2(a[k]), both(-ref)), both(kLog2e)), e[2 * k], e[2 * k + 1]);
            e[2 * k] = ex2(e[2 * k]);
            e[2 * k + 1] = ex2(e[2 * k + 1]);
        }
    }
    static __device__ __forceinline__ float apart(float x) { return ex2(x * kLog2e); }
    static __device__ __forceinline__ uint32_t pack2(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float (&v)[8]) {
        return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    }
    static __device__ __forceinline__ __nv_bfloat16 rounded(float x) { return __float2bfloat16_rn(x); }
};

constexpr int kLossThreads = 384;
constexpr int kChunks = 4;             // of a part, copied apart
constexpr int kElsewhere = -1, kUncounted = -2;

struct LossCtl {
    uint64_t full[kChunks];
    int abort;
    float top, sum, at;            // of this CTA's part: reference, sum, the target's logit if it is here
    float factor, gain;            // of the gradient
    int hit;                       // the target's entry of this part, kElsewhere, or kUncounted: the token counts for nothing
    float2 part[2][16];            // of the warps: reference, sum
};

// A wait for a copy.  POLLED: for bounds that the hardware may outlast within one try, by tries that do not wait
// (in one kernel with the others it took 186 us where this takes 179).
template <bool POLLED> __device__ __forceinline__ bool landed(uint32_t bar, uint32_t parity, volatile int* abort_flag, const LossParams& p) {
    if (!POLLED) return ptx::mbar_wait(bar, parity, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit);
    for (const long long t0 = clock64(); !ptx::mbar_test_wait(bar, parity);) {
        if (*abort_flag) return false;
        if (clock64() - t0 > p.wait_limit) {
            *abort_flag = 1;
            atomicCAS(p.status, 0, MOARA_ERR_DEVICE_TIMEOUT);
            return false;
        }
    }
    return true;
}

__device__ __forceinline__ float ld_cluster_f32(uint32_t a) { return __uint_as_float(ptx::ld_cluster_u32(a)); }

// A cluster of `split` CTAs takes rows a grid apart, each CTA a part of their columns, whose
// whole 16-byte lines bulk copies put into shared memory, in the row's own alignment, in four
// chunks; the next row's copy of a chunk begins as soon as this row's gradient has been taken from it.
// What lies in front of the first and behind the last whole line is read where it lies, an entry a
// thread.  A thread's sum is relative to the largest logit that it has met, or one that is at most
// 8 below it, so that the row is read twice, not three times.  !STAGED: a part that is too large for
// shared memory is read again from L2.  8192 x 32000 bf16: 175 to 178 us (floor 155), without the gradient 119 (floor 77: a row's
// next copies wait for its sums).
template <class T, bool STAGED, bool POLLED>
__global__ void __launch_bounds__(kLossThreads, 3) k_policy_loss(const __grid_constant__ LossParams p) {
    extern __shared__ __align__(16) uint8_t raw[];
    using L = Line<T>;
    constexpr int N = L::N;
    __shared__ LossCtl ctl;
    const int rank = blockIdx.x % p.split, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int first = rank * p.part, len = max(0, min(p.vocab - first, p.part));
    volatile int* abort_flag = &ctl.abort;
    if (threadIdx.x == 0) {
        ctl.abort = 0;
        if (STAGED) {
            for (int c = 0; c < kChunks; ++c) ptx::mbar_init(ptx::smem_u32(&ctl.full[c]), 1);
            ptx::fence_barrier_init();
            ptx::fence_proxy_async_smem();
        }
    }
    __syncthreads();
    pdl_begin();
    const uint32_t full = ptx::smem_u32(&ctl.full[0]), own = ptx::smem_u32(&ctl);
    const long long step = gridDim.x / p.split;
    const int chunk = (p.part / N + kChunks) / kChunks;          // lines
    // a row's part: its entries in front of the first whole line, and the whole lines
    struct Place {
        const T* z;
        int front, lines;
    };
    auto place = [&](long long row) {
        Place x;
        x.z = static_cast<const T*>(p.z) + row * p.ldz + first;
        x.front = min(len, static_cast<int>(-reinterpret_cast<uintptr_t>(x.z) & 15) / static_cast<int>(sizeof(T)));
        x.lines = (len - x.front) / N;
        return x;
    };
    // an empty chunk's phase ends all the same
    auto copy = [&](const Place& x, int c) {
        const int from = c * chunk, to = min(x.lines, (c + 1) * chunk);
        const uint32_t bytes = to > from ? (to - from) * 16u : 0u;
        ptx::mbar_arrive_expect_tx(full + 8 * c, bytes);
        for (uint32_t at = 0; at < bytes; at += 16384)
            ptx::bulk_load(ptx::smem_u32(raw) + from * 16 + at, reinterpret_cast<const uint8_t*>(x.z + x.front) + from * 16ll + at,
                           min(16384u, bytes - at), full + 8 * c);
    };
    long long row = blockIdx.x / p.split;
    Place x = place(row);
    if (STAGED && threadIdx.x == 0)
        for (int c = 0; c < kChunks; ++c) copy(x, c);
    uint32_t phase = 0;
    Sum sums[3];                                 // of the first thread: loss, KL term, clipped
    for (; row < p.rows; row += step, phase ^= 1) {
        const bool more = row + step < p.rows;
        const uint4* const lines = STAGED ? reinterpret_cast<const uint4*>(raw) : reinterpret_cast<const uint4*>(x.z + x.front);
        // the entry beside the lines that this thread has, or -1
        int beside = static_cast<int>(threadIdx.x);
        if (beside >= x.front) beside += x.lines * N;
        if (beside >= len) beside = -1;
        // what the first thread needs of the token, fetched beside the row
        int64_t target = 0;
        float w = 0.0f, a = 0.0f, old = 0.0f, other = 0.0f;
        if (threadIdx.x == 0) {
            target = p.target[row];
            w = p.weight != nullptr ? p.weight[row] : p.mean;
            a = p.adv[row];
            old = p.old_logp[row];
            if (p.ref_logp != nullptr) other = p.ref_logp[row];
        }
        // top: the thread's largest logit when its reference was taken
        float top = -INFINITY, ref = 0.0f, sum = 0.0f;
        for (int c = 0; c < kChunks; ++c) {
            if (STAGED && !landed<POLLED>(full + 8 * c, phase, abort_flag, p)) wait_drain(full + 8 * c, phase);
            const int end = min(x.lines, (c + 1) * chunk);
            for (int i = c * chunk + threadIdx.x; i < end; i += blockDim.x) {
                const uint4 v = lines[i];
                const float high = L::top(v);
                if (high > top + 8.0f) {
                    // of a first finite logit: nothing but zeros (or NaN) has been added
                    if (top > -INFINITY) sum = sum * L::apart(top - high);
                    top = high;
                    ref = high;
                }
                float e[N];
                L::exponentials(v, ref, e);
#pragma unroll
                for (int k = N / 2; k > 0; k /= 2)
#pragma unroll
                    for (int y = 0; y < k; ++y) e[y] += e[y + k];
                sum += e[0];
            }
        }
        if (beside >= 0) {
            const float v = static_cast<float>(x.z[beside]);
            if (v > top + 8.0f) {
                if (top > -INFINITY) sum *= L::apart(top - v);
                top = v;
                ref = v;
            }
            sum += L::exponential(v, ref);
        }
        // all threads' relative to their largest reference: within the warp, then the CTA
        auto join = [&](float& top, float& sum, int most) {
            float high = top;
            for (int o = most / 2; o > 0; o /= 2) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
            // what has no finite logit has a sum of 0, or NaN
            sum = top > -INFINITY ? sum * L::apart(top - high) : sum;
            for (int o = most / 2; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            top = high;
        };
        float base = top;
        join(base, sum, 32);
        float2* const part = ctl.part[phase];
        if (lane == 0) part[warp] = make_float2(base, sum);
        __syncthreads();
        {
            const float2 t = lane < warps ? part[lane] : make_float2(-INFINITY, 0.0f);
            base = t.x;
            sum = t.y;
            join(base, sum, 16);
            base = __shfl_sync(0xffffffffu, base, 0);
            sum = __shfl_sync(0xffffffffu, sum, 0);
        }
        const bool ok = *abort_flag == 0;        // the same in every thread: a wait ran out before the barrier above
        const float mine = base == -INFINITY ? 0.0f : base;             // this part's reference
        if (threadIdx.x == 0) {
            const bool counts = target >= 0 && target < p.vocab;
            const int column = counts ? static_cast<int>(target) : 0, owner = column / p.part;
            ctl.top = base;
            ctl.sum = ok ? sum : NAN;
            if (counts && owner == rank) ctl.at = static_cast<float>(x.z[column - first]);
        }
        if (p.split > 1) {
            __syncwarp();
            ptx::cluster_sync();
        }
        if (threadIdx.x == 0) {
            const bool counts = target >= 0 && target < p.vocab;
            const int column = counts ? static_cast<int>(target) : 0, owner = column / p.part;
            float tops[8], parts[8], total = 0.0f, at = 0.0f;
            if (p.split == 1) {
                total = ctl.sum;
                at = ctl.at;
            } else {
                base = -INFINITY;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    if (r >= p.split) break;
                    const uint32_t peer = ptx::mapa(own, r);
                    tops[r] = ld_cluster_f32(peer + static_cast<uint32_t>(offsetof(LossCtl, top)));
                    parts[r] = ld_cluster_f32(peer + static_cast<uint32_t>(offsetof(LossCtl, sum)));
                    base = fmaxf(base, tops[r]);
                }
                at = ld_cluster_f32(ptx::mapa(own, owner) + static_cast<uint32_t>(offsetof(LossCtl, at)));
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    if (r >= p.split) break;
                    total += tops[r] == -INFINITY ? parts[r] : parts[r] * L::apart(tops[r] - base);
                }
            }
            const float base0 = base == -INFINITY ? 0.0f : base;
            // log(total) from its exponent and the rest, which lies in [1, 2)
            Sum lp;
            lp.add(at);
            lp.add(-base0);
            if (total > 0.0f && total < INFINITY) {
                lp.subtract_ln2(static_cast<float>(static_cast<int>(__float_as_uint(total) >> 23) - 127));
                lp.add(-logf(__uint_as_float((__float_as_uint(total) & 0x7FFFFFu) | 0x3F800000u)));
            } else {
                lp.add(-logf(total));                       // without any probability, or not a number
            }
            float gain = 0.0f;
            const bool taken = counts && w != 0.0f;
            if (taken) {
                const float t = lp.minus(old);
                float rho = expf(t);
                // an advantage of zero has no part, whatever the ratio
                if (a == 0.0f && rho == INFINITY) rho = 1.0f;
                // NaN advantages and ratios stay NaN
                const float bound = rho < p.low ? p.low : rho > p.high ? p.high : rho;
                const bool clipped = bound * a < rho * a;
                float loss = clipped ? -bound * a : -rho * a, d = clipped ? 0.0f : -rho * a;
                float y = 0.0f, k = 0.0f, grown = 0.0f;
                if (p.ref_logp != nullptr) {
                    y = -lp.minus(other);
                    k = exp_beyond_linear(y);
                    grown = expm1f(y);
                    loss = fmaf(p.kl, k, loss);
                    d = fmaf(-p.kl, grown, d);
                }
                float term = loss * w, extra = k * w;
                gain = w * d;
                if (rho == INFINITY || grown == INFINITY) {
                    // an exponential beyond fp32's range, whose product need not be: by its root, twice
                    const float r = expf(0.5f * t), g = expf(0.5f * y);
                    term = clipped ? -bound * a * w : rho == INFINITY ? -(w * a) * r * r : -rho * a * w;
                    gain = clipped ? 0.0f : term;
                    if (grown == INFINITY) {
                        extra = w * g * g;
                        term += w * p.kl * g * g;
                        gain -= w * p.kl * g * g;
                    } else if (p.ref_logp != nullptr) {
                        term += p.kl * extra;
                        gain -= w * p.kl * grown;
                    }
                }
                sums[0].add(term);
                if (p.ref_logp != nullptr) sums[1].add(extra);
                if (clipped) sums[2].add(w);
            }
            if (rank == 0) p.logp[row] = counts ? lp.value() : 0.0f;
            ctl.gain = gain;
            // relative to this part's reference
            ctl.factor = -gain * ((ctl.top == -INFINITY ? 1.0f : L::apart(mine - base0)) / total);
            ctl.hit = !taken ? kUncounted : owner == rank ? column - first : kElsewhere;
        }
        if (p.split > 1) {
            __syncwarp();
            ptx::cluster_sync();                 // no CTA goes on while another reads its sums
        } else {
            __syncthreads();
        }
        const float factor = ctl.factor, gain = ctl.gain;
        const int hit = ctl.hit;
        const bool zero = hit == kUncounted, wanted = p.dz != nullptr && ok;
        T* const dz = static_cast<T*>(p.dz) + row * p.lddz + first;
        // whether the gradient's entries lie in lines as the logits' do
        const bool same = (reinterpret_cast<uintptr_t>(dz + x.front) & 15) == 0;
        auto slope = [&](float z) { return zero ? 0.0f : L::exponential(z, mine) * factor; };
        // the target's entry, by the thread that writes its line, read before that is over-written
        const int hit_line = hit >= x.front && hit < x.front + x.lines * N ? (hit - x.front) / N : -1;
        const bool hits = wanted && !zero && (hit_line >= 0 ? hit_line % chunk % blockDim.x == threadIdx.x : hit >= 0 && hit == beside);
        const float hit_value = hits ? slope(static_cast<float>(x.z[hit])) + gain : 0.0f;
        const float beside_value = wanted && beside >= 0 ? slope(static_cast<float>(x.z[beside])) : 0.0f;
        Place next = x;
        if (more) next = place(row + step);
        for (int c = 0; c < kChunks; ++c) {
            const int end = wanted ? min(x.lines, (c + 1) * chunk) : 0;
            uint4* const out = reinterpret_cast<uint4*>(dz + x.front);
            if (zero && same) {
                for (int i = c * chunk + threadIdx.x; i < end; i += blockDim.x) out[i] = make_uint4(0, 0, 0, 0);
            } else if (zero) {
                for (int i = c * chunk + threadIdx.x; i < end; i += blockDim.x)
                    for (int e = 0; e < N; ++e) dz[x.front + i * N + e] = L::rounded(0.0f);
            } else if (same) {
                for (int i = c * chunk + threadIdx.x; i < end; i += blockDim.x) {
                    float e[N];
                    L::exponentials(lines[i], mine, e);
#pragma unroll
                    for (int y = 0; y < N; ++y) e[y] *= factor;
                    out[i] = L::pack(e);
                }
            } else {
                for (int i = c * chunk + threadIdx.x; i < end; i += blockDim.x) {
                    float e[N];
                    L::exponentials(lines[i], mine, e);
#pragma unroll
                    for (int y = 0; y < N; ++y) dz[x.front + i * N + y] = L::rounded(e[y] * factor);
                }
            }
            if (more && STAGED) {
                __syncthreads();                 // the chunk has been read
                if (threadIdx.x == 0) copy(next, c);
            }
        }
        if (wanted && beside >= 0) dz[beside] = L::rounded(beside_value);
        if (hits) dz[hit] = L::rounded(hit_value);
        x = next;
    }
    if (threadIdx.x == 0 && rank == 0)
        for (int k = 0; k < 3; ++k) p.terms[3 * (blockIdx.x / p.split) + k] = make_float2(sums[k].hi, sums[k].lo);
}

// The clusters' sums, added up in a fixed order: at most kLossClusters of them.
constexpr int kLossClusters = 152 * 16;
__global__ void __launch_bounds__(128) k_loss_sums(const float2* terms, int count, float* out) {
    __shared__ float2 part[3][4];
    pdl_begin();
    Sum s[3];
#pragma unroll 4
    for (int r = threadIdx.x; r < count; r += 128)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const float2 t = terms[3 * r + k];
            s[k].add(t.x);
            s[k].lo += t.y;
        }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            const float h = __shfl_down_sync(0xffffffffu, s[k].hi, o), l = __shfl_down_sync(0xffffffffu, s[k].lo, o);
            s[k].add(h);
            s[k].lo += l;
        }
        if (lane == 0) part[k][warp] = make_float2(s[k].hi, s[k].lo);
    }
    __syncthreads();
    if (threadIdx.x >= 3) return;
    Sum all;
    for (int w = 0; w < 4; ++w) {
        all.add(part[threadIdx.x][w].x);
        all.lo += part[threadIdx.x][w].y;
    }
    out[threadIdx.x] = all.value();
}

// Bytes of a row's part, beyond which it is split: the clusters' barriers cost more than a second CTA
// on the SM gives (701 x 50001 fp32: 71 us in two parts, 89 in four)
constexpr int kPart = 112 * 1024;
constexpr int kStage = 200 * 1024;     // most bytes of a part in shared memory

template <class T, bool STAGED, bool POLLED> cudaError_t launch_loss(const LossParams& p, int& clusters, cudaStream_t s) {
    const auto fn = k_policy_loss<T, STAGED, POLLED>;
    const int bytes = STAGED ? (p.part * static_cast<int>(sizeof(T)) + 15) / 16 * 16 + 16 : 0;
    if (bytes > 40 * 1024) {
        static std::atomic<uint64_t> done{0};
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess) return e;
        if (device >= 64 || !(done.load() >> device & 1)) {
            e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kStage + 64);
            if (e != cudaSuccess) return e;
            if (device < 64) done.fetch_or(1ull << device);
        }
    }
    // CTAs that an SM holds by shared memory (1.5 KB beside the part); they share the threads that
    // its registers are enough for
    const int lines = p.part / Line<T>::N + 2, fit = std::max(1, std::min(16, (226 << 10) / (bytes + 1536)));
    const int threads = std::min({kLossThreads, std::max(64, 3 * kLossThreads / fit / 32 * 32), std::max(64, (lines + 31) / 32 * 32)});
    const int resident = std::max(1, std::min(fit, 3 * kLossThreads / threads));
    clusters = std::min(p.rows, 152 * resident / p.split);
    return launch(fn, dim3(static_cast<unsigned int>(clusters) * p.split), dim3(threads), bytes, s, p.split, p);
}

template <class T> cudaError_t loss_as(LossParams& p, int& clusters, cudaStream_t s) {
    constexpr int N = Line<T>::N;
    // a row over more CTAs while they are few, each with some 4 KB and more, and where its part
    // would fill an SM's shared memory alone
    p.split = 1;
    const auto part = [&](int split) { return ((p.vocab - 1) / split + N) / N * N; };
    while (p.split < 8 && (part(p.split) * static_cast<long long>(sizeof(T)) > kPart ||
                           (2LL * p.split * p.rows <= 304 && part(2 * p.split) * sizeof(T) >= 4096)))
        p.split *= 2;
    p.part = part(p.split);
    if (p.part * static_cast<long long>(sizeof(T)) > kStage) return launch_loss<T, false, false>(p, clusters, s);
    return p.wait_limit < 1 << 20 ? launch_loss<T, true, true>(p, clusters, s) : launch_loss<T, true, false>(p, clusters, s);
}

}  // namespace

cudaError_t launch_policy_loss(const PolicyLoss& a, cudaStream_t s, int64_t* launches) {
    LossParams p{};
    p.z = a.z;
    p.dz = a.dz;
    p.target = a.target;
    p.old_logp = a.old_logp;
    p.ref_logp = a.ref_logp;
    p.adv = a.adv;
    p.weight = a.weight;
    p.logp = a.logp;
    p.terms = static_cast<float2*>(a.terms);
    p.ldz = a.ldz;
    p.lddz = a.lddz;
    p.rows = a.rows;
    p.vocab = a.vocab;
    p.low = a.low;
    p.high = a.high;
    p.kl = a.kl;
    p.mean = 1.0f / static_cast<float>(a.rows);
    p.status = a.status;
    p.wait_limit = a.wait_limit;
    int clusters = 0;
    ++*launches;
    cudaError_t e = a.dtype == MOARA_DTYPE_BF16 ? loss_as<__nv_bfloat16>(p, clusters, s) : loss_as<float>(p, clusters, s);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch(k_loss_sums, dim3(1), dim3(128), 0, s, 1, static_cast<const float2*>(p.terms), clusters, a.sums);
}

size_t policy_loss_workspace(int rows) { return static_cast<size_t>(std::min(rows, kLossClusters)) * 3 * sizeof(float2); }

}  // namespace moara
