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
constexpr double kLn2 = 0.69314718055994530942;

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

// 16 bytes of a row as pairs of fp32 numbers, their largest (NaN left out: it returns in the
// sum), and exponentials relative to a reference: powers of two, whose argument is one fused
// operation for bf16 logits, an error far below the gradient's rounding; fp32 logits take z - ref
// exactly as far as fp32 holds it, and what the product with log2 e rounds off as a factor
// (1 + its natural power).
template <class T> struct Line;

template <> struct Line<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ uint64_t pair(const uint4& w, int e) {
        return e == 0 ? f32x2(__uint_as_float(w.x), __uint_as_float(w.y)) : f32x2(__uint_as_float(w.z), __uint_as_float(w.w));
    }
    static __device__ __forceinline__ float top(const uint4& w) {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    static __device__ __forceinline__ float reference(float top) { return top; }
    static __device__ __forceinline__ uint64_t exponentials(uint64_t z, float ref) {
        const uint64_t t = add2(z, both(-ref)), l = both(kLog2e), x = mul2(t, l);
        float a, b, c, d;
        split(x, a, b);
        // of minus infinity the rest is NaN: its exponential is 0 whatever it is
        split(fma2(t, l, mul2(x, both(-1.0f))), c, d);
        const uint64_t y = f32x2(ex2(a), ex2(b));
        return fma2(y, mul2(f32x2(a == -INFINITY ? 0.0f : c, b == -INFINITY ? 0.0f : d), both(0.69314718f)), y);
    }
    static __device__ __forceinline__ float apart(float x) { return expf(x); }      // of a difference of references
    static __device__ __forceinline__ double natural(float ref) { return ref; }
    static __device__ __forceinline__ uint4 pack(const uint64_t (&v)[2]) {
        float a, b, c, d;
        split(v[0], a, b);
        split(v[1], c, d);
        return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
    }
    static __device__ __forceinline__ float rounded(float x) { return x; }
};

template <> struct Line<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ uint64_t pair(const uint4& w, int e) {
        return widen2(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w);
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t y;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
        return y;
    }
    static __device__ __forceinline__ float top(const uint4& w) {
        const uint32_t t = max2(max2(w.x, w.y), max2(w.z, w.w));
        return fmaxf(__uint_as_float(t << 16), __uint_as_float(t & 0xFFFF0000u));
    }
    static __device__ __forceinline__ float reference(float top) { return top * kLog2e; }
    static __device__ __forceinline__ uint64_t exponentials(uint64_t z, float ref) {
        float a, b;
        split(fma2(z, both(kLog2e), both(-ref)), a, b);
        return f32x2(ex2(a), ex2(b));
    }
    static __device__ __forceinline__ float apart(float x) { return ex2(x); }
    static __device__ __forceinline__ double natural(float ref) { return ref * kLn2; }
    static __device__ __forceinline__ uint32_t pack2(uint64_t v) {
        float a, b;
        split(v, a, b);
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const uint64_t (&v)[4]) {
        return make_uint4(pack2(v[0]), pack2(v[1]), pack2(v[2]), pack2(v[3]));
    }
    static __device__ __forceinline__ __nv_bfloat16 rounded(float x) { return __float2bfloat16_rn(x); }
};

// A sum held in two fp32 numbers: what an addition rounds off goes to the second.
struct Sum {
    float hi = 0.0f, lo = 0.0f;
    __device__ __forceinline__ void add(float x) {
        const float s = hi + x, b = s - hi;
        lo += (hi - (s - b)) + (x - b);
        hi = s;
    }
};

struct LossCtl {
    uint64_t full;
    int abort;
    float top, sum, at;            // of this CTA's part: reference, sum, the target's logit if it is here
    float factor, gain;            // of the gradient
    int hit;
    float part[2][32];
};

__device__ __forceinline__ float ld_cluster_f32(uint32_t a) { return __uint_as_float(ptx::ld_cluster_u32(a)); }

// A cluster of `split` CTAs takes rows a grid apart, each CTA a part of their columns, whose
// whole 16-byte lines a bulk copy puts into shared memory, in the row's own alignment; the next
// row's copy begins as soon as this one has been read.  The first and the last line are read where
// they lie if they are not whole, with -infinity beside the part.  !STAGED: a part that is too
// large for shared memory is read again from L2.
template <class T, bool STAGED>
__global__ void __launch_bounds__(512, 3) k_policy_loss(const __grid_constant__ LossParams p) {
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
            ptx::mbar_init(ptx::smem_u32(&ctl.full), 1);
            ptx::fence_barrier_init();
            ptx::fence_proxy_async_smem();
        }
    }
    __syncthreads();
    pdl_begin();
    const uint32_t bar = ptx::smem_u32(&ctl.full), own = ptx::smem_u32(&ctl);
    const long long step = gridDim.x / p.split;
    // a row's part in lines: entries in front of it in its first line, lines, whole ones among them
    struct Place {
        const T* line0;
        int off, lines, inner0, inner1;
    };
    auto place = [&](long long row) {
        const T* z = static_cast<const T*>(p.z) + row * p.ldz + first;
        Place x;
        x.off = static_cast<int>(reinterpret_cast<uintptr_t>(z) & 15) / static_cast<int>(sizeof(T));
        x.line0 = z - x.off;
        x.lines = (x.off + len + N - 1) / N;
        x.inner0 = x.off != 0;
        x.inner1 = max(x.inner0, (x.off + len) / N);
        return x;
    };
    auto copy = [&](const Place& x) {
        const uint32_t bytes = (x.inner1 - x.inner0) * 16u;
        if (bytes == 0) return;
        ptx::mbar_arrive_expect_tx(bar, bytes);
        for (uint32_t at = 0; at < bytes; at += 16384)
            ptx::bulk_load(ptx::smem_u32(raw) + x.inner0 * 16 + at, reinterpret_cast<const uint8_t*>(x.line0) + x.inner0 * 16 + at,
                           min(16384u, bytes - at), bar);
    };
    long long row = blockIdx.x / p.split;
    Place x = place(row);
    if (STAGED && threadIdx.x == 0) copy(x);
    uint32_t phase = 0;
    Sum sums[3];                                 // of the first thread: loss, KL term, clipped
    for (; row < p.rows; row += step) {
        auto fetch = [&](int line) {
            if (line >= x.inner0 && line < x.inner1)
                return STAGED ? reinterpret_cast<const uint4*>(raw)[line] : reinterpret_cast<const uint4*>(x.line0)[line];
            uint4 w;
            T* t = reinterpret_cast<T*>(&w);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int c = line * N + e - x.off;
                t[e] = c >= 0 && c < len ? x.line0[line * N + e] : L::rounded(-INFINITY);
            }
            return w;
        };
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
        if (STAGED && x.inner1 > x.inner0) {
            if (!ptx::mbar_wait(bar, phase, abort_flag, p.status, MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit)) wait_drain(bar, phase);
            phase ^= 1;
        }
        auto all = [&](float v, bool largest, float* part) {
#pragma unroll
            for (int o = 16; o > 0; o /= 2) {
                const float y = __shfl_xor_sync(0xffffffffu, v, o);
                v = largest ? fmaxf(v, y) : v + y;
            }
            if (lane == 0) part[warp] = v;
            __syncthreads();
            v = lane < warps ? part[lane] : largest ? -INFINITY : 0.0f;
#pragma unroll
            for (int o = 16; o > 0; o /= 2) {
                const float y = __shfl_xor_sync(0xffffffffu, v, o);
                v = largest ? fmaxf(v, y) : v + y;
            }
            return v;
        };
        float top = -INFINITY;
#pragma unroll 4
        for (int i = threadIdx.x; i < x.lines; i += blockDim.x) top = fmaxf(top, L::top(fetch(i)));
        top = all(top, true, ctl.part[0]);
        // a part without a finite logit: its exponentials are 0 (or NaN, or infinity's)
        const float ref = top == -INFINITY ? 0.0f : L::reference(top);
        uint64_t pairs = 0;
#pragma unroll 4
        for (int i = threadIdx.x; i < x.lines; i += blockDim.x) {
            const uint4 v = fetch(i);
#pragma unroll
            for (int e = 0; e < N / 2; ++e) pairs = add2(pairs, L::exponentials(L::pair(v, e), ref));
        }
        float sum, odd;
        split(pairs, sum, odd);
        sum = all(sum + odd, false, ctl.part[1]);
        const bool ok = *abort_flag == 0;        // the same in every thread: a wait ran out before the barriers above
        if (threadIdx.x == 0) {
            const bool counts = target >= 0 && target < p.vocab;
            const int column = counts ? static_cast<int>(target) : 0, owner = column / p.part;
            ctl.top = top == -INFINITY ? -INFINITY : ref;
            ctl.sum = ok ? sum : NAN;
            if (counts && owner == rank) ctl.at = static_cast<float>(x.line0[column - first + x.off]);
        }
        if (p.split > 1) {
            __syncwarp();
            ptx::cluster_sync();
        }
        if (threadIdx.x == 0) {
            const bool counts = target >= 0 && target < p.vocab;
            const int column = counts ? static_cast<int>(target) : 0, owner = column / p.part;
            float tops[8], parts[8], base = -INFINITY, total = 0.0f, at = 0.0f;
            if (p.split == 1) {
                base = ctl.top;
                total = ctl.sum;
                at = ctl.at;
            } else {
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
            double lp;
            if (total > 0.0f && total < INFINITY) {
                const int e = static_cast<int>(__float_as_uint(total) >> 23) - 127;
                const float rest = logf(__uint_as_float((__float_as_uint(total) & 0x7FFFFFu) | 0x3F800000u));
                lp = static_cast<double>(at) - (L::natural(base0) + (e * kLn2 + rest));
            } else {
                lp = static_cast<double>(at) - (L::natural(base0) + logf(total));
            }
            float gain = 0.0f;
            const bool taken = counts && w != 0.0f;
            if (taken) {
                const float rho = expf(static_cast<float>(lp - old));
                // NaN advantages and ratios stay NaN
                const float bound = rho < p.low ? p.low : rho > p.high ? p.high : rho;
                const bool clipped = bound * a < rho * a;
                float loss = clipped ? -bound * a : -rho * a, d = clipped ? 0.0f : -rho * a;
                if (p.ref_logp != nullptr) {
                    const float y = static_cast<float>(other - lp), k = exp_beyond_linear(y);
                    loss = fmaf(p.kl, k, loss);
                    d = fmaf(-p.kl, expm1f(y), d);
                    sums[1].add(k * w);
                }
                sums[0].add(loss * w);
                if (clipped) sums[2].add(w);
                gain = w * d;
            }
            if (rank == 0) p.logp[row] = counts ? static_cast<float>(lp) : 0.0f;
            ctl.gain = gain;
            // relative to this part's reference; infinite where nothing of it is to be multiplied
            ctl.factor = taken ? -gain * ((ctl.top == -INFINITY ? 1.0f : L::apart(ref - base0)) / total) : INFINITY;
            // the target's place among the part's lines, none for -1
            ctl.hit = counts && owner == rank ? column - first + x.off : -1;
        }
        if (p.split > 1) {
            __syncwarp();
            ptx::cluster_sync();                 // no CTA goes on while another reads its sums
        } else {
            __syncthreads();
        }
        const Place mine = x;
        if (p.dz != nullptr && ok) {
            const float factor = ctl.factor, gain = ctl.gain;
            const int hit = ctl.hit, hit_line = hit < 0 ? -1 : hit / N;
            const bool zero = factor == INFINITY;
            T* dz = static_cast<T*>(p.dz) + row * p.lddz + first;
            const bool same = (reinterpret_cast<uintptr_t>(dz) & 15) == mine.off * sizeof(T);
            T* out0 = dz - mine.off;
#pragma unroll 4
            for (int i = threadIdx.x; i < mine.lines; i += blockDim.x) {
                const uint4 z = fetch(i);
                uint64_t v[N / 2];
#pragma unroll
                for (int e = 0; e < N / 2; ++e) v[e] = zero ? 0 : mul2(L::exponentials(L::pair(z, e), ref), both(factor));
                if (i == hit_line && !zero) {
#pragma unroll
                    for (int e = 0; e < N / 2; ++e)
                        if (hit % N / 2 == e) v[e] = add2(v[e], hit & 1 ? f32x2(0.0f, gain) : f32x2(gain, 0.0f));
                }
                if (same && i >= mine.inner0 && i < mine.inner1) {
                    reinterpret_cast<uint4*>(out0)[i] = L::pack(v);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const int c = i * N + e - mine.off;
                        float y[2];
                        split(v[e / 2], y[0], y[1]);
                        if (c >= 0 && c < len) dz[c] = L::rounded(y[e & 1]);
                    }
                }
            }
        }
        if (row + step < p.rows) {
            x = place(row + step);
            __syncthreads();                     // the row has been read
            if (STAGED && threadIdx.x == 0) copy(x);
        }
    }
    if (threadIdx.x == 0 && rank == 0)
        for (int k = 0; k < 3; ++k) p.terms[3 * (blockIdx.x / p.split) + k] = make_float2(sums[k].hi, sums[k].lo);
}

// The clusters' sums, added up in a fixed order: at most kLossClusters of them.
constexpr int kLossClusters = 152 * 8;
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
    // an infinite sum has NaN beside it
    out[threadIdx.x] = fabsf(all.hi) < INFINITY ? all.hi + all.lo : all.hi;
}

constexpr int kStage = 200 * 1024;     // most bytes of a part in shared memory

template <class T, bool STAGED> cudaError_t launch_loss(const LossParams& p, int& clusters, cudaStream_t s) {
    const auto fn = k_policy_loss<T, STAGED>;
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
    const int lines = p.part / Line<T>::N + 2;
    const int threads = std::min(512, std::max(64, (lines + 31) / 32 * 32));
    // CTAs that an SM holds, by registers and shared memory (1.5 KB beside the part)
    const int resident = std::max(1, std::min({8, 1536 / threads, (226 << 10) / (bytes + 1536)}));
    clusters = std::min(p.rows, 152 * resident / p.split);
    return launch(fn, dim3(static_cast<unsigned int>(clusters) * p.split), dim3(threads), bytes, s, p.split, p);
}

template <class T> cudaError_t loss_as(LossParams& p, int& clusters, cudaStream_t s) {
    constexpr int N = Line<T>::N;
    // a row over more CTAs while they are few, each with some 4 KB and more, and where its part
    // would fill an SM's shared memory alone
    p.split = 1;
    const auto part = [&](int split) { return ((p.vocab - 1) / split + N) / N * N; };
    while (p.split < 8 && (part(p.split) * static_cast<long long>(sizeof(T)) > 72 * 1024 ||
                           (2LL * p.split * p.rows <= 304 && part(2 * p.split) * sizeof(T) >= 4096)))
        p.split *= 2;
    p.part = part(p.split);
    return p.part * static_cast<long long>(sizeof(T)) <= kStage ? launch_loss<T, true>(p, clusters, s)
                                                                : launch_loss<T, false>(p, clusters, s);
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
