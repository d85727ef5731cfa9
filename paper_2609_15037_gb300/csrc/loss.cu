// Clipped policy loss of a batch of tokens from their logits, with its gradient.
//   lp = z_a - log sum_j exp z_j, rho = exp(lp - old), x = ref - lp
//   loss = -min(rho A, clamp(rho, low, high) A) + kl (exp x - x - 1)
//   dz_j = g (1[j = a] - exp(z_j) / sum),   g = w (kl (1 - exp x) - [not clipped] rho A)
// DRAM-bound: the logits are read once and their gradient written once.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

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
    float* terms;
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

struct LossCtl {
    uint64_t full;
    int abort;
    float top, sum, at;            // of this CTA's part: reference, sum, the target's logit if it is here
    float factor, gain;            // of the gradient
    float part[32];
};

__device__ __forceinline__ float ld_cluster_f32(uint32_t a) { return __uint_as_float(ptx::ld_cluster_u32(a)); }

// A cluster of `split` CTAs takes a row, each a part of its columns, which a bulk copy
// puts into shared memory in the 16-byte lines of the row's own alignment; what lies in
// the first and last line beside the part is -infinity there.  !STAGED: a part that is
// too large for that is read again from L2.
template <class T, bool STAGED>
__global__ void __launch_bounds__(1024) k_policy_loss(const __grid_constant__ LossParams p) {
    extern __shared__ __align__(16) uint8_t raw[];
    using L = Line<T>;
    constexpr int N = L::N;
    __shared__ LossCtl ctl;
    const int rank = blockIdx.x % p.split, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long row = blockIdx.x / p.split;
    const int first = rank * p.part, len = max(0, min(p.vocab - first, p.part));
    const T* z = static_cast<const T*>(p.z) + row * p.ldz + first;
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(z) & 15) / static_cast<int>(sizeof(T));
    const T* line0 = z - off;                                   // of the part's first line
    const int lines = (off + len + N - 1) / N;
    const int inner0 = off != 0, inner1 = (off + len) / N;      // whole lines
    if (threadIdx.x == 0) {
        ctl.abort = 0;
        if (STAGED) {
            ptx::mbar_init(ptx::smem_u32(&ctl.full), 1);
            ptx::fence_barrier_init();
        }
    }
    __syncthreads();
    pdl_begin();
    T* const stage = reinterpret_cast<T*>(raw);
    // an element of the part's lines, -infinity outside the part
    auto edge = [&](int i) -> T {
        const int c = i - off;
        return c >= 0 && c < len ? line0[i] : L::rounded(-INFINITY);
    };
    auto gather = [&](int line) {
        uint4 w;
        T* t = reinterpret_cast<T*>(&w);
#pragma unroll
        for (int e = 0; e < N; ++e) t[e] = edge(line * N + e);
        return w;
    };
    auto fetch = [&](int line) -> uint4 {
        if (STAGED) return reinterpret_cast<const uint4*>(raw)[line];
        return line >= inner0 && line < inner1 ? reinterpret_cast<const uint4*>(line0)[line] : gather(line);
    };
    const int64_t target = p.target[row];
    const bool counts = target >= 0 && target < p.vocab;
    const int owner = counts ? static_cast<int>(target / p.part) : 0;
    bool ok = true;
    if (STAGED) {
        if (threadIdx.x == 0 && inner1 > inner0) {
            const uint32_t bar = ptx::smem_u32(&ctl.full), bytes = (inner1 - inner0) * 16u;
            ptx::mbar_arrive_expect_tx(bar, bytes);
            for (uint32_t at = 0; at < bytes; at += 16384)
                ptx::bulk_load(ptx::smem_u32(raw) + inner0 * 16 + at, reinterpret_cast<const uint8_t*>(line0) + inner0 * 16 + at,
                               min(16384u, bytes - at), bar);
        }
        // the first and the last line, where they are not whole
        if (threadIdx.x >= 32 && threadIdx.x < 32 + 2 * N) {
            const int e = threadIdx.x - 32, line = e < N ? 0 : lines - 1;
            const bool whole = line >= inner0 && line < inner1;
            if (lines > 0 && !whole) stage[line * N + e % N] = edge(line * N + e % N);
        }
        if (inner1 > inner0)
            ok = ptx::mbar_wait(ptx::smem_u32(&ctl.full), 0, &ctl.abort, p.status, MOARA_ERR_DEVICE_TIMEOUT, p.wait_limit);
        if (!ok) wait_drain(ptx::smem_u32(&ctl.full), 0);
        ok = __syncthreads_and(ok);
    }
    auto all = [&](float v, bool largest) {
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            const float w = __shfl_xor_sync(0xffffffffu, v, o);
            v = largest ? fmaxf(v, w) : v + w;
        }
        if (lane == 0) ctl.part[warp] = v;
        __syncthreads();
        const int warps = blockDim.x >> 5;
        v = lane < warps ? ctl.part[lane] : largest ? -INFINITY : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            const float w = __shfl_xor_sync(0xffffffffu, v, o);
            v = largest ? fmaxf(v, w) : v + w;
        }
        __syncthreads();
        return v;
    };
    float top = -INFINITY;
    for (int i = threadIdx.x; i < lines; i += blockDim.x) top = fmaxf(top, L::top(fetch(i)));
    top = all(top, true);
    // a part without a finite logit: its exponentials are 0 (or NaN, or infinity's)
    const float ref = top == -INFINITY ? 0.0f : L::reference(top);
    uint64_t sums2 = 0;
    for (int i = threadIdx.x; i < lines; i += blockDim.x) {
        const uint4 w = fetch(i);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) sums2 = add2(sums2, L::exponentials(L::pair(w, e), ref));
    }
    float sum, odd;
    split(sums2, sum, odd);
    sum = all(sum + odd, false);
    if (threadIdx.x == 0) {
        ctl.top = top == -INFINITY ? -INFINITY : ref;
        ctl.sum = ok ? sum : NAN;
        if (counts && owner == rank) {
            const int i = static_cast<int>(target - first) + off;
            ctl.at = static_cast<float>(STAGED ? stage[i] : line0[i]);
        }
    }
    if (p.split > 1) ptx::cluster_sync();
    else __syncthreads();
    if (threadIdx.x == 0) {
        float base = -INFINITY, total = 0.0f, at = 0.0f;
        float tops[8], sums[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if (r >= p.split) break;
            tops[r] = p.split == 1 ? ctl.top : ld_cluster_f32(ptx::mapa(ptx::smem_u32(&ctl.top), r));
            sums[r] = p.split == 1 ? ctl.sum : ld_cluster_f32(ptx::mapa(ptx::smem_u32(&ctl.sum), r));
            base = fmaxf(base, tops[r]);
        }
        if (counts) at = p.split == 1 ? ctl.at : ld_cluster_f32(ptx::mapa(ptx::smem_u32(&ctl.at), owner));
        const float base0 = base == -INFINITY ? 0.0f : base;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if (r >= p.split) break;
            total += tops[r] == -INFINITY ? sums[r] : sums[r] * L::apart(tops[r] - base0);
        }
        // log(total) from its exponent and the rest, which lies in [1, 2)
        int e = 0;
        float log_total;
        double lp;
        if (total > 0.0f && total < INFINITY) {
            e = static_cast<int>(__float_as_uint(total) >> 23) - 127;
            log_total = logf(__uint_as_float((__float_as_uint(total) & 0x7FFFFFu) | 0x3F800000u));
            lp = static_cast<double>(at) - (L::natural(base0) + (e * kLn2 + log_total));
        } else {
            lp = static_cast<double>(at) - (L::natural(base0) + logf(total));
        }
        const float w = p.weight != nullptr ? p.weight[row] : p.mean;
        float gain = 0.0f, loss = 0.0f, kl = 0.0f, cut = 0.0f;
        const bool taken = counts && w != 0.0f;
        if (taken) {
            const float a = p.adv[row], rho = expf(static_cast<float>(lp - p.old_logp[row]));
            // NaN advantages and ratios stay NaN
            const float bound = rho < p.low ? p.low : rho > p.high ? p.high : rho;
            const bool clipped = bound * a < rho * a;
            loss = clipped ? -bound * a : -rho * a;
            float d = clipped ? 0.0f : -rho * a;
            if (p.ref_logp != nullptr) {
                const float x = static_cast<float>(p.ref_logp[row] - lp);
                kl = exp_beyond_linear(x);
                loss = fmaf(p.kl, kl, loss);
                d = fmaf(-p.kl, expm1f(x), d);
            }
            cut = clipped ? w : 0.0f;
            kl *= w;
            loss *= w;
            gain = w * d;
        }
        if (rank == 0) {
            p.logp[row] = counts ? static_cast<float>(lp) : 0.0f;
            p.terms[3 * row] = loss;
            p.terms[3 * row + 1] = kl;
            p.terms[3 * row + 2] = cut;
        }
        ctl.gain = gain;
        // relative to this part's reference; infinite where nothing of it is to be multiplied
        ctl.factor = taken ? -gain * ((ctl.top == -INFINITY ? 1.0f : L::apart(ref - base0)) / total) : INFINITY;
    }
    if (p.split > 1) ptx::cluster_sync();       // no CTA leaves while another reads its sums
    else __syncthreads();
    if (p.dz == nullptr || !ok) return;
    const float factor = ctl.factor, gain = ctl.gain;
    const bool zero = factor == INFINITY;
    T* dz = static_cast<T*>(p.dz) + row * p.lddz + first;
    const bool same = (reinterpret_cast<uintptr_t>(dz) & 15) == off * sizeof(T);
    T* out0 = dz - off;
    const int hit = counts && owner == rank ? static_cast<int>(target - first) + off : -1, hit_line = hit < 0 ? -1 : hit / N;
    for (int i = threadIdx.x; i < lines; i += blockDim.x) {
        const uint4 w = fetch(i);
        uint64_t v[N / 2];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) v[e] = zero ? 0 : mul2(L::exponentials(L::pair(w, e), ref), both(factor));
        if (i == hit_line && !zero) {
#pragma unroll
            for (int e = 0; e < N / 2; ++e)
                if (hit % N / 2 == e) v[e] = add2(v[e], hit & 1 ? f32x2(0.0f, gain) : f32x2(gain, 0.0f));
        }
        if (same && i >= inner0 && i < inner1) {
            reinterpret_cast<uint4*>(out0)[i] = L::pack(v);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int c = i * N + e - off;
                float x[2];
                split(v[e / 2], x[0], x[1]);
                if (c >= 0 && c < len) dz[c] = L::rounded(x[e & 1]);
            }
        }
    }
}

// The three sums over the rows, in their order by thread; what an addition rounds off is kept.
__global__ void __launch_bounds__(1024) k_loss_sums(const float* terms, int rows, float* sums) {
    __shared__ float2 part[3][32];
    pdl_begin();
    float hi[3] = {}, lo[3] = {};
    auto add = [&](int k, float x) {
        const float s = hi[k] + x, b = s - hi[k];
        lo[k] += (hi[k] - (s - b)) + (x - b);
        hi[k] = s;
    };
    for (int r = threadIdx.x; r < rows; r += blockDim.x)
#pragma unroll
        for (int k = 0; k < 3; ++k) add(k, terms[3LL * r + k]);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto across = [&](int k) {
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            const float h = __shfl_down_sync(0xffffffffu, hi[k], o), l = __shfl_down_sync(0xffffffffu, lo[k], o);
            add(k, h);
            lo[k] += l;
        }
    };
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        across(k);
        if (lane == 0) part[k][warp] = make_float2(hi[k], lo[k]);
    }
    __syncthreads();
    if (warp > 0) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const bool has = lane < static_cast<int>(blockDim.x >> 5);
        hi[k] = has ? part[k][lane].x : 0.0f;
        lo[k] = has ? part[k][lane].y : 0.0f;
        across(k);
        if (lane == 0) sums[k] = hi[k] + lo[k];
    }
}

constexpr int kStage = 200 * 1024;     // most bytes of a part in shared memory

template <class T, bool STAGED> cudaError_t launch_loss(const LossParams& p, cudaStream_t s) {
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
    const int threads = std::min(STAGED ? 512 : 1024, std::max(64, (lines + 31) / 32 * 32));
    return launch(fn, dim3(static_cast<unsigned int>(p.rows) * p.split), dim3(threads), bytes, s, p.split, p);
}

template <class T> cudaError_t loss_as(LossParams& p, cudaStream_t s) {
    constexpr int N = Line<T>::N;
    // a row over more CTAs while they are few, each with some 4 KB and more, and where its part
    // would fill an SM's shared memory alone
    p.split = 1;
    const auto part = [&](int split) { return ((p.vocab - 1) / split + N) / N * N; };
    while (p.split < 8 && (part(p.split) * static_cast<long long>(sizeof(T)) > 72 * 1024 ||
                           (2LL * p.split * p.rows <= 304 && part(2 * p.split) * sizeof(T) >= 4096)))
        p.split *= 2;
    p.part = part(p.split);
    return p.part * static_cast<long long>(sizeof(T)) <= kStage ? launch_loss<T, true>(p, s) : launch_loss<T, false>(p, s);
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
    p.terms = a.terms;
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
    ++*launches;
    cudaError_t e = a.dtype == MOARA_DTYPE_BF16 ? loss_as<__nv_bfloat16>(p, s) : loss_as<float>(p, s);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch(k_loss_sums, dim3(1), dim3(std::min(1024, (a.rows + 31) / 32 * 32)), 0, s, 1, static_cast<const float*>(a.terms),
                  a.rows, a.sums);
}

}  // namespace moara
