// Root-mean-square norm of rows, with the residual's addition, and its gradients.
//   h = x + r (rounded to its type), s = 1 / sqrt(mean h^2 + eps), y = (h s) g
//   dx = dh + s (d - n mean(d n)) with d = dy g, n = h s;   dg = sum over rows of dy n
// DRAM-bound: each array is read or written once.
#include <cuda_bf16.h>

#include <algorithm>

#include "launch.cuh"
#include "layers.h"

namespace moara {
namespace {

using bf16 = __nv_bfloat16;

// V entries in one access, as fp32.
template <class T, int V> __device__ __forceinline__ void load(const T* p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = static_cast<float>(p[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const float4 a = *reinterpret_cast<const float4*>(p + e);
            v[e] = a.x; v[e + 1] = a.y; v[e + 2] = a.z; v[e + 3] = a.w;
        }
    } else {
        uint32_t w[V / 2];
        if constexpr (V == 8) {
            const uint4 a = *reinterpret_cast<const uint4*>(p);
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(p);
            w[0] = a.x; w[1] = a.y;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <class T> __device__ __forceinline__ T rounded(float x) {
    if constexpr (sizeof(T) == 4) return x;
    else return __float2bfloat16_rn(x);
}

template <class T, int V> __device__ __forceinline__ void store(T* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        p[0] = rounded<T>(v[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(p + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    } else if constexpr (V == 8) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    } else {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    }
}

// The same at column c of a row with n columns, zero behind its end.
template <class T, int V> __device__ __forceinline__ void load_at(const T* row, int c, int n, float (&v)[V]) {
    if (c + V <= n) {
        load<T, V>(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = c + e < n ? static_cast<float>(row[c + e]) : 0.0f;
    }
}

template <class T, int V> __device__ __forceinline__ void store_at(T* row, int c, int n, const float (&v)[V]) {
    if (c + V <= n) {
        store<T, V>(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < n) row[c + e] = rounded<T>(v[e]);
    }
}

// A sum held in two fp32 numbers: what an addition rounds off goes to the second.  (The
// GPU adds 2 fp64 numbers per clock and SM: a row's sum in those would take longer than
// its way through DRAM.)
struct Sum {
    float hi = 0.0f, lo = 0.0f;
    __device__ __forceinline__ void add(float x) {
        const float s = hi + x, b = s - hi;
        lo += (hi - (s - b)) + (x - b);
        hi = s;
    }
    __device__ __forceinline__ void add(const Sum& o) {
        add(o.hi);
        lo += o.lo;
    }
};

// 1 / sqrt(sum / n + eps): a Newton step on the residual of rsqrtf, in two numbers
// throughout, so that the result is the nearest fp32 number but for rare ties.
__device__ __forceinline__ float inverse_rms(const Sum& s, int n, float eps) {
    if (!(s.hi < INFINITY)) return rsqrtf(s.hi);             // lo is NaN beside it
    const float f = static_cast<float>(n), total = s.hi + s.lo, rest = (s.hi - total) + s.lo;
    const float q = total / f, ql = (fmaf(-q, f, total) + rest) / f;
    Sum m;
    m.hi = q;
    m.lo = ql;
    m.add(eps);
    const float a = m.hi + m.lo, al = (m.hi - a) + m.lo;
    const float r = rsqrtf(a);
    if (!(r > 0.0f && r < INFINITY)) return r;               // of infinity, zero or NaN
    const float p = r * r, pl = fmaf(r, r, -p);
    const float e = fmaf(-a, p, 1.0f) - (a * pl + al * p);
    return fmaf(0.5f * r, e, r);
}

// Sum of a group of threads (whole warps), in every one of them.  part: two slots of 32
// for each group, taken in turn, so that one barrier a row is enough.
__device__ __forceinline__ Sum group_sum(Sum s, int group, float2* part) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        Sum t;
        t.hi = __shfl_xor_sync(0xffffffffu, s.hi, o);
        t.lo = __shfl_xor_sync(0xffffffffu, s.lo, o);
        // the same result in both lanes
        const bool first = s.hi > t.hi || (s.hi == t.hi && s.lo >= t.lo);
        Sum a = first ? s : t;
        a.add(first ? t : s);
        s = a;
    }
    const int warps = group >> 5;
    if (warps == 1) return s;
    const int lane = threadIdx.x & 31, w = threadIdx.x % group >> 5;
    if (lane == 0) part[w] = make_float2(s.hi, s.lo);
    __syncthreads();
    Sum all;
    for (int i = 0; i < warps; ++i) {
        Sum t;
        t.hi = part[i].x;
        t.lo = part[i].y;
        all.add(t);
    }
    return all;
}

struct ForwardParams {
    const void* x;
    const void* r;
    void* h;
    void* y;
    const float* gain;
    float* rstd;
    long long ldx, ldr, ldh, ldy;
    int rows, cols, group;
    float eps;
};

// A group of threads takes a row and keeps it in registers, E entries a thread; E = 0:
// a row of more than 16384 entries is read again, from L2, once its sum is known.
template <class T, class TY, int V, int E>
__global__ void __launch_bounds__(1024) k_norm(const ForwardParams p) {
    __shared__ float2 parts[32];
    const int group = p.group, per = blockDim.x / group, mine = threadIdx.x / group, i = threadIdx.x % group;
    const long long row = static_cast<long long>(blockIdx.x) * per + mine;
    const bool real = row < p.rows;
    const int n = p.cols;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* r = p.r == nullptr ? nullptr : static_cast<const T*>(p.r) + row * p.ldr;
    T* h = p.r == nullptr ? nullptr : static_cast<T*>(p.h) + row * p.ldh;
    TY* y = p.y == nullptr ? nullptr : static_cast<TY*>(p.y) + row * p.ldy;
    pdl_begin();
    constexpr int NV = E == 0 ? 1 : E / V;
    float f[NV][V];
    Sum s;
    auto take = [&](int c, float (&v)[V]) {
        load_at<T, V>(x, c, n, v);
        if (r != nullptr) {
            float w[V];
            load_at<T, V>(r, c, n, w);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = static_cast<float>(rounded<T>(v[e] + w[e]));
        }
    };
    auto square = [&](const float (&v)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float q = v[e] * v[e];
            s.add(q);
            if (sizeof(T) == 4) s.lo += fmaf(v[e], v[e], -q);   // of bf16 entries it is exact
        }
    };
    auto put = [&](int c, const float (&v)[V], float rstd) {
        float g[V], o[V];
        load_at<float, V>(p.gain, c, n, g);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = v[e] * rstd * g[e];
        store_at<TY, V>(y, c, n, o);
    };
    if constexpr (E > 0) {
        if (real) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * group + i) * V;
                if (c < n) take(c, f[j]);
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * group + i) * V;
                if (c >= n) continue;
                square(f[j]);
                if (h != nullptr) store_at<T, V>(h, c, n, f[j]);
            }
        }
    } else if (real) {
        for (int c = i * V; c < n; c += group * V) {
            take(c, f[0]);
            square(f[0]);
            if (h != nullptr) store_at<T, V>(h, c, n, f[0]);
        }
    }
    s = group_sum(s, group, parts + mine * (group >> 5));
    if (!real) return;
    const float rstd = inverse_rms(s, n, p.eps);
    if (i == 0) p.rstd[row] = rstd;
    if (y == nullptr) return;
    if constexpr (E > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * group + i) * V;
            if (c < n) put(c, f[j], rstd);
        }
    } else {
        const T* from = h != nullptr ? h : x;                // a thread's own entries
        for (int c = i * V; c < n; c += group * V) {
            load_at<T, V>(from, c, n, f[0]);
            put(c, f[0], rstd);
        }
    }
}

struct BackwardParams {
    const void* dy;
    const void* h;
    const void* dh;
    void* dx;
    const float* gain;
    const float* rstd;
    float* partials;
    long long lddy, ldh, lddh, lddx;
    int rows, cols, group;
};

// CTAs take rows a grid apart and leave their columns' sums of dy n.  E entries a thread
// in registers, with the columns' sums; E = 0: rows of more than 8192 entries are read
// again, the sums are in shared memory.
template <class T, class TY, int V, int E>
__global__ void __launch_bounds__(E == 0 ? 1024 : 512) k_norm_backward(const BackwardParams p) {
    extern __shared__ float columns[];
    __shared__ float2 parts[2][32];
    const int group = p.group, per = blockDim.x / group, mine = threadIdx.x / group, i = threadIdx.x % group;
    const int n = p.cols;
    constexpr int NV = E == 0 ? 1 : E / V;
    float acc[NV][V] = {};
    if (E == 0)
        for (int c = threadIdx.x; c < n; c += blockDim.x) columns[c] = 0.0f;
    if (E == 0) __syncthreads();
    pdl_begin();
    int turn = 0;
    const float inv = 1.0f / static_cast<float>(n);
    for (long long row0 = static_cast<long long>(blockIdx.x) * per; row0 < p.rows;
         row0 += static_cast<long long>(gridDim.x) * per, turn ^= 1) {
        const long long row = row0 + mine;
        const bool real = row < p.rows;
        const TY* dy = static_cast<const TY*>(p.dy) + row * p.lddy;
        const T* h = static_cast<const T*>(p.h) + row * p.ldh;
        const T* dh = p.dh == nullptr ? nullptr : static_cast<const T*>(p.dh) + row * p.lddh;
        T* dx = static_cast<T*>(p.dx) + row * p.lddx;
        float a[NV][V], b[NV][V], rstd = 0.0f;
        Sum dot;
        // a: dy, b: h s
        auto take = [&](int c, float (&u)[V], float (&v)[V]) {
            load_at<TY, V>(dy, c, n, u);
            load_at<T, V>(h, c, n, v);
        };
        auto product = [&](int c, const float (&u)[V], float (&v)[V]) {
            float g[V], q = 0.0f;
            load_at<float, V>(p.gain, c, n, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[e] *= rstd;
                q = fmaf(u[e] * g[e], v[e], q);
                if (e % 4 == 3 || e == V - 1) {
                    dot.add(q);
                    q = 0.0f;
                }
            }
        };
        auto put = [&](int c, const float (&u)[V], const float (&v)[V], float mean) {
            float g[V], o[V];
            load_at<float, V>(p.gain, c, n, g);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = rstd * fmaf(-v[e], mean, u[e] * g[e]);
            if (dh != nullptr) {
                float w[V];
                load_at<T, V>(dh, c, n, w);
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] += w[e];
            }
            store_at<T, V>(dx, c, n, o);
        };
        if (real) {
            rstd = p.rstd[row];
            if constexpr (E > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * group + i) * V;
                    if (c < n) take(c, a[j], b[j]);
                }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * group + i) * V;
                    if (c < n) product(c, a[j], b[j]);
                }
            } else {
                for (int c = i * V; c < n; c += group * V) {
                    take(c, a[0], b[0]);
                    product(c, a[0], b[0]);
                }
            }
        }
        dot = group_sum(dot, group, parts[turn] + mine * (group >> 5));
        if (!real) continue;
        const float mean = (dot.hi + dot.lo) * inv;
        if constexpr (E > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * group + i) * V;
                if (c >= n) continue;
                put(c, a[j], b[j], mean);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[j][e] = fmaf(a[j][e], b[j][e], acc[j][e]);
            }
        } else {
            for (int c = i * V; c < n; c += group * V) {
                take(c, a[0], b[0]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    b[0][e] *= rstd;
                    if (c + e < n) columns[c + e] = fmaf(a[0][e], b[0][e], columns[c + e]);
                }
                put(c, a[0], b[0], mean);
            }
        }
    }
    float* out = p.partials + static_cast<long long>(blockIdx.x) * n;
    if constexpr (E > 0) {
        if (per > 1) {
            // the groups' sums, in order
            for (int k = 0; k < per; ++k) {
                __syncthreads();
                if (mine != k) continue;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int c = (j * group + i) * V + e;
                        if (c < n) columns[c] = k == 0 ? acc[j][e] : columns[c] + acc[j][e];
                    }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < n; c += blockDim.x) out[c] = columns[c];
            return;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * group + i) * V;
            if (c < n) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (c + e < n) out[c + e] = acc[j][e];
            }
        }
    } else {
        __syncthreads();
        for (int c = threadIdx.x; c < n; c += blockDim.x) out[c] = columns[c];
    }
}

// Column sums of the partial rows, in their order: 32 columns a CTA, 16 warps share the rows.
__global__ void __launch_bounds__(512) k_norm_gain(const float* partials, int count, int n, float* dgain) {
    __shared__ float2 sums[16][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    pdl_begin();
    Sum s;
    if (c < n)
        for (int r = w; r < count; r += 16) s.add(partials[static_cast<long long>(r) * n + c]);
    sums[w][lane] = make_float2(s.hi, s.lo);
    __syncthreads();
    if (w > 0 || c >= n) return;
    for (int k = 1; k < 16; ++k) {
        Sum t;
        t.hi = sums[k][lane].x;
        t.lo = sums[k][lane].y;
        s.add(t);
    }
    dgain[c] = s.hi + s.lo;
}

bool lines(const void* p, int64_t ld, int size, int v) {
    const uintptr_t bytes = std::min(16, v * size);
    return p == nullptr || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld % v == 0);
}

// Threads of a row of n entries, e of them each.
int group_of(int n, int e) { return (n + 32 * e - 1) / (32 * e) * 32; }

template <class T, class TY, int V> cudaError_t forward_as(const ForwardParams& q, cudaStream_t s) {
    ForwardParams p = q;
    const int n = p.cols;
    const bool wide = n > 16384;
    const int e = n <= 8192 ? 8 : 16;
    p.group = wide ? 1024 : group_of(n, e);
    const int per = std::max(1, 256 / p.group);
    const auto fn = wide ? k_norm<T, TY, V, 0> : e == 8 ? k_norm<T, TY, V, 8> : k_norm<T, TY, V, 16>;
    return launch(fn, dim3((p.rows - 1) / per + 1), dim3(p.group * per), 0, s, 1, p);
}

template <class T, class TY> cudaError_t forward_of(const ForwardParams& p, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = lines(p.x, p.ldx, sizeof(T), V) && lines(p.r, p.ldr, sizeof(T), V) && lines(p.h, p.ldh, sizeof(T), V) &&
                     lines(p.y, p.ldy, sizeof(TY), V) && lines(p.gain, 0, 4, V);
    return vec ? forward_as<T, TY, V>(p, s) : forward_as<T, TY, 1>(p, s);
}

struct BackwardShape {
    int entries, group, per, ctas;
};

BackwardShape backward_shape(int rows, int n) {
    BackwardShape b;
    b.entries = n <= 4096 ? 8 : n <= 8192 ? 16 : 0;
    b.group = b.entries == 0 ? 1024 : group_of(n, b.entries);
    b.per = std::max(1, 256 / b.group);
    const int resident = std::max(1, 1536 / (b.group * b.per));
    const long long need = (static_cast<long long>(rows) - 1) / b.per + 1;
    b.ctas = static_cast<int>(std::min<long long>(need, 152LL * (b.entries == 0 ? 1 : resident)));
    return b;
}

template <class T, class TY, int V> cudaError_t backward_as(const BackwardParams& q, const BackwardShape& b, cudaStream_t s) {
    BackwardParams p = q;
    p.group = b.group;
    const size_t smem = b.entries == 0 || b.per > 1 ? static_cast<size_t>(p.cols) * 4 : 0;
    const auto fn = b.entries == 0   ? k_norm_backward<T, TY, V, 0>
                    : b.entries == 8 ? k_norm_backward<T, TY, V, 8>
                                     : k_norm_backward<T, TY, V, 16>;
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormCols * 4);
        if (e != cudaSuccess) return e;
    }
    return launch(fn, dim3(b.ctas), dim3(b.group * b.per), smem, s, 1, p);
}

template <class T, class TY> cudaError_t backward_of(const BackwardParams& p, const BackwardShape& b, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = lines(p.dy, p.lddy, sizeof(TY), V) && lines(p.h, p.ldh, sizeof(T), V) &&
                     lines(p.dh, p.lddh, sizeof(T), V) && lines(p.dx, p.lddx, sizeof(T), V) && lines(p.gain, 0, 4, V);
    return vec ? backward_as<T, TY, V>(p, b, s) : backward_as<T, TY, 1>(p, b, s);
}

}  // namespace

cudaError_t launch_norm(const NormForward& a, cudaStream_t s, int64_t* launches) {
    const ForwardParams p{a.x, a.r, a.h, a.y, a.gain, a.rstd, a.ldx, a.ldr, a.ldh, a.ldy, a.rows, a.cols, 0, a.eps};
    ++*launches;
    if (a.dtype == MOARA_DTYPE_BF16)
        return a.y_dtype == MOARA_DTYPE_BF16 ? forward_of<bf16, bf16>(p, s) : forward_of<bf16, float>(p, s);
    return a.y_dtype == MOARA_DTYPE_BF16 ? forward_of<float, bf16>(p, s) : forward_of<float, float>(p, s);
}

int norm_partials(int rows, int cols) { return backward_shape(rows, cols).ctas; }

cudaError_t launch_norm_backward(const NormBackward& a, cudaStream_t s, int64_t* launches) {
    const BackwardParams p{a.dy, a.h, a.dh, a.dx, a.gain, a.rstd, a.partials, a.lddy, a.ldh, a.lddh, a.lddx, a.rows, a.cols, 0};
    const BackwardShape b = backward_shape(a.rows, a.cols);
    ++*launches;
    cudaError_t e;
    if (a.dtype == MOARA_DTYPE_BF16)
        e = a.dy_dtype == MOARA_DTYPE_BF16 ? backward_of<bf16, bf16>(p, b, s) : backward_of<bf16, float>(p, b, s);
    else
        e = a.dy_dtype == MOARA_DTYPE_BF16 ? backward_of<float, bf16>(p, b, s) : backward_of<float, float>(p, b, s);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch(k_norm_gain, dim3((a.cols - 1) / 32 + 1), dim3(512), 0, s, 1, static_cast<const float*>(a.partials), b.ctas,
                  a.cols, a.dgain);
}

}  // namespace moara
