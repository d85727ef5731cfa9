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

// V entries as they lie in memory.
template <class T, int V> struct Raw {
    static constexpr int BYTES = V * static_cast<int>(sizeof(T)), WORDS = (BYTES + 3) / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (BYTES == 2) {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (BYTES == 8) {
            const uint2 a = *reinterpret_cast<const uint2*>(p);
            w[0] = a.x; w[1] = a.y;
        } else {
#pragma unroll
            for (int e = 0; e < WORDS; e += 4) {
                const uint4 a = *reinterpret_cast<const uint4*>(p + e * 4 / static_cast<int>(sizeof(T)));
                w[e] = a.x; w[e + 1] = a.y; w[e + 2] = a.z; w[e + 3] = a.w;
            }
        }
    }
    // column c of a row of n, zeros outside
    __device__ __forceinline__ void load_at(const T* row, int c, int n) {
        if (c >= 0 && c + V <= n) {
            load(row + c);
        } else {
#pragma unroll
            for (int e = 0; e < WORDS; ++e) w[e] = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (c + e < 0 || c + e >= n) continue;
                if constexpr (sizeof(T) == 4) w[e] = reinterpret_cast<const uint32_t*>(row)[c + e];
                else w[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[c + e]) << (16 * (e & 1));
            }
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
};

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

// The same at column c of a row with n columns (c may lie in front of it), zeros outside.
template <class T, int V> __device__ __forceinline__ void load_at(const T* row, int c, int n, float (&v)[V]) {
    if (c >= 0 && c + V <= n) {
        load<T, V>(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = c + e >= 0 && c + e < n ? static_cast<float>(row[c + e]) : 0.0f;
    }
}

template <class T, int V> __device__ __forceinline__ void store_at(T* row, int c, int n, const float (&v)[V]) {
    if (c >= 0 && c + V <= n) {
        store<T, V>(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e >= 0 && c + e < n) row[c + e] = rounded<T>(v[e]);
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
    int phase, pitch;      // SHIFT: of the first row's first entry in its line, and from row to row
};

// Rows that do not begin on 16-byte lines are taken in the lines they lie in, which all
// their arrays share (SHIFT): a row's first line begins `off` entries in front of it.  What belongs
// to columns (gain, sums) is in shared memory then, a column's V-th neighbours beside it, so
// that the lanes of a warp, V columns apart, meet different banks.
template <int V> __device__ __forceinline__ int column(int c, int n) { return c % V * (n / V + 1) + c / V; }

template <int V> __device__ __forceinline__ void stage_gain(float* to, const float* gain, int n) {
    for (int c = threadIdx.x; c < n; c += blockDim.x) to[column<V>(c, n)] = gain[c];
    __syncthreads();
}

template <bool SHIFT, int V>
__device__ __forceinline__ void gain_at(const float* gain, const float* staged, int c, int n, float (&g)[V]) {
    if constexpr (SHIFT) {
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = c + e >= 0 && c + e < n ? staged[column<V>(c + e, n)] : 0.0f;
    } else {
        load_at<float, V>(gain, c, n, g);
    }
}

// A group of threads takes a row and keeps it in registers, E entries a thread: 32, so that
// the sum over the group costs little beside them, or 8 where rows are too few to fill the GPU.
// E = 0: a row of more than 32768 entries is read again, from L2, once its sum is known.
template <class T, class TY, int V, int E, bool SHIFT>
__global__ void __launch_bounds__(1024) k_norm(const ForwardParams p) {
    extern __shared__ float staged[];
    __shared__ float2 parts[2][32];
    const int group = p.group, per = blockDim.x / group, mine = threadIdx.x / group, i = threadIdx.x % group;
    const int n = p.cols;
    pdl_begin();
    if (SHIFT) stage_gain<V>(staged, p.gain, n);
    constexpr int NV = E == 0 ? 1 : E / V;
    int turn = 0;
    for (long long row0 = static_cast<long long>(blockIdx.x) * per; row0 < p.rows;
         row0 += static_cast<long long>(gridDim.x) * per, turn ^= 1) {
        const long long row = row0 + mine;
        const bool real = row < p.rows;
        const T* x = static_cast<const T*>(p.x) + row * p.ldx;
        const T* r = p.r == nullptr ? nullptr : static_cast<const T*>(p.r) + row * p.ldr;
        T* h = p.r == nullptr ? nullptr : static_cast<T*>(p.h) + row * p.ldh;
        TY* y = p.y == nullptr ? nullptr : static_cast<TY*>(p.y) + row * p.ldy;
        const int off = SHIFT ? static_cast<int>((p.phase + row % V * p.pitch) % V) : 0;
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
            gain_at<SHIFT, V>(p.gain, staged, c, n, g);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = v[e] * rstd * g[e];
            store_at<TY, V>(y, c, n, o);
        };
        if constexpr (E > 0) {
            if (real) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * group + i) * V - off;
                    if (c < n) take(c, f[j]);
                }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * group + i) * V - off;
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
        s = group_sum(s, group, parts[turn] + mine * (group >> 5));
        if (!real) continue;
        const float rstd = inverse_rms(s, n, p.eps);
        if (i == 0) p.rstd[row] = rstd;
        if (y == nullptr) continue;
        if constexpr (E > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * group + i) * V - off;
                if (c < n) put(c, f[j], rstd);
            }
        } else {
            const T* from = h != nullptr ? h : x;            // a thread's own entries
            for (int c = i * V; c < n; c += group * V) {
                load_at<T, V>(from, c, n, f[0]);
                put(c, f[0], rstd);
            }
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
    int phase, pitch;
};

// CTAs take rows a grid apart and leave their columns' sums of dy n.  E entries a thread
// stay in registers as they came, with the columns' sums; E = 0: rows of more than 16384
// entries are read again, the sums are in shared memory.  SHIFT: there too; a column's sum has
// another thread from row to row, behind the barrier of the row's mean.
template <class T, class TY, int V, int E, bool SHIFT>
__global__ void __launch_bounds__(E == 0 ? 1024 : 512) k_norm_backward(const BackwardParams p) {
    extern __shared__ float columns[];
    float* const staged = columns + (p.cols / V + 1) * V;         // SHIFT: the gain
    __shared__ float2 parts[2][32];
    const int group = p.group, per = blockDim.x / group, mine = threadIdx.x / group, i = threadIdx.x % group;
    const int n = p.cols;
    constexpr int NV = E == 0 ? 1 : E / V;
    float acc[NV][V] = {};
    if (E == 0 || SHIFT) {
        for (int c = threadIdx.x; c < n; c += blockDim.x) columns[SHIFT ? column<V>(c, n) : c] = 0.0f;
        __syncthreads();
    }
    pdl_begin();
    if (SHIFT) stage_gain<V>(staged, p.gain, n);
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
        const int off = SHIFT ? static_cast<int>((p.phase + row % V * p.pitch) % V) : 0;
        Raw<TY, V> a[NV];
        Raw<T, V> b[NV], w[NV];
        float rstd = 0.0f;
        Sum dot;
        auto product = [&](int c, int j) {
            float g[V], q = 0.0f;
            gain_at<SHIFT, V>(p.gain, staged, c, n, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                q = fmaf(a[j].get(e) * g[e], b[j].get(e) * rstd, q);
                if (e % 4 == 3 || e == V - 1) {
                    dot.add(q);
                    q = 0.0f;
                }
            }
        };
        // dx, and the columns' sums by `add`
        auto put = [&](int c, int j, float mean, auto add) {
            float g[V], o[V];
            gain_at<SHIFT, V>(p.gain, staged, c, n, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float u = a[j].get(e), v = b[j].get(e) * rstd;
                add(e, u, v);
                o[e] = rstd * fmaf(-v, mean, u * g[e]);
                if (dh != nullptr) o[e] += w[j].get(e);
            }
            store_at<T, V>(dx, c, n, o);
        };
        if (real) {
            rstd = p.rstd[row];
            if constexpr (E > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * group + i) * V - off;
                    if (c >= n) continue;
                    a[j].load_at(dy, c, n);
                    b[j].load_at(h, c, n);
                }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * group + i) * V - off;
                    if (c < n && dh != nullptr) w[j].load_at(dh, c, n);
                }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * group + i) * V - off;
                    if (c < n) product(c, j);
                }
            } else {
                for (int c = i * V; c < n; c += group * V) {
                    a[0].load_at(dy, c, n);
                    b[0].load_at(h, c, n);
                    product(c, 0);
                }
            }
        }
        dot = group_sum(dot, group, parts[turn] + mine * (group >> 5));
        if (SHIFT) __syncwarp();                 // a group of one warp has no other barrier
        if (!real) continue;
        const float mean = (dot.hi + dot.lo) * inv;
        if constexpr (E > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * group + i) * V - off;
                if (c >= n) continue;
                put(c, j, mean, [&](int e, float u, float v) {
                    if constexpr (SHIFT) {
                        if (c + e < 0 || c + e >= n) return;
                        float& sum = columns[column<V>(c + e, n)];
                        sum = fmaf(u, v, sum);
                    } else {
                        acc[j][e] = fmaf(u, v, acc[j][e]);
                    }
                });
            }
        } else {
            for (int c = i * V; c < n; c += group * V) {
                a[0].load_at(dy, c, n);
                b[0].load_at(h, c, n);
                if (dh != nullptr) w[0].load_at(dh, c, n);
                put(c, 0, mean, [&](int e, float u, float v) {
                    if (c + e < n) columns[c + e] = fmaf(u, v, columns[c + e]);
                });
            }
        }
    }
    float* out = p.partials + static_cast<long long>(blockIdx.x) * n;
    if constexpr (E > 0 && !SHIFT) {
        // the groups' sums, in order
        for (int k = 0; k < per; ++k) {
            if (per > 1) __syncthreads();
            if (mine != k) continue;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int c = (j * group + i) * V + e;
                    if (c >= n) continue;
                    const float sum = k == 0 ? acc[j][e] : columns[c] + acc[j][e];
                    if (k + 1 < per) columns[c] = sum;
                    else out[c] = sum;
                }
        }
    } else {
        __syncthreads();
        for (int c = threadIdx.x; c < n; c += blockDim.x) out[c] = columns[SHIFT ? column<V>(c, n) : c];
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

// Whether the rows of all arrays lie alike in their 16-byte lines: `phase` entries into one
// of V entries in the first row, `pitch` more with every row.
struct Lines {
    int v;
    bool ok = true, any = false;
    int phase = 0, pitch = 0;
    explicit Lines(int entries) : v(entries) {}
    Lines& add(const void* p, int64_t ld, int size) {
        if (p == nullptr) return *this;
        const int line = 16 / size < v ? 16 / size : v;          // entries of this array's line that count
        const uintptr_t at = reinterpret_cast<uintptr_t>(p) / size;
        const int first = static_cast<int>(at % v), step = static_cast<int>(ld % v);
        if (!any) {
            any = true;
            phase = first;
            pitch = step;
        }
        ok = ok && (first - phase) % line == 0 && (step - pitch) % line == 0;
        return *this;
    }
    bool aligned() const { return ok && phase == 0 && pitch == 0; }
};

constexpr long long kFull = 152 * 2048;          // threads that the GPU holds

// Threads of a row of n entries, e of them each.
int group_of(int n, int e) { return (n + 32 * e - 1) / (32 * e) * 32; }

template <class F> cudaError_t allow_shared(F fn, size_t bytes) {
    if (bytes <= 48 * 1024) return cudaSuccess;
    return cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
}

template <class T, class TY, int V, bool SHIFT> cudaError_t forward_as(const ForwardParams& q, cudaStream_t s) {
    ForwardParams p = q;
    const int n = p.cols, reach = n + (SHIFT ? V - 1 : 0);
    // entry by entry there are no registers for 32
    const bool wide = reach > (V == 1 ? 8192 : 32768);
    const int e = V == 1 || (reach <= 8192 && static_cast<long long>(p.rows) * group_of(n, 8) < kFull) ? 8 : 32;
    p.group = wide ? 1024 : group_of(reach, e);
    const int per = std::max(1, 256 / p.group);
    int ctas = (p.rows - 1) / per + 1;
    size_t smem = 0;
    if (SHIFT) {
        smem = static_cast<size_t>(n / V + 1) * V * 4;
        ctas = std::min<int>(ctas, 152 * std::max<int>(1, std::min<size_t>(2048 / (p.group * per), (200 << 10) / smem)));
    }
    const auto fn = wide ? k_norm<T, TY, V, 0, false> : e == 8 ? k_norm<T, TY, V, 8, SHIFT> : k_norm<T, TY, V, V == 1 ? 8 : 32, SHIFT>;
    const cudaError_t err = allow_shared(fn, smem);
    if (err != cudaSuccess) return err;
    return launch(fn, dim3(ctas), dim3(p.group * per), smem, s, 1, p);
}

template <class T, class TY> cudaError_t forward_of(ForwardParams p, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    Lines l(V);
    l.add(p.x, p.ldx, sizeof(T)).add(p.r, p.ldr, sizeof(T)).add(p.h, p.ldh, sizeof(T)).add(p.y, p.ldy, sizeof(TY));
    if (l.aligned() && reinterpret_cast<uintptr_t>(p.gain) % 16 == 0) return forward_as<T, TY, V, false>(p, s);
    p.phase = l.phase;
    p.pitch = l.pitch;
    return l.ok && p.cols <= 32000 ? forward_as<T, TY, V, true>(p, s) : forward_as<T, TY, 1, false>(p, s);
}

struct BackwardShape {
    int entries, group, per, ctas;
};

// v: entries of an access (1: of rows whose lines differ); shift: rows in their own lines
BackwardShape backward_shape(int rows, int n, int v, bool shift) {
    BackwardShape b;
    const int reach = n + (shift ? v - 1 : 0);
    const bool few = reach <= 4096 && (v == 1 || static_cast<long long>(rows) * group_of(n, 8) < kFull / 2);
    b.entries = few ? 8 : v == 1 || reach > 16384 ? 0 : 32;
    b.group = b.entries == 0 ? 1024 : group_of(reach, b.entries);
    b.per = shift ? 1 : std::max(1, 128 / b.group);
    int resident = b.entries == 0 ? 1 : std::max(1, (b.entries == 32 ? 512 : 1536) / (b.group * b.per));
    if (shift) resident = std::max(1, std::min(std::min(16, resident), (200 << 10) / (8 * (n + v))));
    const long long need = (static_cast<long long>(rows) - 1) / b.per + 1;
    b.ctas = static_cast<int>(std::min<long long>(need, 152LL * resident));
    return b;
}

template <class T, class TY, int V, bool SHIFT> cudaError_t backward_as(const BackwardParams& q, int& ctas, cudaStream_t s) {
    BackwardParams p = q;
    const BackwardShape b = backward_shape(p.rows, p.cols, V, SHIFT);
    const bool wide = b.entries == 0;
    p.group = b.group;
    ctas = b.ctas;
    const size_t one = static_cast<size_t>(p.cols / V + 1) * V * 4;
    const bool shift = SHIFT && !wide;
    const size_t smem = shift ? 2 * one : wide || b.per > 1 ? static_cast<size_t>(p.cols) * 4 : 0;
    const auto fn = wide             ? k_norm_backward<T, TY, V, 0, false>
                    : b.entries == 8 ? k_norm_backward<T, TY, V, 8, SHIFT>
                                     : k_norm_backward<T, TY, V, V == 1 ? 8 : 32, SHIFT>;
    const cudaError_t e = allow_shared(fn, smem);
    if (e != cudaSuccess) return e;
    return launch(fn, dim3(b.ctas), dim3(b.group * b.per), smem, s, 1, p);
}

template <class T, class TY> cudaError_t backward_of(BackwardParams p, int& ctas, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    Lines l(V);
    l.add(p.h, p.ldh, sizeof(T)).add(p.dy, p.lddy, sizeof(TY)).add(p.dh, p.lddh, sizeof(T)).add(p.dx, p.lddx, sizeof(T));
    if (l.aligned() && reinterpret_cast<uintptr_t>(p.gain) % 16 == 0) return backward_as<T, TY, V, false>(p, ctas, s);
    p.phase = l.phase;
    p.pitch = l.pitch;
    return l.ok && p.cols + V <= 16384 ? backward_as<T, TY, V, true>(p, ctas, s) : backward_as<T, TY, 1, false>(p, ctas, s);
}

}  // namespace

cudaError_t launch_norm(const NormForward& a, cudaStream_t s, int64_t* launches) {
    const ForwardParams p{a.x, a.r, a.h, a.y, a.gain, a.rstd, a.ldx, a.ldr, a.ldh, a.ldy, a.rows, a.cols, 0, a.eps, 0, 0};
    ++*launches;
    if (a.dtype == MOARA_DTYPE_BF16)
        return a.y_dtype == MOARA_DTYPE_BF16 ? forward_of<bf16, bf16>(p, s) : forward_of<bf16, float>(p, s);
    return a.y_dtype == MOARA_DTYPE_BF16 ? forward_of<float, bf16>(p, s) : forward_of<float, float>(p, s);
}

// The most of any form that the rows may take.
int norm_partials(int rows, int cols) {
    int most = 0;
    for (int v : {1, 4, 8})
        for (bool shift : {false, true})
            if (!(shift && v == 1)) most = std::max(most, backward_shape(rows, cols, v, shift).ctas);
    return most;
}

cudaError_t launch_norm_backward(const NormBackward& a, cudaStream_t s, int64_t* launches) {
    const BackwardParams p{a.dy,  a.h,    a.dh,   a.dx,   a.gain, a.rstd, a.partials, a.lddy,
                           a.ldh, a.lddh, a.lddx, a.rows, a.cols, 0,      0,          0};
    int ctas = 0;
    ++*launches;
    cudaError_t e;
    if (a.dtype == MOARA_DTYPE_BF16)
        e = a.dy_dtype == MOARA_DTYPE_BF16 ? backward_of<bf16, bf16>(p, ctas, s) : backward_of<bf16, float>(p, ctas, s);
    else
        e = a.dy_dtype == MOARA_DTYPE_BF16 ? backward_of<float, bf16>(p, ctas, s) : backward_of<float, float>(p, ctas, s);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch(k_norm_gain, dim3((a.cols - 1) / 32 + 1), dim3(512), 0, s, 1, static_cast<const float*>(a.partials), ctas,
                  a.cols, a.dgain);
}

}  // namespace moara
