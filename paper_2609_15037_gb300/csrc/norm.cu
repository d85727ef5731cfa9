// Root-mean-square norm of rows, with the residual's addition, and its gradients.
//   h = x + r (rounded to its type), s = 1 / sqrt(mean h^2 + eps), y = (h s) g
//   dx = dh + s (d - n mean(d n)) with d = dy g, n = h s;   dg = sum over rows of dy n
// DRAM-bound: each array is read or written once.
#include <cuda_bf16.h>

#include <algorithm>

#include "f32x2.cuh"
#include "launch.cuh"
#include "layers.h"

namespace moara {
namespace {

using bf16 = __nv_bfloat16;

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
    // entries 2e and 2e + 1; of a single one, it and a zero
    __device__ __forceinline__ uint64_t pair(int e) const {
        if constexpr (V == 1) return f32x2(__uint_as_float(sizeof(T) == 4 ? w[0] : w[0] << 16), 0.0f);
        else if constexpr (sizeof(T) == 4) return f32x2(__uint_as_float(w[2 * e]), __uint_as_float(w[2 * e + 1]));
        else return widen2(w[e]);
    }
    __device__ __forceinline__ void set(int e, uint64_t x) {
        float a, b;
        split(x, a, b);
        if constexpr (sizeof(T) == 4) {
            w[V == 1 ? 0 : 2 * e] = __float_as_uint(a);
            if constexpr (V > 1) w[2 * e + 1] = __float_as_uint(b);
        } else {
            w[e] = pack2(a, b);
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (BYTES == 2) {
            *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
        } else if constexpr (BYTES == 4) {
            *reinterpret_cast<uint32_t*>(p) = w[0];
        } else if constexpr (BYTES == 8) {
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int e = 0; e < WORDS; e += 4)
                *reinterpret_cast<uint4*>(p + e * 4 / static_cast<int>(sizeof(T))) = make_uint4(w[e], w[e + 1], w[e + 2], w[e + 3]);
        }
    }
    __device__ __forceinline__ void store_at(T* row, int c, int n) const {
        if (c >= 0 && c + V <= n) {
            store(row + c);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (c + e < 0 || c + e >= n) continue;
                if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(row)[c + e] = w[e];
                else reinterpret_cast<uint16_t*>(row)[c + e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
            }
        }
    }
};

// x + r, rounded once (two bf16 numbers at a time; what fp32 would round off first is never
// more than a trace below the larger one's last bit)
template <class T, int V> __device__ __forceinline__ void add_raw(Raw<T, V>& x, const Raw<T, V>& r) {
#pragma unroll
    for (int e = 0; e < Raw<T, V>::WORDS; ++e) {
        if constexpr (sizeof(T) == 4) x.w[e] = __float_as_uint(__uint_as_float(x.w[e]) + __uint_as_float(r.w[e]));
        else asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(x.w[e]) : "r"(x.w[e]), "r"(r.w[e]));
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

// Two of them beside one another.
struct Sums {
    uint64_t hi = 0, lo = 0;
    __device__ __forceinline__ void add(uint64_t x) {
        const uint64_t s = add2(hi, x), b = sub2(s, hi);
        lo = add2(lo, add2(sub2(hi, sub2(s, b)), sub2(x, b)));
        hi = s;
    }
    __device__ __forceinline__ Sum both() const {
        Sum a, b;
        split(hi, a.hi, b.hi);
        split(lo, a.lo, b.lo);
        a.add(b);
        return a;
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
__device__ __forceinline__ void gain_at(const float* gain, const float* staged, int c, int n, Raw<float, V>& g) {
    if constexpr (SHIFT) {
#pragma unroll
        for (int e = 0; e < V; ++e) g.w[e] = c + e >= 0 && c + e < n ? __float_as_uint(staged[column<V>(c + e, n)]) : 0u;
    } else {
        g.load_at(gain, c, n);
    }
}

// A group of threads takes a row and keeps it in registers, E entries a thread: 32 of bf16 or
// 16 of fp32, so that the sum over the group costs little beside them, or 8 where rows are too
// few to fill the GPU.  E = 0: a row of more than 1024 threads' entries is read again, from L2, once
// its sum is known.
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
        constexpr int P = (V + 1) / 2;                       // pairs of an access
        Raw<T, V> f[NV];                                     // h
        Sums sums;
        auto take = [&](int c, Raw<T, V>& v) {
            v.load_at(x, c, n);
            if (r != nullptr) {
                Raw<T, V> w;
                w.load_at(r, c, n);
                add_raw(v, w);
            }
        };
        auto square = [&](const Raw<T, V>& v) {
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const uint64_t a = v.pair(e), q = mul2(a, a);
                sums.add(q);
                // of bf16 entries the square is exact
                if (sizeof(T) == 4) sums.lo = add2(sums.lo, fma2(a, a, mul2(q, both(-1.0f))));
            }
        };
        auto put = [&](int c, const Raw<T, V>& v, float rstd) {
            Raw<float, V> g;
            Raw<TY, V> o;
            gain_at<SHIFT, V>(p.gain, staged, c, n, g);
#pragma unroll
            for (int e = 0; e < P; ++e) o.set(e, mul2(mul2(v.pair(e), both(rstd)), g.pair(e)));
            o.store_at(y, c, n);
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
                    if (h != nullptr) f[j].store_at(h, c, n);
                }
            }
        } else if (real) {
            for (int c = i * V; c < n; c += group * V) {
                take(c, f[0]);
                square(f[0]);
                if (h != nullptr) f[0].store_at(h, c, n);
            }
        }
        const Sum s = group_sum(sums.both(), group, parts[turn] + mine * (group >> 5));
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
                f[0].load_at(from, c, n);
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

// Columns c and c + 1 (V = 1: c alone) of the sums, where they exist.
template <int V, class At> __device__ __forceinline__ void add_column(float* columns, int c, int n, uint64_t u, uint64_t v, At at) {
    float a[2], b[2];
    split(u, a[0], a[1]);
    split(v, b[0], b[1]);
#pragma unroll
    for (int e = 0; e < (V == 1 ? 1 : 2); ++e)
        if (c + e >= 0 && c + e < n) columns[at(c + e)] = fmaf(a[e], b[e], columns[at(c + e)]);
}

// CTAs take rows a grid apart and leave their columns' sums of dy n.  E entries a thread
// stay in registers as they came, with the columns' sums; E = 0: rows of more than 512 threads'
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
    uint64_t acc[NV][(V + 1) / 2] = {};
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
        constexpr int P = (V + 1) / 2;
        float rstd = 0.0f;
        Sums dots;
        auto product = [&](int c, int j) {
            Raw<float, V> g;
            gain_at<SHIFT, V>(p.gain, staged, c, n, g);
            uint64_t q = 0;
#pragma unroll
            for (int e = 0; e < P; ++e) q = fma2(mul2(a[j].pair(e), g.pair(e)), mul2(b[j].pair(e), both(rstd)), q);
            dots.add(q);
        };
        // dx, and the columns' sums by `add`
        auto put = [&](int c, int j, float mean, auto add) {
            Raw<float, V> g;
            gain_at<SHIFT, V>(p.gain, staged, c, n, g);
            Raw<T, V> o;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const uint64_t u = a[j].pair(e), v = mul2(b[j].pair(e), both(rstd));
                add(e, u, v);
                const uint64_t d = fma2(v, both(-mean), mul2(u, g.pair(e)));
                o.set(e, dh != nullptr ? fma2(both(rstd), d, w[j].pair(e)) : mul2(both(rstd), d));
            }
            o.store_at(dx, c, n);
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
        const Sum dot = group_sum(dots.both(), group, parts[turn] + mine * (group >> 5));
        if (SHIFT) __syncwarp();                 // a group of one warp has no other barrier
        if (!real) continue;
        const float mean = (dot.hi + dot.lo) * inv;
        if constexpr (E > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * group + i) * V - off;
                if (c >= n) continue;
                put(c, j, mean, [&](int e, uint64_t u, uint64_t v) {
                    if constexpr (SHIFT) add_column<V>(columns, c + 2 * e, n, u, v, [&](int k) { return column<V>(k, n); });
                    else acc[j][e] = fma2(u, v, acc[j][e]);
                });
            }
        } else {
            for (int c = i * V; c < n; c += group * V) {
                a[0].load_at(dy, c, n);
                b[0].load_at(h, c, n);
                if (dh != nullptr) w[0].load_at(dh, c, n);
                put(c, 0, mean, [&](int e, uint64_t u, uint64_t v) {
                    add_column<V>(columns, c + 2 * e, n, u, v, [](int k) { return k; });
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
                    float x, y;
                    split(acc[j][e / 2], x, y);
                    const float mine_sum = e & 1 ? y : x, sum = k == 0 ? mine_sum : columns[c] + mine_sum;
                    if (k + 1 < per) columns[c] = sum;
                    else out[c] = sum;
                }
        }
    } else {
        __syncthreads();
        for (int c = threadIdx.x; c < n; c += blockDim.x) out[c] = columns[SHIFT ? column<V>(c, n) : c];
    }
}

// Column sums of the partial rows, in their order: 32 columns a CTA, 16 warps with four rows at a
// time share the rows; a lane has four columns.
__global__ void __launch_bounds__(512) k_norm_gain(const float* partials, int count, int n, float* dgain) {
    __shared__ float2 sums[64][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane % 8 * 4, r0 = w * 4 + lane / 8;
    pdl_begin();
    Sum s[4];
    const bool whole = n % 4 == 0;                           // rows begin on 16-byte lines
#pragma unroll 4
    for (int r = r0; r < count; r += 64) {
        const float* row = partials + static_cast<long long>(r) * n;
        float4 x = make_float4(0, 0, 0, 0);
        if (whole && c < n) {
            x = *reinterpret_cast<const float4*>(row + c);
        } else {
            if (c < n) x.x = row[c];
            if (c + 1 < n) x.y = row[c + 1];
            if (c + 2 < n) x.z = row[c + 2];
            if (c + 3 < n) x.w = row[c + 3];
        }
        s[0].add(x.x);
        s[1].add(x.y);
        s[2].add(x.z);
        s[3].add(x.w);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[r0][lane % 8 * 4 + e] = make_float2(s[e].hi, s[e].lo);
    __syncthreads();
    // two columns a warp, 16 lanes each with four of the 64 sums
    const int k = w * 2 + lane / 16;
    Sum t;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        Sum u;
        u.hi = sums[lane % 16 * 4 + e][k].x;
        u.lo = sums[lane % 16 * 4 + e][k].y;
        t.add(u);
    }
#pragma unroll
    for (int o = 8; o > 0; o /= 2) {
        Sum u;
        u.hi = __shfl_down_sync(0xffffffffu, t.hi, o);
        u.lo = __shfl_down_sync(0xffffffffu, t.lo, o);
        t.add(u);
    }
    if (lane % 16 == 0 && blockIdx.x * 32 + k < n) dgain[blockIdx.x * 32 + k] = t.hi + t.lo;
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
template <class T> constexpr int many = sizeof(T) == 2 ? 32 : 16;

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
    constexpr int MANY = V == 1 ? 8 : many<T>;
    const bool wide = reach > 1024 * MANY;
    const int e = reach <= 8192 && static_cast<long long>(p.rows) * group_of(n, 8) < kFull ? 8 : MANY;
    p.group = wide ? 1024 : group_of(reach, e);
    const int per = std::max(1, 256 / p.group);
    int ctas = (p.rows - 1) / per + 1;
    size_t smem = 0;
    if (SHIFT) {
        smem = static_cast<size_t>(n / V + 1) * V * 4;
        ctas = std::min<int>(ctas, 152 * std::max<int>(1, std::min<size_t>(2048 / (p.group * per), (200 << 10) / smem)));
    }
    const auto fn = wide ? k_norm<T, TY, V, 0, false> : e == 8 ? k_norm<T, TY, V, 8, SHIFT> : k_norm<T, TY, V, MANY, SHIFT>;
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
    return l.ok && p.cols + V <= 1024 * many<T> ? forward_as<T, TY, V, true>(p, s) : forward_as<T, TY, 1, false>(p, s);
}

struct BackwardShape {
    int entries, group, per, ctas;
};

// v: entries of an access (1: of rows whose lines differ); shift: rows in their own lines;
// most: entries of a thread
BackwardShape backward_shape(int rows, int n, int v, bool shift, int most) {
    BackwardShape b;
    const int reach = n + (shift ? v - 1 : 0);
    const bool few = reach <= 4096 && (v == 1 || static_cast<long long>(rows) * group_of(n, 8) < kFull / 2);
    b.entries = few ? 8 : v == 1 || reach > 512 * most ? 0 : most;
    b.group = b.entries == 0 ? 1024 : group_of(reach, b.entries);
    b.per = shift ? 1 : std::max(1, 128 / b.group);
    int resident = b.entries == 0 ? 1 : std::max(1, (b.entries == 8 ? 1536 : 512) / (b.group * b.per));
    if (shift) resident = std::max(1, std::min(std::min(16, resident), (200 << 10) / (8 * (n + v))));
    const long long need = (static_cast<long long>(rows) - 1) / b.per + 1;
    b.ctas = static_cast<int>(std::min<long long>(need, 152LL * resident));
    return b;
}

template <class T, class TY, int V, bool SHIFT> cudaError_t backward_as(const BackwardParams& q, int& ctas, cudaStream_t s) {
    BackwardParams p = q;
    constexpr int MANY = V == 1 ? 8 : many<T>;
    const BackwardShape b = backward_shape(p.rows, p.cols, V, SHIFT, MANY);
    const bool wide = b.entries == 0;
    p.group = b.group;
    ctas = b.ctas;
    const size_t one = static_cast<size_t>(p.cols / V + 1) * V * 4;
    const bool shift = SHIFT && !wide;
    const size_t smem = shift ? 2 * one : wide || b.per > 1 ? static_cast<size_t>(p.cols) * 4 : 0;
    const auto fn = wide             ? k_norm_backward<T, TY, V, 0, false>
                    : b.entries == 8 ? k_norm_backward<T, TY, V, 8, SHIFT>
                                     : k_norm_backward<T, TY, V, MANY, SHIFT>;
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
    return l.ok && p.cols + V <= 512 * many<T> ? backward_as<T, TY, V, true>(p, ctas, s) : backward_as<T, TY, 1, false>(p, ctas, s);
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
            if (!(shift && v == 1)) most = std::max(most, backward_shape(rows, cols, v, shift, v == 1 ? 8 : 4 * v).ctas);
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
