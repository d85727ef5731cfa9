// Root-mean-square norm of rows, with the residual's addition, and its gradients.
//   h = x + r (rounded to its type), s = 1 / sqrt(mean h^2 + eps), y = (h s) g
//   dx = dh + s (d - n mean(d n)) with d = dy g, n = h s;   dg = sum over rows of dy n
// DRAM-bound: each array is read or written once.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

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
    // beside an infinite sum there is NaN
    __device__ __forceinline__ float value() const { return fabsf(hi) < INFINITY ? hi + lo : hi; }
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

// Squares of an access: each lane of a pair adds up its own in fp32 (three roundings at most),
// and the group's total goes to the sums.
template <class T, int V> __device__ __forceinline__ void add_squares(Sums& sums, const Raw<T, V>& v) {
    uint64_t q = 0;
#pragma unroll
    for (int e = 0; e < (V + 1) / 2; ++e) {
        const uint64_t a = v.pair(e);
        q = e == 0 ? mul2(a, a) : fma2(a, a, q);
    }
    sums.add(q);
}

// 1 / sqrt(sum / n + eps): a Newton step on the residual of rsqrtf, in two numbers
// throughout, so that it adds one rounding to the sum's error.  A mean that is too small for the step's squares (or
// for fp32's normal numbers: no eps, and next to nothing in a long row) is taken 2^100 times as large.
__device__ __forceinline__ float inverse_rms(Sum s, int n, float eps) {
    if (!(s.hi < INFINITY)) return rsqrtf(s.hi);             // lo is NaN beside it
    const bool small = s.hi < 0x1p-40f && eps < 0x1p-60f;
    if (small) {
        s.hi *= 0x1p100f;
        s.lo *= 0x1p100f;
        eps *= 0x1p100f;
    }
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
    const float e = fmaf(-a, p, 1.0f) - (a * pl + al * p), root = fmaf(0.5f * r, e, r);
    return small ? root * 0x1p50f : root;
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

// The same where columns c .. c + V - 1 all exist: from the first one's class on, entry e is e
// classes further, and a place further where the classes end.
template <int V> struct Classes {
    int at, pitch, wrap, back;
    __device__ __forceinline__ Classes(int c, int n) {
        pitch = n / V + 1;
        at = c % V * pitch + c / V;
        wrap = V - c % V;
        back = V * pitch - 1;
    }
    __device__ __forceinline__ int of(int e) const { return at + e * pitch - (e >= wrap ? back : 0); }
};

template <bool SHIFT, int V>
__device__ __forceinline__ void gain_whole(const float* gain, const float* staged, int c, int n, Raw<float, V>& g) {
    if constexpr (SHIFT) {
        const Classes<V> k(c, n);
#pragma unroll
        for (int e = 0; e < V; ++e) g.w[e] = __float_as_uint(staged[k.of(e)]);
    } else {
        g.load(gain + c);
    }
}

template <int V> __device__ __forceinline__ void add_whole(float* columns, int c, int n, int e, uint64_t u, uint64_t v) {
    const Classes<V> k(c, n);
    float a[2], b[2];
    split(u, a[0], a[1]);
    split(v, b[0], b[1]);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        float& sum = columns[k.of(2 * e + y)];
        sum = fmaf(a[y], b[y], sum);
    }
}

// Few rows: a group of threads takes a row and keeps it in registers, E = 8 entries a thread.
// E = 0: rows of more than 1024 threads' entries, or whose arrays lie differently in their lines,
// are read again, from L2, once their sum is known.  1554 x 18083 fp32: 106 us, its
// gradients 133 (entry by entry 175 and 202; 18080 columns 93 and 126).
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
                    add_squares(sums, f[j]);
                    if (h != nullptr) f[j].store_at(h, c, n);
                }
            }
        } else if (real) {
            for (int c = i * V - off; c < n; c += group * V) {
                take(c, f[0]);
                add_squares(sums, f[0]);
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
            for (int c = i * V - off; c < n; c += group * V) {
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
                for (int c = i * V - off; c < n; c += group * V) {
                    a[0].load_at(dy, c, n);
                    b[0].load_at(h, c, n);
                    product(c, 0);
                }
            }
        }
        const Sum dot = group_sum(dots.both(), group, parts[turn] + mine * (group >> 5));
        if (SHIFT) __syncwarp();                 // a group of one warp has no other barrier
        if (!real) continue;
        const float mean = dot.value() * inv;
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
            for (int c = i * V - off; c < n; c += group * V) {
                a[0].load_at(dy, c, n);
                b[0].load_at(h, c, n);
                if (dh != nullptr) w[0].load_at(dh, c, n);
                put(c, 0, mean, [&](int e, uint64_t u, uint64_t v) {
                    add_column<V>(columns, c + 2 * e, n, u, v, [&](int k) { return SHIFT ? column<V>(k, n) : k; });
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

// ---------------------------------------------------------------------------
// Many rows.  A thread has four accesses of a row in each array, and its
// copies of the next rows run into shared memory of its own while it works on this one: no
// registers wait for DRAM, and what a thread reads it has copied itself, so that a row's sum is the
// only barrier.  A row's first and last line are read where they lie if they are not whole.
// 16384 x 4096 bf16 with the residual: 95 us (floor 79; with loads into registers 107).  Its gradients: 115 us, and 6 for the
// gain's sums; an earlier form with 32 entries a thread in registers took 108 by a profiler's clock where this takes 117, so
// that the copies gain nothing there.
// ---------------------------------------------------------------------------
template <int BYTES> __device__ __forceinline__ void copy_async(void* to, const void* from) {
    const uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(to));
    if constexpr (BYTES == 8) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(a), "l"(from) : "memory");
    } else {
#pragma unroll
        for (int e = 0; e < BYTES; e += 16)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(a + e), "l"(static_cast<const char*>(from) + e) : "memory");
    }
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest N groups of this thread's copies have landed.
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

constexpr int kAccesses = 4;

// Where a thread's copy of access j lies: beside its neighbours' (64 bytes a thread in a row of
// their own, in swizzled order, took 137 us where this takes 98).
template <int BYTES> __device__ __forceinline__ int place_of(int j) { return j * static_cast<int>(blockDim.x) * BYTES; }

// f(j, c, whole) for each access of a thread in a row that begins `off` entries into its first
// line; whole: none of its entries lies outside the row, known for all four of most threads.
template <int V, int A, class F> __device__ __forceinline__ void accesses(int i, int group, int off, int n, F f) {
    const int c0 = i * V - off, step = group * V;
    if (c0 >= 0 && c0 + (A - 1) * step + V <= n) {
#pragma unroll
        for (int j = 0; j < A; ++j) f(j, c0 + j * step, std::true_type());
    } else {
#pragma unroll
        for (int j = 0; j < A; ++j) {
            const int c = c0 + j * step;
            if (c >= n) continue;
            if (c >= 0 && c + V <= n) f(j, c, std::true_type());
            else f(j, c, std::false_type());
        }
    }
}

template <class T, class TY, int V, int STAGES, bool SHIFT>
__global__ void __launch_bounds__(1024) k_norm_many(const ForwardParams p) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ float2 parts[2][32];
    using R = Raw<T, V>;
    constexpr int P = V / 2, OWN = kAccesses * R::BYTES;     // of an array's copies, a thread
    const int group = p.group, per = blockDim.x / group, mine = threadIdx.x / group, i = threadIdx.x % group;
    const int n = p.cols, array = blockDim.x * OWN;
    uint8_t* const slots = dynamic + threadIdx.x * R::BYTES; // of x; of r `array` bytes further
    float* const staged = reinterpret_cast<float*>(dynamic + STAGES * 2 * array);
    pdl_begin();
    if (SHIFT) stage_gain<V>(staged, p.gain, n);
    const long long step = static_cast<long long>(gridDim.x) * per;
    auto off_of = [&](long long row) { return SHIFT ? static_cast<int>((p.phase + row % V * p.pitch) % V) : 0; };
    auto prefetch = [&](long long row, int stage) {
        if (row < p.rows) {
            const T* x = static_cast<const T*>(p.x) + row * p.ldx;
            const T* r = static_cast<const T*>(p.r) + row * p.ldr;
            uint8_t* const to = slots + stage * 2 * array;
            accesses<V, kAccesses>(i, group, off_of(row), n, [&](int j, int c, auto whole) {
                if constexpr (!decltype(whole)::value) return;
                copy_async<R::BYTES>(to + place_of<R::BYTES>(j), x + c);
                if (p.r != nullptr) copy_async<R::BYTES>(to + array + place_of<R::BYTES>(j), r + c);
            });
        }
        copies_commit();
    };
    const long long first = static_cast<long long>(blockIdx.x) * per + mine;
#pragma unroll
    for (int k = 0; k + 1 < STAGES; ++k) prefetch(first + k * step, k);
    int turn = 0, stage = 0;
    for (long long row = first; row - mine < p.rows; row += step, turn ^= 1) {
        prefetch(row + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
        const bool real = row < p.rows;
        const T* x = static_cast<const T*>(p.x) + row * p.ldx;
        const T* r = p.r == nullptr ? nullptr : static_cast<const T*>(p.r) + row * p.ldr;
        T* h = p.r == nullptr ? nullptr : static_cast<T*>(p.h) + row * p.ldh;
        TY* y = p.y == nullptr ? nullptr : static_cast<TY*>(p.y) + row * p.ldy;
        const int off = off_of(row);
        const uint8_t* const from = slots + stage * 2 * array;
        R f[kAccesses];                                      // h
        Sums sums;
        copies_wait<STAGES - 1>();
        if (real)
            accesses<V, kAccesses>(i, group, off, n, [&](int j, int c, auto whole) {
                R w;
                if constexpr (decltype(whole)::value) {
                    f[j].load(reinterpret_cast<const T*>(from + place_of<R::BYTES>(j)));
                    if (r != nullptr) w.load(reinterpret_cast<const T*>(from + array + place_of<R::BYTES>(j)));
                } else {
                    f[j].load_at(x, c, n);
                    if (r != nullptr) w.load_at(r, c, n);
                }
                if (r != nullptr) {
                    add_raw(f[j], w);
                    if constexpr (decltype(whole)::value) f[j].store(h + c);
                    else f[j].store_at(h, c, n);
                }
                add_squares(sums, f[j]);
            });
        if (++stage == STAGES) stage = 0;
        const Sum s = group_sum(sums.both(), group, parts[turn] + mine * (group >> 5));
        if (!real) continue;
        const float rstd = inverse_rms(s, n, p.eps);
        if (i == 0) p.rstd[row] = rstd;
        if (y == nullptr) continue;
        accesses<V, kAccesses>(i, group, off, n, [&](int j, int c, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            Raw<float, V> g;
            Raw<TY, V> o;
            if constexpr (WHOLE) gain_whole<SHIFT, V>(p.gain, staged, c, n, g);
            else gain_at<SHIFT, V>(p.gain, staged, c, n, g);
#pragma unroll
            for (int e = 0; e < P; ++e) o.set(e, mul2(mul2(f[j].pair(e), both(rstd)), g.pair(e)));
            if constexpr (WHOLE) o.store(y + c);
            else o.store_at(y, c, n);
        });
    }
}

// The same for the gradients: dy and h are read from shared memory in both passes, dh in the
// second.  SHIFT: the columns' sums are in shared memory too, one group a CTA; a column's sum has
// another thread from row to row, behind the barrier of the row's mean.
template <class T, class TY, int V, int A, bool SHIFT>
__global__ void __launch_bounds__(512) k_norm_backward_many(const BackwardParams p) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ float2 parts[2][32];
    using R = Raw<T, V>;
    using RY = Raw<TY, V>;
    constexpr int P = V / 2, STAGES = 2, OWN = A * R::BYTES, OWN_Y = A * RY::BYTES;
    const int group = p.group, per = blockDim.x / group, mine = threadIdx.x / group, i = threadIdx.x % group;
    const int n = p.cols, threads = blockDim.x, all = (2 * OWN + OWN_Y) * threads;        // bytes of a stage
    uint8_t* const slots = dynamic + threadIdx.x * R::BYTES; // of h; of dh behind all threads' h
    uint8_t* const slots_y = dynamic + 2 * OWN * threads + threadIdx.x * RY::BYTES;
    float* const columns = reinterpret_cast<float*>(dynamic + STAGES * all);
    float* const staged = columns + (n / V + 1) * V;         // SHIFT: the gain
    if (SHIFT) {
        for (int c = threadIdx.x; c < n; c += threads) columns[column<V>(c, n)] = 0.0f;
        __syncthreads();
    }
    pdl_begin();
    if (SHIFT) stage_gain<V>(staged, p.gain, n);
    const long long step = static_cast<long long>(gridDim.x) * per;
    auto off_of = [&](long long row) { return SHIFT ? static_cast<int>((p.phase + row % V * p.pitch) % V) : 0; };
    auto prefetch = [&](long long row, int stage) {
        if (row < p.rows) {
            const TY* dy = static_cast<const TY*>(p.dy) + row * p.lddy;
            const T* h = static_cast<const T*>(p.h) + row * p.ldh;
            const T* dh = static_cast<const T*>(p.dh) + row * p.lddh;
            accesses<V, A>(i, group, off_of(row), n, [&](int j, int c, auto whole) {
                if constexpr (!decltype(whole)::value) return;
                copy_async<RY::BYTES>(slots_y + stage * all + place_of<RY::BYTES>(j), dy + c);
                copy_async<R::BYTES>(slots + stage * all + place_of<R::BYTES>(j), h + c);
                if (p.dh != nullptr) copy_async<R::BYTES>(slots + stage * all + OWN * threads + place_of<R::BYTES>(j), dh + c);
            });
        }
        copies_commit();
    };
    uint64_t acc[A][P] = {};
    const long long first = static_cast<long long>(blockIdx.x) * per + mine;
    prefetch(first, 0);
    int turn = 0;
    const float inv = 1.0f / static_cast<float>(n);
    for (long long row = first; row - mine < p.rows; row += step, turn ^= 1) {
        prefetch(row + step, turn ^ 1);
        const bool real = row < p.rows;
        const TY* dy = static_cast<const TY*>(p.dy) + row * p.lddy;
        const T* h = static_cast<const T*>(p.h) + row * p.ldh;
        const T* dh = p.dh == nullptr ? nullptr : static_cast<const T*>(p.dh) + row * p.lddh;
        T* dx = static_cast<T*>(p.dx) + row * p.lddx;
        const int off = off_of(row);
        const float rstd = real ? p.rstd[row] : 0.0f;
        const uint64_t scale = both(rstd);
        auto take = [&](int j, int c, auto whole, RY& a, R& b, Raw<float, V>& g) {
            if constexpr (decltype(whole)::value) {
                a.load(reinterpret_cast<const TY*>(slots_y + turn * all + place_of<RY::BYTES>(j)));
                b.load(reinterpret_cast<const T*>(slots + turn * all + place_of<R::BYTES>(j)));
            } else {
                a.load_at(dy, c, n);
                b.load_at(h, c, n);
            }
            if constexpr (decltype(whole)::value) gain_whole<SHIFT, V>(p.gain, staged, c, n, g);
            else gain_at<SHIFT, V>(p.gain, staged, c, n, g);
        };
        Sums dots;
        copies_wait<1>();
        if (real)
            accesses<V, A>(i, group, off, n, [&](int j, int c, auto whole) {
                RY a;
                R b;
                Raw<float, V> g;
                take(j, c, whole, a, b, g);
                uint64_t q = 0;
#pragma unroll
                for (int e = 0; e < P; ++e) q = fma2(mul2(a.pair(e), g.pair(e)), mul2(b.pair(e), scale), q);
                dots.add(q);
            });
        const Sum dot = group_sum(dots.both(), group, parts[turn] + mine * (group >> 5));
        if (SHIFT) __syncwarp();                 // a group of one warp has no other barrier
        if (!real) continue;
        const uint64_t mean = both(-dot.value() * inv);
        accesses<V, A>(i, group, off, n, [&](int j, int c, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            RY a;
            R b, w, o;
            Raw<float, V> g;
            take(j, c, whole, a, b, g);
            if (dh != nullptr) {
                if constexpr (WHOLE) w.load(reinterpret_cast<const T*>(slots + turn * all + OWN * threads + place_of<R::BYTES>(j)));
                else w.load_at(dh, c, n);
            }
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const uint64_t u = a.pair(e), v = mul2(b.pair(e), scale);
                if constexpr (SHIFT && WHOLE) add_whole<V>(columns, c, n, e, u, v);
                else if constexpr (SHIFT) add_column<V>(columns, c + 2 * e, n, u, v, [&](int k) { return column<V>(k, n); });
                else acc[j][e] = fma2(u, v, acc[j][e]);
                const uint64_t d = fma2(v, mean, mul2(u, g.pair(e)));
                o.set(e, dh != nullptr ? fma2(scale, d, w.pair(e)) : mul2(scale, d));
            }
            if constexpr (WHOLE) o.store(dx + c);
            else o.store_at(dx, c, n);
        });
    }
    float* out = p.partials + static_cast<long long>(blockIdx.x) * n;
    if constexpr (SHIFT) {
        __syncthreads();
        for (int c = threadIdx.x; c < n; c += threads) out[c] = columns[column<V>(c, n)];
    } else {
        // the groups' sums, in order
        for (int k = 0; k < per; ++k) {
            if (per > 1) __syncthreads();
            if (mine != k) continue;
#pragma unroll
            for (int j = 0; j < A; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int c = (j * group + i) * V + e;
                    if (c >= n) continue;
                    float x, y;
                    split(acc[j][e / 2], x, y);
                    const float own = e & 1 ? y : x, sum = k == 0 ? own : columns[c] + own;
                    if (k + 1 < per) columns[c] = sum;
                    else out[c] = sum;
                }
        }
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
    if (lane % 16 == 0 && blockIdx.x * 32 + k < n) dgain[blockIdx.x * 32 + k] = t.value();
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

constexpr size_t kShared = 222 << 10;

// A launch that may take up to kShared bytes of shared memory.  The kernel's limit is set to that once per
// device: it belongs to the function, and one set to a call's own bytes may be lowered by another thread's
// call before the launch.
template <auto FN, class P> cudaError_t launch_wide(int ctas, int threads, size_t smem, cudaStream_t s, const P& p) {
    if (smem > 40 * 1024) {
        static std::atomic<uint64_t> done{0};
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess) return e;
        if (device >= 64 || !(done.load() >> device & 1)) {
            e = cudaFuncSetAttribute(FN, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kShared));
            if (e != cudaSuccess) return e;
            if (device < 64) done.fetch_or(1ull << device);
        }
    }
    return launch(FN, dim3(ctas), dim3(threads), smem, s, 1, p);
}

template <class T, class TY, int V, bool SHIFT> cudaError_t forward_as(const ForwardParams& q, cudaStream_t s) {
    ForwardParams p = q;
    const int n = p.cols, reach = n + (SHIFT ? V - 1 : 0);
    const size_t gain = SHIFT ? static_cast<size_t>(n / V + 1) * V * 4 : 0;
    const bool few = reach <= 8192 && static_cast<long long>(p.rows) * group_of(reach, 8) < kFull;
    if constexpr (V > 1) {
        if (!few && reach <= 1024 * kAccesses * V) {
            p.group = group_of(reach, kAccesses * V);
            const int per = std::max(1, 128 / p.group), threads = p.group * per;
            const size_t stage = static_cast<size_t>(threads) * 2 * kAccesses * V * sizeof(T);
            const int resident = std::max(1, std::min(16, 512 / threads));
            const size_t room = kShared / resident, fixed = 1024 + gain;
            const int stages = room < fixed ? 0 : static_cast<int>(std::min<size_t>(3, (room - fixed) / stage));
            const size_t smem = stages * stage + gain;
            const int ctas = std::min((p.rows - 1) / per + 1, 152 * resident);
            if (stages >= 3) return launch_wide<k_norm_many<T, TY, V, 3, SHIFT>>(ctas, threads, smem, s, p);
            if (stages == 2) return launch_wide<k_norm_many<T, TY, V, 2, SHIFT>>(ctas, threads, smem, s, p);
            if (stages == 1) return launch_wide<k_norm_many<T, TY, V, 1, SHIFT>>(ctas, threads, smem, s, p);
            // none beside the gain of a wide row
        }
    }
    const bool wide = reach > 8192;
    p.group = wide ? 1024 : group_of(reach, 8);
    const int per = std::max(1, 256 / p.group);
    int ctas = (p.rows - 1) / per + 1;
    if (SHIFT) ctas = std::min<int>(ctas, 152 * std::max<int>(1, std::min<size_t>(2048 / (p.group * per), kShared / (gain + 1024))));
    return wide ? launch_wide<k_norm<T, TY, V, 0, SHIFT>>(ctas, p.group * per, gain, s, p)
                : launch_wide<k_norm<T, TY, V, 8, SHIFT>>(ctas, p.group * per, gain, s, p);
}

template <class T, class TY> cudaError_t forward_of(ForwardParams p, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    Lines l(V);
    l.add(p.x, p.ldx, sizeof(T)).add(p.r, p.ldr, sizeof(T)).add(p.h, p.ldh, sizeof(T)).add(p.y, p.ldy, sizeof(TY));
    if (l.aligned() && reinterpret_cast<uintptr_t>(p.gain) % 16 == 0) return forward_as<T, TY, V, false>(p, s);
    p.phase = l.phase;
    p.pitch = l.pitch;
    return l.ok ? forward_as<T, TY, V, true>(p, s) : forward_as<T, TY, 1, false>(p, s);
}

struct BackwardShape {
    int entries, accesses, group, per, ctas;
    size_t smem;
    bool fits;             // into shared memory
};

// Entries of a thread: 8 for few rows, 4 accesses of v for many, 0 for rows that are read again.
// v: entries of an access (1: of rows whose lines differ); shift: rows in their own lines; bytes of an
// access's copies of a row's three arrays.
BackwardShape backward_shape(int rows, int n, int v, bool shift, int bytes) {
    BackwardShape b;
    // rows in their own lines need more shared memory: more threads share a row
    const int accesses = shift && n + v <= 512 * 2 * v ? 2 : kAccesses;
    const int reach = n + (shift ? v - 1 : 0);
    const size_t one = static_cast<size_t>(n / v + 1) * v * 4, extra = shift ? 2 * one : 0;
    const bool few = reach <= 4096 && (v == 1 || static_cast<long long>(rows) * group_of(reach, 8) < kFull / 2);
    const auto threads_of = [&](int entries) {
        b.group = group_of(reach, entries);
        b.per = shift ? 1 : std::max(1, 128 / b.group);
        return b.group * b.per;
    };
    b.fits = true;
    b.accesses = 0;
    int resident = 1;
    if (few) {
        b.entries = 8;
        const int threads = threads_of(8);
        resident = std::max(1, 1536 / threads);
        b.smem = shift ? extra : b.per > 1 ? static_cast<size_t>(n) * 4 : 0;
        if (shift) resident = std::max<int>(1, std::min<size_t>(std::min(16, resident), kShared / (extra + 1024)));
    } else {
        if (v > 1 && reach <= 512 * kAccesses * v) {
            const int threads = threads_of(accesses * v);
            b.accesses = accesses;
            b.smem = 2 * static_cast<size_t>(threads) * accesses * bytes + (shift ? extra : b.per > 1 ? one : 0);
            resident = std::max<int>(1, std::min<size_t>(std::min(16, (shift ? 1024 : 512) / threads), kShared / (b.smem + 1024)));
        }
        b.entries = b.accesses * v;
        if (b.entries == 0 || b.smem > kShared) {
            b.entries = b.accesses = 0;
            b.group = 1024;
            b.per = resident = 1;
            b.smem = shift ? extra : static_cast<size_t>(n) * 4;
            b.fits = b.smem <= kShared;
        }
    }
    const long long need = (static_cast<long long>(rows) - 1) / b.per + 1;
    b.ctas = static_cast<int>(std::min<long long>(need, 152LL * resident));
    return b;
}

template <class T, class TY, int V, bool SHIFT> cudaError_t backward_as(const BackwardParams& q, int& ctas, cudaStream_t s) {
    BackwardParams p = q;
    const BackwardShape b = backward_shape(p.rows, p.cols, V, SHIFT, V * (2 * sizeof(T) + sizeof(TY)));
    p.group = b.group;
    ctas = b.ctas;
    const int threads = b.group * b.per;
    if constexpr (SHIFT)
        if (b.accesses == 2) return launch_wide<k_norm_backward_many<T, TY, V, 2, SHIFT>>(ctas, threads, b.smem, s, p);
    if constexpr (V > 1)
        if (b.accesses > 0) return launch_wide<k_norm_backward_many<T, TY, V, kAccesses, SHIFT>>(ctas, threads, b.smem, s, p);
    return b.entries == 0 ? launch_wide<k_norm_backward<T, TY, V, 0, SHIFT>>(ctas, threads, b.smem, s, p)
                          : launch_wide<k_norm_backward<T, TY, V, 8, SHIFT>>(ctas, threads, b.smem, s, p);
}

template <class T, class TY> cudaError_t backward_of(BackwardParams p, int& ctas, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    Lines l(V);
    l.add(p.h, p.ldh, sizeof(T)).add(p.dy, p.lddy, sizeof(TY)).add(p.dh, p.lddh, sizeof(T)).add(p.dx, p.lddx, sizeof(T));
    if (l.aligned() && reinterpret_cast<uintptr_t>(p.gain) % 16 == 0) return backward_as<T, TY, V, false>(p, ctas, s);
    p.phase = l.phase;
    p.pitch = l.pitch;
    constexpr int BYTES = V * (2 * sizeof(T) + sizeof(TY));
    const bool fits = l.ok && backward_shape(p.rows, p.cols, V, true, BYTES).fits;
    return fits ? backward_as<T, TY, V, true>(p, ctas, s) : backward_as<T, TY, 1, false>(p, ctas, s);
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
            for (int bytes : {6, 8, 10, 12})
                if (!(shift && v == 1)) most = std::max(most, backward_shape(rows, cols, v, shift, v * bytes).ctas);
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
    // begins once the sums are there: CTAs that wait would take the places of some of the CTAs in
    // front, all of which have to be resident to share the rows evenly (16384 x 4096 bf16: 180 us instead of 117)
    return launch_if(false, k_norm_gain, dim3((a.cols - 1) / 32 + 1), dim3(512), 0, s, 1, static_cast<const float*>(a.partials), ctas,
                  a.cols, a.dgain);
}

}  // namespace moara
