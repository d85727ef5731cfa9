// The context behind the C entry points, and what their translation units
// share: error texts, alignment checks, the device guard.
#pragma once

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>
#include <vector>

#include "internal.h"
#include "tc.h"

struct moara_ctx {
    int device = 0;
    moara_hparams hp{};
    std::vector<moara_module_desc> mods;
    std::vector<moara::ModDev> moddev;
    std::vector<int64_t> refresh_count;
    moara::ModDev* d_mods = nullptr;
    int cap = 0;
    int* d_status = nullptr;
    int* h_status = nullptr;
    void* refresh_ws = nullptr;
    size_t refresh_ws_bytes = 0;
    std::string last_error;
    int64_t launches = 0;
    moara::TcState* tc = nullptr;
    // host-gradient step: two device staging buffers, a copy stream, events
    void* stage[2] = {nullptr, nullptr};
    size_t stage_bytes = 0;
    cudaStream_t copy_stream = nullptr;
    cudaEvent_t copy_done[2] = {nullptr, nullptr};
    cudaEvent_t compute_done[2] = {nullptr, nullptr};
    // per-kernel CUDA-event timing (moara_profile_enable)
    bool prof = false;
    struct Rec { int phase; cudaEvent_t a, b; };
    std::vector<Rec> recs;
    std::vector<cudaEvent_t> free_events;
    cudaEvent_t open_event = nullptr;
    double prof_ms[MOARA_NUM_PHASES] = {0};
    int64_t prof_n[MOARA_NUM_PHASES] = {0};
    // alignment diagnostic: three double accumulators per module of a call
    double* align_acc = nullptr;
    int align_cap = 0;
    // global-norm clipping: {total norm, coefficient}, per-CTA partial sums,
    // the caller's extra sum of squares
    float* d_clip = nullptr;
    double* d_clip_part = nullptr;
    int clip_part_cap = 0;
    const float* clip_extra = nullptr;
};

namespace moara {

inline int fail(moara_ctx* ctx, int code, const char* fmt, ...) {
    if (ctx != nullptr) {
        char buf[512];
        va_list ap;
        va_start(ap, fmt);
        std::vsnprintf(buf, sizeof(buf), fmt, ap);
        va_end(ap);
        ctx->last_error = buf;
    }
    return code;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct DeviceGuard {
    int prev = -1;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        if (prev != dev) cudaSetDevice(dev);
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

inline int cuda_fail(moara_ctx* ctx, cudaError_t e, const char* what) {
    return fail(ctx, MOARA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

}  // namespace moara
