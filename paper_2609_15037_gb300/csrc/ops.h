// Launchers of the operators beside the projected step (adamw.cu, fp4.cu,
// fp4_product.cu); arguments are checked by ops_api.cpp.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/moara.h"

namespace moara {

// ------------------------------------------------------------------- AdamW
// Tensors of a launch, all in its parameter block (at most 32764 bytes).  Calls of few
// tensors take a smaller block: copying 32 KB is 1.5 us of a launch's 4.5.
constexpr int kAdamTensors = 360, kAdamFew = 72;
constexpr int kAdamChunk = 2048;       // entries that one CTA takes at a time
// Chunk of 8-bit moments in a call with many entries: a CTA's search for its tensor and
// its addresses are spread over eight blocks per warp.  Below kAdamMany entries the
// GPU is not full with so many entries a CTA.
constexpr int kAdamLong = 8 * kAdamChunk;
constexpr long long kAdamMany = 152LL * 8 * kAdamLong;

struct AdamTensor {
    long long n;
    void* p;
    const void* g;
    uint16_t* copy;
    void* m;
    void* v;
    float* ms;
    float* vs;
    float keep;            // 1 - lr wd
    float step;            // lr / (1 - beta1^t)
    uint32_t key;          // of the random bits of (seed, id, t)
    uint32_t kind;         // kAdam* flags
};
constexpr uint32_t kAdamParamBf16 = 1, kAdamGradBf16 = 2, kAdamBlock8 = 4, kAdamVector = 8;

struct AdamCall {
    int count, chunk8;
    float b1, b2, c1, c2;              // betas, 1 - betas
    float rbc2;                        // 1 / sqrt(1 - beta2^t)
    float eps;
    const float* scale;
};

template <int CAP> struct AdamBatchOf : AdamCall {
    uint32_t start[CAP + 1];           // first chunk of each tensor
    AdamTensor t[CAP];
};
using AdamBatch = AdamBatchOf<kAdamTensors>;
static_assert(sizeof(AdamBatch) <= 32764, "the batch fits the kernel parameter space");

// key of the random bits of one tensor at one step
uint32_t adamw_key(uint64_t seed, uint32_t id, int64_t t);
cudaError_t launch_adamw(const AdamBatch& b, cudaStream_t s, int64_t* launches);

struct MomentTensor {
    long long n;
    const void* m;
    const void* v;
    const float* ms;
    const float* vs;
    float* om;
    float* ov;
    int block8;
};
constexpr int kMomentTensors = 480;
struct MomentBatch {
    MomentTensor t[kMomentTensors];
    uint32_t start[kMomentTensors + 1];
    int count;
};
static_assert(sizeof(MomentBatch) <= 32764, "the batch fits the kernel parameter space");

cudaError_t launch_moments(const MomentBatch& b, cudaStream_t s, int64_t* launches);

// ------------------------------------------------------------- gradient norm
constexpr int kNormTensors = 1200, kNormFew = 72;
constexpr int kGradChunk = 8192;       // entries a CTA takes at a time
constexpr int kGradCtas = 152 * 4;     // most CTAs of a launch, and its partial sums
struct NormTensor {
    const void* g;
    long long n;
    uint32_t start;                    // first chunk
    uint32_t kind;                     // kAdamGradBf16, kAdamVector
};
struct NormCall {
    int count;
    uint32_t chunks;
    int first;                         // partial sums of earlier launches of the call
    int last;                          // whether this launch finishes the call
    float max_norm;
    const float* extra;
    float* out;
    double* partials;
    unsigned int* ticket;
};

template <int CAP> struct NormBatchOf : NormCall {
    NormTensor t[CAP];
};
using NormBatch = NormBatchOf<kNormTensors>;
static_assert(sizeof(NormBatch) <= 32764, "the batch fits the kernel parameter space");

cudaError_t launch_grad_norm(const NormBatch& b, int ctas, cudaStream_t s, int64_t* launches);

// ------------------------------------------------------------------- MXFP4
inline int fp4_blocks(int cols) { return (cols - 1) / 32 + 1; }              // 32-column blocks of a row
inline int fp4_tiles(int x) { return (x - 1) / 128 + 1; }
inline size_t fp4_q_bytes(int rows, int cols) { return static_cast<size_t>(rows) * fp4_blocks(cols) * 16; }
inline size_t fp4_sf_bytes(int rows, int cols) { return static_cast<size_t>(fp4_tiles(rows)) * fp4_tiles(cols) * 512; }

cudaError_t launch_fp4_quantize(const void* X, int dtype, int rows, int cols, int64_t ld, void* q, void* sf, void* qt,
                                void* sft, cudaStream_t s, int64_t* launches);
cudaError_t launch_fp4_dequantize(const void* q, const void* sf, int rows, int cols, void* out, int dtype, int64_t ldo,
                                  cudaStream_t s, int64_t* launches);

struct Fp4Product {
    int M, N, K;
    const void* aq;
    const void* asf;
    const void* bq;
    const void* bsf;
    void* D;
    int dtype;
    int64_t ldd;
    const void* X;         // A as fp32 or bf16 rows, quantised on the way (aq, asf unused), or null
    int x_dtype;
    int64_t ldx;
    long long wait_limit;  // clock cycles of a bounded wait before it gives up
};
// Whether a product of M rows can quantise A itself.
bool fp4_quantizes(int M);
// early: the launch in front wrote A and nothing else, and lets this one begin beside it.
// status: device word for MOARA_ERR_DEVICE_TIMEOUT
cudaError_t launch_fp4_product(const Fp4Product& p, bool early, int* status, cudaStream_t s, int64_t* launches);

}  // namespace moara
