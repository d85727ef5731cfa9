// Launchers of the operators of a decoder's layers (norm.cu, fp4.cu, attention.cu,
// loss.cu); arguments are checked by layers_api.cpp.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/moara.h"

namespace moara {

// -------------------------------------------------------- root-mean-square norm
constexpr int kNormCols = 49152;       // widest row: a column's sum of the gain's gradient in shared memory

struct NormForward {
    int rows, cols;
    const void* x;
    const void* r;         // residual, or null
    int dtype;             // of x, r and h
    const float* gain;
    float eps;
    void* h;               // null without a residual
    void* y;               // null: h and rstd alone
    int y_dtype;
    float* rstd;
    int64_t ldx, ldr, ldh, ldy;
};
cudaError_t launch_norm(const NormForward& a, cudaStream_t s, int64_t* launches);

struct NormBackward {
    int rows, cols;
    const void* dy;
    int dy_dtype;
    const void* h;
    int dtype;             // of h, dh and dx
    const float* gain;
    const float* rstd;
    const void* dh;        // gradient of h from elsewhere, or null
    void* dx;
    float* dgain;
    float* partials;       // norm_partials(rows, cols) rows of cols sums
    int64_t lddy, ldh, lddh, lddx;
};
// CTAs of the backward pass, each of which leaves a row of sums for the gain's gradient.
int norm_partials(int rows, int cols);
cudaError_t launch_norm_backward(const NormBackward& a, cudaStream_t s, int64_t* launches);

// y = h * rstd * gain as MXFP4 operands, as launch_fp4_quantize
cudaError_t launch_norm_quantize(const void* h, int dtype, int rows, int cols, int64_t ld, const float* rstd,
                                 const float* gain, void* q, void* sf, void* qt, void* sft, cudaStream_t s,
                                 int64_t* launches);

// ---------------------------------------------------------------- policy loss
struct PolicyLoss {
    int rows, vocab;
    const void* z;
    int dtype;
    int64_t ldz;
    const int64_t* target;
    const float* old_logp;
    const float* ref_logp; // null without the KL term
    const float* adv;
    const float* weight;   // null: 1 / rows
    float low, high, kl;   // the ratio's bounds, the KL term's factor
    float* sums;
    float* logp;
    void* dz;              // null: no gradient
    int64_t lddz;
    void* terms;           // policy_loss_workspace(rows) bytes
    int* status;
    long long wait_limit;
};
size_t policy_loss_workspace(int rows);
cudaError_t launch_policy_loss(const PolicyLoss& a, cudaStream_t s, int64_t* launches);

// ------------------------------------------------------------------ attention
// One of a sequence's tiles (of 128 rows, or of 256): the sequence's first token and length, and
// its first entry in the list.
struct AttentionTile {
    int begin, length, first, pad;
};

struct Attention {
    const void* q;
    const void* k;
    const void* v;
    void* out;
    void* rest;            // null: not wanted
    float* lse;            // heads x tokens
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;       // pitches in entries
    int tokens, heads, kv_heads, dim;
    float scale;
    const AttentionTile* pairs;    // of 256 rows
    int n_pairs;
    long long work;        // pairs of a tile of queries and one of keys that it sees, of a head
    int* status;
    long long wait_limit;
};
cudaError_t launch_attention(const Attention& a, cudaStream_t s, int64_t* launches);

struct AttentionGrad {
    const void* dout;
    const void* q;
    const void* k;
    const void* v;
    const void* out;
    const void* rest;      // or null
    const float* lse;
    float* delta;          // heads x tokens, and one more word
    void* dq;
    void* dk;
    void* dv;
    int64_t do_row, do_head, q_row, q_head, k_row, k_head, v_row, v_head;
    int tokens, heads, kv_heads, dim;
    float scale;
    const AttentionTile* tiles;    // of 128 rows
    int n_tiles;
    int longest;           // tiles of the longest sequence
    long long work;        // pairs of a query tile and a key tile that it sees
    int* status;
    long long wait_limit;
};
cudaError_t launch_attention_backward(const AttentionGrad& a, cudaStream_t s, int64_t* launches);

}  // namespace moara
