// C entries of the operators beside the projected step: AdamW over many
// tensors, the norm of many gradients, MXFP4 operands and products.  Contracts
// are in moara.h; every argument is checked before the first launch.
#include <climits>
#include <cmath>

#include "ctx.h"
#include "ops.h"

using moara::align_up;
using moara::aligned16;
using moara::cuda_fail;
using moara::DeviceGuard;
using moara::fail;

namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool float_type(int dtype) { return dtype == MOARA_DTYPE_F32 || dtype == MOARA_DTYPE_BF16; }

size_t type_size(int dtype) { return dtype == MOARA_DTYPE_BF16 ? 2 : 4; }

// Chunks of n entries, or -1 when a launch cannot number them.
long long chunks_of(int64_t n, int chunk) {
    const long long c = n / chunk + (n % chunk != 0);
    return c <= INT_MAX ? c : -1;
}

int check_moments(moara_ctx* ctx, int i, const moara_adamw_tensor& t) {
    if (t.n < 0) return fail(ctx, MOARA_ERR_SHAPE, "tensor %d: n must be >= 0", i);
    if (chunks_of(t.n, moara::kAdamChunk) < 0) return fail(ctx, MOARA_ERR_SHAPE, "tensor %d: n is too large", i);
    if (t.state_dtype != MOARA_DTYPE_F32 && t.state_dtype != MOARA_DTYPE_BLOCK8)
        return fail(ctx, MOARA_ERR_INVALID_ARG, "tensor %d: state_dtype must be MOARA_DTYPE_F32 or MOARA_DTYPE_BLOCK8", i);
    if (t.n == 0) return MOARA_OK;
    if (t.exp_avg == nullptr || t.exp_avg_sq == nullptr)
        return fail(ctx, MOARA_ERR_INVALID_ARG, "tensor %d: a moment is NULL", i);
    if (t.state_dtype == MOARA_DTYPE_F32) {
        if (!aligned(t.exp_avg, 4) || !aligned(t.exp_avg_sq, 4))
            return fail(ctx, MOARA_ERR_ALIGN, "tensor %d: a moment is not aligned to its type", i);
    } else {
        if (t.exp_avg_scale == nullptr || t.exp_avg_sq_scale == nullptr)
            return fail(ctx, MOARA_ERR_INVALID_ARG, "tensor %d: 8-bit moments need their scales", i);
        if (!aligned(t.exp_avg_scale, 4) || !aligned(t.exp_avg_sq_scale, 4))
            return fail(ctx, MOARA_ERR_ALIGN, "tensor %d: a scale array is not aligned to its type", i);
    }
    return MOARA_OK;
}

int check_adamw(moara_ctx* ctx, int i, const moara_adamw_tensor& t, float lr) {
    const int rc = check_moments(ctx, i, t);
    if (rc != MOARA_OK) return rc;
    if (!float_type(t.param_dtype) || !float_type(t.grad_dtype))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "tensor %d: param and grad are fp32 or bf16", i);
    if (t.param_bf16 != nullptr && t.param_dtype != MOARA_DTYPE_F32)
        return fail(ctx, MOARA_ERR_INVALID_ARG, "tensor %d: a bf16 copy needs an fp32 param", i);
    if (!(t.weight_decay >= 0.0f) || !std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale) ||
        !std::isfinite(lr * t.lr_scale * t.weight_decay))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "tensor %d: weight_decay must be finite and >= 0, lr_scale finite", i);
    if (t.n == 0) return MOARA_OK;
    if (t.param == nullptr || t.grad == nullptr)
        return fail(ctx, MOARA_ERR_INVALID_ARG, "tensor %d: param or grad is NULL", i);
    if (!aligned(t.param, type_size(t.param_dtype)) || !aligned(t.grad, type_size(t.grad_dtype)) ||
        !aligned(t.param_bf16, 2))
        return fail(ctx, MOARA_ERR_ALIGN, "tensor %d: param, grad or param_bf16 is not aligned to its type", i);
    return MOARA_OK;
}

int check_matrix(moara_ctx* ctx, const char* what, int rows, int cols) {
    if (rows < 1 || cols < 1) return fail(ctx, MOARA_ERR_SHAPE, "%s: rows and columns must be >= 1", what);
    // indexes run up to a CTA's share behind the last row and column
    if (rows > INT_MAX - 2048 || cols > INT_MAX - 2048 ||
        static_cast<long long>(moara::fp4_tiles(rows)) * moara::fp4_tiles(cols) > INT_MAX / 64)
        return fail(ctx, MOARA_ERR_SHAPE, "%s: the matrix is too large", what);
    return MOARA_OK;
}

int check_strided(moara_ctx* ctx, const char* what, const void* p, int dtype, int cols, int64_t ld) {
    if (!float_type(dtype)) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s must be fp32 or bf16", what);
    if (p == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s is NULL", what);
    if (!aligned(p, type_size(dtype))) return fail(ctx, MOARA_ERR_ALIGN, "%s is not aligned to its type", what);
    if (ld < cols) return fail(ctx, MOARA_ERR_SHAPE, "%s: the row pitch is below the number of columns", what);
    return MOARA_OK;
}

int check_operand(moara_ctx* ctx, const char* what, const void* q, const void* sf) {
    if (q == nullptr || sf == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s: q or sf is NULL", what);
    if (!aligned16(q) || !aligned16(sf)) return fail(ctx, MOARA_ERR_ALIGN, "%s: q or sf is not 16-byte aligned", what);
    return MOARA_OK;
}

int check_product(moara_ctx* ctx, int M, int N, int K, const void* bq, const void* bsf, const void* D, int d_dtype,
                  int64_t ldd) {
    if (ctx->tc == nullptr) return fail(ctx, MOARA_ERR_UNSUPPORTED, "no tensor-core state on this device");
    int rc = check_matrix(ctx, "A", M, K);
    if (rc == MOARA_OK) rc = check_matrix(ctx, "B", N, K);
    if (rc == MOARA_OK) rc = check_matrix(ctx, "D", M, N);
    if (rc == MOARA_OK) rc = check_operand(ctx, "B", bq, bsf);
    if (rc == MOARA_OK) rc = check_strided(ctx, "D", D, d_dtype, N, ldd);
    return rc;
}

// The operand of A between its quantisation and its product.
size_t linear_workspace(int M, int K) {
    return moara::fp4_quantizes(M) ? 0 : align_up(moara::fp4_q_bytes(M, K), 256) + moara::fp4_sf_bytes(M, K);
}

}  // namespace

extern "C" {

int moara_adamw_step(moara_ctx* ctx, int count, const moara_adamw_tensor* tensors, const moara_adamw_hparams* hp,
                     int64_t t, float lr, const float* grad_scale, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    if (hp == nullptr || count < 0 || (count > 0 && tensors == nullptr))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "hparams or tensors is NULL, or count is negative");
    if (!(hp->beta1 >= 0.0f && hp->beta1 < 1.0f) || !(hp->beta2 >= 0.0f && hp->beta2 < 1.0f))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "betas must lie in [0, 1)");
    if (!(hp->eps >= 0.0f) || !std::isfinite(hp->eps))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (t < 1) return fail(ctx, MOARA_ERR_INVALID_ARG, "t must be >= 1");
    if (!std::isfinite(lr)) return fail(ctx, MOARA_ERR_INVALID_ARG, "lr must be finite");
    if (!aligned(grad_scale, 4)) return fail(ctx, MOARA_ERR_ALIGN, "grad_scale is not aligned to its type");
    for (int i = 0; i < count; ++i) {
        const int rc = check_adamw(ctx, i, tensors[i], lr);
        if (rc != MOARA_OK) return rc;
    }
    DeviceGuard g(ctx->device);
    const double bc1 = 1.0 - std::pow(static_cast<double>(hp->beta1), static_cast<double>(t));
    const double bc2 = 1.0 - std::pow(static_cast<double>(hp->beta2), static_cast<double>(t));
    moara::AdamBatch b;
    b.b1 = hp->beta1;
    b.b2 = hp->beta2;
    b.c1 = static_cast<float>(1.0 - static_cast<double>(hp->beta1));
    b.c2 = static_cast<float>(1.0 - static_cast<double>(hp->beta2));
    b.rbc2 = static_cast<float>(1.0 / std::sqrt(bc2));
    b.eps = hp->eps;
    b.scale = grad_scale;
    long long entries = 0;
    for (int i = 0; i < count; ++i) entries += tensors[i].n < moara::kAdamMany ? tensors[i].n : moara::kAdamMany;
    b.chunk8 = entries < moara::kAdamMany ? moara::kAdamChunk : moara::kAdamLong;
    long long chunks = 0;
    b.count = 0;
    auto flush = [&]() -> cudaError_t {
        if (b.count == 0) return cudaSuccess;
        b.start[b.count] = static_cast<uint32_t>(chunks);
        const cudaError_t e = moara::launch_adamw(b, static_cast<cudaStream_t>(stream), &ctx->launches);
        b.count = 0;
        chunks = 0;
        return e;
    };
    for (int i = 0; i < count; ++i) {
        const moara_adamw_tensor& d = tensors[i];
        if (d.n == 0) continue;
        const long long c = chunks_of(d.n, d.state_dtype == MOARA_DTYPE_BLOCK8 ? b.chunk8 : moara::kAdamChunk);
        if (b.count == moara::kAdamTensors || chunks + c > INT_MAX) {
            const cudaError_t e = flush();
            if (e != cudaSuccess) return cuda_fail(ctx, e, "AdamW launch");
        }
        moara::AdamTensor& x = b.t[b.count];
        x.n = d.n;
        x.p = d.param;
        x.g = d.grad;
        x.copy = d.param_bf16;
        x.m = d.exp_avg;
        x.v = d.exp_avg_sq;
        x.ms = d.exp_avg_scale;
        x.vs = d.exp_avg_sq_scale;
        const double l = static_cast<double>(lr) * d.lr_scale;
        x.keep = static_cast<float>(1.0 - l * d.weight_decay);
        x.step = static_cast<float>(l / bc1);
        x.key = moara::adamw_key(hp->seed, d.id, t);
        x.kind = (d.param_dtype == MOARA_DTYPE_BF16 ? moara::kAdamParamBf16 : 0u) |
                 (d.grad_dtype == MOARA_DTYPE_BF16 ? moara::kAdamGradBf16 : 0u) |
                 (d.state_dtype == MOARA_DTYPE_BLOCK8 ? moara::kAdamBlock8 : 0u);
        if (aligned16(d.param) && aligned16(d.grad) && aligned16(d.param_bf16) && aligned16(d.exp_avg) &&
            aligned16(d.exp_avg_sq))
            x.kind |= moara::kAdamVector;
        b.start[b.count++] = static_cast<uint32_t>(chunks);
        chunks += c;
    }
    const cudaError_t e = flush();
    if (e != cudaSuccess) return cuda_fail(ctx, e, "AdamW launch");
    return MOARA_OK;
}

int moara_adamw_moments(moara_ctx* ctx, int count, const moara_adamw_tensor* tensors, float* const* exp_avg,
                        float* const* exp_avg_sq, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    if (count < 0 || (count > 0 && (tensors == nullptr || exp_avg == nullptr || exp_avg_sq == nullptr)))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "a NULL array, or count is negative");
    for (int i = 0; i < count; ++i) {
        const int rc = check_moments(ctx, i, tensors[i]);
        if (rc != MOARA_OK) return rc;
        if (!aligned(exp_avg[i], 4) || !aligned(exp_avg_sq[i], 4))
            return fail(ctx, MOARA_ERR_ALIGN, "tensor %d: an output is not aligned to its type", i);
    }
    DeviceGuard g(ctx->device);
    moara::MomentBatch b;
    b.count = 0;
    long long chunks = 0;
    for (int i = 0; i <= count; ++i) {
        const long long c = i < count ? chunks_of(tensors[i].n, moara::kAdamChunk) : 0;
        if (b.count > 0 && (i == count || b.count == moara::kMomentTensors || chunks + c > INT_MAX)) {
            b.start[b.count] = static_cast<uint32_t>(chunks);
            const cudaError_t e = moara::launch_moments(b, static_cast<cudaStream_t>(stream), &ctx->launches);
            if (e != cudaSuccess) return cuda_fail(ctx, e, "moments launch");
            b.count = 0;
            chunks = 0;
        }
        if (i == count || c == 0) continue;
        const moara_adamw_tensor& d = tensors[i];
        b.t[b.count] = moara::MomentTensor{d.n, d.exp_avg, d.exp_avg_sq, d.exp_avg_scale, d.exp_avg_sq_scale,
                                           exp_avg[i], exp_avg_sq[i], d.state_dtype == MOARA_DTYPE_BLOCK8};
        b.start[b.count++] = static_cast<uint32_t>(chunks);
        chunks += c;
    }
    return MOARA_OK;
}

// The workspace: a ticket in the first 16 bytes, then each launch's partial sums.
int moara_grad_norm_workspace_bytes(int count, size_t* out) {
    if (out == nullptr || count < 0) return MOARA_ERR_INVALID_ARG;
    const size_t launches = count > 0 ? (static_cast<size_t>(count) - 1) / moara::kNormTensors + 1 : 1;
    *out = 16 + launches * moara::kGradCtas * sizeof(double);
    return MOARA_OK;
}

int moara_grad_norm(moara_ctx* ctx, int count, const void* const* G, const int64_t* n, const int* dtype,
                    float max_norm, const float* extra_sq, float* out, void* workspace, size_t workspace_bytes,
                    void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    if (count < 0 || out == nullptr || (count > 0 && (G == nullptr || n == nullptr || dtype == nullptr)))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "a NULL array or output, or count is negative");
    if (std::isnan(max_norm)) return fail(ctx, MOARA_ERR_INVALID_ARG, "max_norm is not a number");
    if (!aligned(out, 4) || !aligned(extra_sq, 4))
        return fail(ctx, MOARA_ERR_ALIGN, "out or extra_sq is not aligned to its type");
    long long total = 0;
    for (int i = 0; i < count; ++i) {
        if (n[i] < 0) return fail(ctx, MOARA_ERR_SHAPE, "gradient %d: n must be >= 0", i);
        if (!float_type(dtype[i])) return fail(ctx, MOARA_ERR_INVALID_ARG, "gradient %d must be fp32 or bf16", i);
        if (n[i] > 0 && G[i] == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "gradient %d is NULL", i);
        if (!aligned(G[i], type_size(dtype[i])))
            return fail(ctx, MOARA_ERR_ALIGN, "gradient %d is not aligned to its type", i);
        const long long c = chunks_of(n[i], moara::kGradChunk);
        total = c < 0 ? LLONG_MAX : total + c;
        if (c < 0 || total > INT_MAX) return fail(ctx, MOARA_ERR_SHAPE, "the gradients are too large");
    }
    size_t need = 0;
    moara_grad_norm_workspace_bytes(count, &need);
    if (workspace == nullptr || workspace_bytes < need)
        return fail(ctx, MOARA_ERR_WORKSPACE, "the norm needs %zu bytes of workspace", need);
    if (!aligned16(workspace)) return fail(ctx, MOARA_ERR_ALIGN, "workspace is not 16-byte aligned");
    DeviceGuard g(ctx->device);
    moara::NormBatch b;
    b.max_norm = max_norm;
    b.extra = extra_sq;
    b.out = out;
    b.ticket = static_cast<unsigned int*>(workspace);
    b.partials = reinterpret_cast<double*>(static_cast<char*>(workspace) + 16);
    b.first = 0;
    for (int i = 0;;) {
        b.count = 0;
        b.chunks = 0;
        for (; i < count && b.count < moara::kNormTensors; ++i) {
            if (n[i] == 0) continue;
            moara::NormTensor& t = b.t[b.count++];
            t.g = G[i];
            t.n = n[i];
            t.start = b.chunks;
            t.kind = (dtype[i] == MOARA_DTYPE_BF16 ? moara::kAdamGradBf16 : 0u) | (aligned16(G[i]) ? moara::kAdamVector : 0u);
            b.chunks += static_cast<uint32_t>(chunks_of(n[i], moara::kGradChunk));
        }
        b.last = i == count;
        const int ctas = static_cast<int>(b.chunks < 1 ? 1 : b.chunks < moara::kGradCtas ? b.chunks : moara::kGradCtas);
        const cudaError_t e = moara::launch_grad_norm(b, ctas, static_cast<cudaStream_t>(stream), &ctx->launches);
        if (e != cudaSuccess) return cuda_fail(ctx, e, "gradient norm launch");
        b.first += ctas;
        if (b.last) return MOARA_OK;
    }
}

int moara_fp4_bytes(int rows, int cols, size_t* q_bytes, size_t* sf_bytes) {
    if (q_bytes == nullptr || sf_bytes == nullptr) return MOARA_ERR_INVALID_ARG;
    if (rows < 1 || cols < 1) return MOARA_ERR_SHAPE;
    *q_bytes = moara::fp4_q_bytes(rows, cols);
    *sf_bytes = moara::fp4_sf_bytes(rows, cols);
    return MOARA_OK;
}

int moara_fp4_quantize(moara_ctx* ctx, const void* X, int dtype, int rows, int cols, int64_t ld, void* q, void* sf,
                       void* qt, void* sft, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    int rc = check_matrix(ctx, "X", rows, cols);
    if (rc == MOARA_OK) rc = check_strided(ctx, "X", X, dtype, cols, ld);
    if (rc != MOARA_OK) return rc;
    if (q == nullptr && sf == nullptr && qt == nullptr && sft == nullptr)
        return fail(ctx, MOARA_ERR_INVALID_ARG, "no output is given");
    if (q != nullptr || sf != nullptr) rc = check_operand(ctx, "by rows", q, sf);
    if (rc == MOARA_OK && (qt != nullptr || sft != nullptr)) rc = check_operand(ctx, "by columns", qt, sft);
    if (rc != MOARA_OK) return rc;
    DeviceGuard g(ctx->device);
    const cudaError_t e = moara::launch_fp4_quantize(X, dtype, rows, cols, ld, q, sf, qt, sft,
                                                     static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "quantisation launch");
    return MOARA_OK;
}

int moara_fp4_dequantize(moara_ctx* ctx, const void* q, const void* sf, int rows, int cols, void* out, int dtype,
                         int64_t ldo, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    int rc = check_matrix(ctx, "the operand", rows, cols);
    if (rc == MOARA_OK) rc = check_operand(ctx, "the operand", q, sf);
    if (rc == MOARA_OK) rc = check_strided(ctx, "out", out, dtype, cols, ldo);
    if (rc != MOARA_OK) return rc;
    DeviceGuard g(ctx->device);
    const cudaError_t e = moara::launch_fp4_dequantize(q, sf, rows, cols, out, dtype, ldo,
                                                       static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "operand values launch");
    return MOARA_OK;
}

int moara_fp4_product(moara_ctx* ctx, int M, int N, int K, const void* a_q, const void* a_sf, const void* b_q,
                      const void* b_sf, void* D, int d_dtype, int64_t ldd, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    int rc = check_product(ctx, M, N, K, b_q, b_sf, D, d_dtype, ldd);
    if (rc == MOARA_OK) rc = check_operand(ctx, "A", a_q, a_sf);
    if (rc != MOARA_OK) return rc;
    DeviceGuard g(ctx->device);
    const moara::Fp4Product p{M, N, K, a_q, a_sf, b_q, b_sf, D, d_dtype, ldd, nullptr, 0, 0, moara::tc_wait_limit(ctx->tc)};
    const cudaError_t e = moara::launch_fp4_product(p, false, ctx->d_status, static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "product launch");
    return MOARA_OK;
}

int moara_fp4_linear_workspace_bytes(int M, int N, int K, size_t* out) {
    if (out == nullptr) return MOARA_ERR_INVALID_ARG;
    if (M < 1 || N < 1 || K < 1) return MOARA_ERR_SHAPE;
    *out = linear_workspace(M, K);
    return MOARA_OK;
}

int moara_fp4_linear(moara_ctx* ctx, int M, int N, int K, const void* X, int x_dtype, int64_t ldx, const void* b_q,
                     const void* b_sf, void* D, int d_dtype, int64_t ldd, void* workspace, size_t workspace_bytes,
                     void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    int rc = check_product(ctx, M, N, K, b_q, b_sf, D, d_dtype, ldd);
    if (rc == MOARA_OK) rc = check_strided(ctx, "X", X, x_dtype, K, ldx);
    if (rc != MOARA_OK) return rc;
    const size_t need = linear_workspace(M, K);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need))
        return fail(ctx, MOARA_ERR_WORKSPACE, "the product needs %zu bytes of workspace", need);
    if (need > 0 && !aligned16(workspace)) return fail(ctx, MOARA_ERR_ALIGN, "workspace is not 16-byte aligned");
    DeviceGuard g(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    moara::Fp4Product p{M, N, K, nullptr, nullptr, b_q, b_sf, D, d_dtype, ldd, X, x_dtype, ldx, moara::tc_wait_limit(ctx->tc)};
    cudaError_t e = cudaSuccess;
    const bool apart = !moara::fp4_quantizes(M);
    if (apart) {
        char* q = static_cast<char*>(workspace);
        char* sf = q + align_up(moara::fp4_q_bytes(M, K), 256);
        e = moara::launch_fp4_quantize(X, x_dtype, M, K, ldx, q, sf, nullptr, nullptr, s, &ctx->launches);
        if (e != cudaSuccess) return cuda_fail(ctx, e, "quantisation launch");
        p.aq = q;
        p.asf = sf;
        p.X = nullptr;
    }
    e = moara::launch_fp4_product(p, apart, ctx->d_status, s, &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "product launch");
    return MOARA_OK;
}

}  // extern "C"
