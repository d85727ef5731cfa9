// C entries of the operators of a decoder's layers: norm, attention, policy loss.
// Contracts are in moara.h; every argument is checked before the first launch.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <vector>

#include "ctx.h"
#include "layers.h"
#include "ops.h"

using moara::aligned16;
using moara::AttentionTile;
using moara::cuda_fail;
using moara::DeviceGuard;
using moara::fail;

namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool float_type(int dtype) { return dtype == MOARA_DTYPE_F32 || dtype == MOARA_DTYPE_BF16; }

int check_rows(moara_ctx* ctx, const char* what, const void* p, int dtype, int cols, int64_t ld) {
    if (!float_type(dtype)) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s must be fp32 or bf16", what);
    if (p == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s is NULL", what);
    if (!aligned(p, dtype == MOARA_DTYPE_BF16 ? 2 : 4)) return fail(ctx, MOARA_ERR_ALIGN, "%s is not aligned to its type", what);
    if (ld < cols) return fail(ctx, MOARA_ERR_SHAPE, "%s: the row pitch is below the number of columns", what);
    return MOARA_OK;
}

// Rows of a matrix in memory.
struct Span {
    const char* name;
    uintptr_t at;
    int64_t width, pitch;                        // bytes
    int rows;
    Span(const char* what, const void* p, int dtype, int rows_, int cols, int64_t ld)
        : name(what), at(reinterpret_cast<uintptr_t>(p)), width(cols * (dtype == MOARA_DTYPE_BF16 ? 2LL : 4LL)),
          pitch(ld * (dtype == MOARA_DTYPE_BF16 ? 2LL : 4LL)), rows(rows_) {
        if (rows == 1) pitch = width;
    }
    __int128 end() const { return static_cast<__int128>(at) + static_cast<__int128>(rows - 1) * pitch + width; }
};

// An output may be the input itself, entry by entry, or lie apart from it: rows are taken in no order.
int check_apart(moara_ctx* ctx, const Span& out, const Span& in) {
    if (in.at == 0 || out.at == 0 || out.end() <= static_cast<__int128>(in.at) || in.end() <= static_cast<__int128>(out.at)) return MOARA_OK;
    // columns beside one another in rows of the same pitch lie apart
    const Span &a = out.at <= in.at ? out : in, &b = out.at <= in.at ? in : out;
    const int64_t d = static_cast<int64_t>(b.at - a.at), off = d % a.pitch;
    const bool ok = a.pitch == b.pitch && ((d == 0 && a.width == b.width) || (off >= a.width && off + b.width <= a.pitch));
    return ok ? MOARA_OK : fail(ctx, MOARA_ERR_INVALID_ARG, "%s overlaps %s without being it", out.name, in.name);
}

int check_floats(moara_ctx* ctx, const char* what, const float* p) {
    if (p == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s is NULL", what);
    if (!aligned(p, 4)) return fail(ctx, MOARA_ERR_ALIGN, "%s is not aligned to its type", what);
    return MOARA_OK;
}

int check_norm_size(moara_ctx* ctx, int rows, int cols) {
    if (rows < 1 || cols < 1) return fail(ctx, MOARA_ERR_SHAPE, "rows and columns must be >= 1");
    if (rows > INT_MAX - 2048) return fail(ctx, MOARA_ERR_SHAPE, "too many rows");
    if (cols > moara::kNormCols) return fail(ctx, MOARA_ERR_UNSUPPORTED, "a row of at most %d columns is needed", moara::kNormCols);
    return MOARA_OK;
}

// wanted: whether Y is
int check_norm(moara_ctx* ctx, const moara::NormForward& a, bool wanted) {
    int rc = check_norm_size(ctx, a.rows, a.cols);
    if (rc == MOARA_OK && wanted) rc = check_rows(ctx, "Y", a.y, a.y_dtype, a.cols, a.ldy);
    if (rc == MOARA_OK) rc = check_rows(ctx, "X", a.x, a.dtype, a.cols, a.ldx);
    if (rc == MOARA_OK && (a.r != nullptr || a.h != nullptr)) {
        rc = check_rows(ctx, "R", a.r, a.dtype, a.cols, a.ldr);
        if (rc == MOARA_OK) rc = check_rows(ctx, "H", a.h, a.dtype, a.cols, a.ldh);
    }
    if (rc == MOARA_OK) rc = check_floats(ctx, "gain", a.gain);
    if (rc == MOARA_OK) rc = check_floats(ctx, "rstd", a.rstd);
    if (rc == MOARA_OK && !(a.eps >= 0.0f && a.eps < INFINITY)) rc = fail(ctx, MOARA_ERR_INVALID_ARG, "eps must be >= 0");
    if (rc != MOARA_OK) return rc;
    const Span x("X", a.x, a.dtype, a.rows, a.cols, a.ldx), r("R", a.r, a.dtype, a.rows, a.cols, a.ldr),
        h("H", a.h, a.dtype, a.rows, a.cols, a.ldh), y("Y", a.y, a.y_dtype, a.rows, a.cols, a.ldy);
    rc = check_apart(ctx, h, x);
    if (rc == MOARA_OK) rc = check_apart(ctx, h, r);
    for (const Span* in : {&x, &r, &h})
        if (rc == MOARA_OK) rc = check_apart(ctx, y, *in);
    return rc;
}

// Head pitches of a tensor of `heads` heads; a pitch that nothing is reached by may be anything.
int check_heads(moara_ctx* ctx, const char* what, const void* p, int64_t& row, int64_t& head, int tokens, int heads, int dim) {
    if (p == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s is NULL", what);
    if (!aligned16(p)) return fail(ctx, MOARA_ERR_ALIGN, "%s is not 16-byte aligned", what);
    if (heads == 1) head = dim;
    if (tokens == 1) row = std::max<int64_t>(dim, head);
    if (row <= 0 || head <= 0 || row % 8 != 0 || head % 8 != 0)
        return fail(ctx, MOARA_ERR_ALIGN, "%s: pitches that are positive multiples of 8 entries are needed", what);
    if (row >= int64_t{1} << 38 || head >= int64_t{1} << 38) return fail(ctx, MOARA_ERR_SHAPE, "%s: a pitch is too large", what);
    return MOARA_OK;
}

int check_out(moara_ctx* ctx, const char* what, const void* p) {
    if (p == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "%s is NULL", what);
    if (!aligned16(p)) return fail(ctx, MOARA_ERR_ALIGN, "%s is not 16-byte aligned", what);
    return MOARA_OK;
}

int check_attention(moara_ctx* ctx, const moara_sequences* seqs, int tokens, int heads, int kv_heads, int dim, float scale) {
    if (ctx->tc == nullptr) return fail(ctx, MOARA_ERR_UNSUPPORTED, "no tensor-core state on this device");
    if (seqs == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "seqs is NULL");
    if (seqs->n_tiles < 0 || seqs->n_pairs < 0 || seqs->tokens < 0)
        return fail(ctx, MOARA_ERR_INVALID_ARG, "seqs holds negative counts");
    if (heads < 1 || kv_heads < 1 || heads % kv_heads != 0)
        return fail(ctx, MOARA_ERR_SHAPE, "kv_heads must divide heads (%d and %d)", kv_heads, heads);
    if (tokens < seqs->tokens || tokens > INT_MAX - 512)
        return fail(ctx, MOARA_ERR_SHAPE, "%d tokens for sequences of %d", tokens, seqs->tokens);
    if (dim < 8 || dim > 128 || dim % 8 != 0)
        return fail(ctx, MOARA_ERR_UNSUPPORTED, "heads of 8, 16, .. 128 entries are needed, not %d", dim);
    if (!(scale > 0.0f && scale < INFINITY)) return fail(ctx, MOARA_ERR_INVALID_ARG, "scale must be positive");
    const long long rows = static_cast<long long>(tokens) * heads;
    if (static_cast<long long>(seqs->n_tiles) * heads > INT_MAX / 16 || seqs->work < 0 || rows / 16 > INT_MAX - 1)
        return fail(ctx, MOARA_ERR_SHAPE, "too many tokens and heads");
    if (seqs->n_tiles > 0) return check_out(ctx, "seqs->tiles", seqs->tiles);
    return MOARA_OK;
}

// {sum of the lengths, tiles, pairs}, or an error
int count_tiles(int count, const int* lengths, long long& tokens, long long& tiles, long long& pairs) {
    if (count < 0 || (count > 0 && lengths == nullptr)) return MOARA_ERR_INVALID_ARG;
    tokens = tiles = pairs = 0;
    for (int i = 0; i < count; ++i) {
        if (lengths[i] < 0) return MOARA_ERR_SHAPE;
        tokens += lengths[i];
        tiles += (static_cast<long long>(lengths[i]) + 127) / 128;
        pairs += (static_cast<long long>(lengths[i]) + 255) / 256;
    }
    return tokens > INT_MAX - 512 ? MOARA_ERR_SHAPE : MOARA_OK;
}

}  // namespace

extern "C" {

int moara_rms_norm(moara_ctx* ctx, int rows, int cols, const void* X, int64_t ldx, const void* R, int64_t ldr,
                   int x_dtype, const float* gain, float eps, void* H, int64_t ldh, void* Y, int y_dtype, int64_t ldy,
                   float* rstd, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    const moara::NormForward a{rows, cols, X, R, x_dtype, gain, eps, H, Y, y_dtype, rstd, ldx, ldr, ldh, ldy};
    const int rc = check_norm(ctx, a, true);
    if (rc != MOARA_OK) return rc;
    DeviceGuard g(ctx->device);
    const cudaError_t e = moara::launch_norm(a, static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "norm launch");
    return MOARA_OK;
}

int moara_rms_norm_quantize(moara_ctx* ctx, int rows, int cols, const void* X, int64_t ldx, const void* R, int64_t ldr,
                            int x_dtype, const float* gain, float eps, void* H, int64_t ldh, void* q, void* sf, void* qt,
                            void* sft, float* rstd, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    const moara::NormForward a{rows, cols, X, R, x_dtype, gain, eps, H, nullptr, x_dtype, rstd, ldx, ldr, ldh, cols};
    const int rc = check_norm(ctx, a, false);
    if (rc != MOARA_OK) return rc;
    if (static_cast<long long>(moara::fp4_tiles(rows)) * moara::fp4_tiles(cols) > INT_MAX / 64)
        return fail(ctx, MOARA_ERR_SHAPE, "the matrix is too large");
    if (q == nullptr && sf == nullptr && qt == nullptr && sft == nullptr)
        return fail(ctx, MOARA_ERR_INVALID_ARG, "no output is given");
    if ((q == nullptr) != (sf == nullptr) || (qt == nullptr) != (sft == nullptr))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "codes and scales are needed together");
    if (!aligned16(q) || !aligned16(sf) || !aligned16(qt) || !aligned16(sft))
        return fail(ctx, MOARA_ERR_ALIGN, "an operand is not 16-byte aligned");
    DeviceGuard g(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = moara::launch_norm(a, s, &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "norm launch");
    e = moara::launch_norm_quantize(R != nullptr ? H : X, x_dtype, rows, cols, R != nullptr ? ldh : ldx, rstd, gain, q, sf, qt,
                                    sft, s, &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "quantisation launch");
    return MOARA_OK;
}

int moara_rms_norm_backward_workspace_bytes(int rows, int cols, size_t* out) {
    if (out == nullptr) return MOARA_ERR_INVALID_ARG;
    if (rows < 1 || cols < 1) return MOARA_ERR_SHAPE;
    if (cols > moara::kNormCols) return MOARA_ERR_UNSUPPORTED;
    *out = static_cast<size_t>(moara::norm_partials(rows, cols)) * cols * sizeof(float);
    return MOARA_OK;
}

int moara_rms_norm_backward(moara_ctx* ctx, int rows, int cols, const void* dY, int dy_dtype, int64_t lddy,
                            const void* H, int h_dtype, int64_t ldh, const float* gain, const float* rstd,
                            const void* dH, int64_t lddh, void* dX, int64_t lddx, float* dgain, void* workspace,
                            size_t workspace_bytes, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    int rc = check_norm_size(ctx, rows, cols);
    if (rc == MOARA_OK) rc = check_rows(ctx, "dY", dY, dy_dtype, cols, lddy);
    if (rc == MOARA_OK) rc = check_rows(ctx, "H", H, h_dtype, cols, ldh);
    if (rc == MOARA_OK && dH != nullptr) rc = check_rows(ctx, "dH", dH, h_dtype, cols, lddh);
    if (rc == MOARA_OK) rc = check_rows(ctx, "dX", dX, h_dtype, cols, lddx);
    if (rc == MOARA_OK) rc = check_floats(ctx, "gain", gain);
    if (rc == MOARA_OK) rc = check_floats(ctx, "rstd", rstd);
    if (rc == MOARA_OK) rc = check_floats(ctx, "dgain", dgain);
    if (rc != MOARA_OK) return rc;
    const Span out("dX", dX, h_dtype, rows, cols, lddx);
    rc = check_apart(ctx, out, Span("dY", dY, dy_dtype, rows, cols, lddy));
    if (rc == MOARA_OK) rc = check_apart(ctx, out, Span("H", H, h_dtype, rows, cols, ldh));
    if (rc == MOARA_OK) rc = check_apart(ctx, out, Span("dH", dH, h_dtype, rows, cols, lddh));
    if (rc != MOARA_OK) return rc;
    size_t need = 0;
    moara_rms_norm_backward_workspace_bytes(rows, cols, &need);
    if (workspace == nullptr || workspace_bytes < need)
        return fail(ctx, MOARA_ERR_WORKSPACE, "the gradients need %zu bytes of workspace", need);
    if (!aligned16(workspace)) return fail(ctx, MOARA_ERR_ALIGN, "workspace is not 16-byte aligned");
    DeviceGuard g(ctx->device);
    const moara::NormBackward a{rows, cols, dY, dy_dtype, H, h_dtype, gain, rstd, dH, dX, dgain,
                                static_cast<float*>(workspace), lddy, ldh, lddh, lddx};
    const cudaError_t e = moara::launch_norm_backward(a, static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "norm gradient launch");
    return MOARA_OK;
}

int moara_sequences_bytes(int count, const int* lengths, size_t* out) {
    if (out == nullptr) return MOARA_ERR_INVALID_ARG;
    long long tokens, tiles, pairs;
    const int rc = count_tiles(count, lengths, tokens, tiles, pairs);
    if (rc == MOARA_OK) *out = static_cast<size_t>(tiles + pairs) * sizeof(AttentionTile);
    return rc;
}

// Pairs of tiles, then tiles, the longest sequences' first.
int moara_sequences_init(int count, const int* lengths, void* to, size_t bytes, moara_sequences* out) {
    if (out == nullptr) return MOARA_ERR_INVALID_ARG;
    long long tokens, tiles, pairs;
    const int rc = count_tiles(count, lengths, tokens, tiles, pairs);
    if (rc != MOARA_OK) return rc;
    const size_t need = static_cast<size_t>(tiles + pairs) * sizeof(AttentionTile);
    if (bytes < need || (need > 0 && to == nullptr)) return MOARA_ERR_WORKSPACE;
    *out = moara_sequences{nullptr, static_cast<int>(tokens), static_cast<int>(tiles), static_cast<int>(pairs), 0, 0};
    try {
        std::vector<AttentionTile> seqs;
        int begin = 0;
        for (int i = 0; i < count; begin += lengths[i++])
            if (lengths[i] > 0) seqs.push_back(AttentionTile{begin, lengths[i], 0, 0});
        std::stable_sort(seqs.begin(), seqs.end(), [](const AttentionTile& a, const AttentionTile& b) { return a.length > b.length; });
        AttentionTile* at = static_cast<AttentionTile*>(to);
        for (const int rows : {256, 128}) {
            int first = 0;
            for (AttentionTile s : seqs) {
                const int n = (s.length - 1) / rows + 1;
                s.first = first;
                at = std::fill_n(at, n, s);
                first += n;
                if (rows == 128) {
                    out->longest = std::max(out->longest, n);
                    out->work += n * (n + 1LL) / 2;
                }
            }
        }
    } catch (const std::bad_alloc&) {
        return MOARA_ERR_WORKSPACE;
    }
    return MOARA_OK;
}

int moara_attention(moara_ctx* ctx, const moara_sequences* seqs, int tokens, int heads, int kv_heads, int dim, float scale,
                    const void* q, int64_t q_row, int64_t q_head, const void* k, int64_t k_row, int64_t k_head,
                    const void* v, int64_t v_row, int64_t v_head, void* out, void* rest, float* lse, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    int rc = check_attention(ctx, seqs, tokens, heads, kv_heads, dim, scale);
    if (rc != MOARA_OK || seqs->n_tiles == 0) return rc;
    rc = check_heads(ctx, "q", q, q_row, q_head, tokens, heads, dim);
    if (rc == MOARA_OK) rc = check_heads(ctx, "k", k, k_row, k_head, tokens, kv_heads, dim);
    if (rc == MOARA_OK) rc = check_heads(ctx, "v", v, v_row, v_head, tokens, kv_heads, dim);
    if (rc == MOARA_OK) rc = check_out(ctx, "out", out);
    if (rc == MOARA_OK && rest != nullptr) rc = check_out(ctx, "rest", rest);
    if (rc == MOARA_OK) rc = check_floats(ctx, "lse", lse);
    if (rc != MOARA_OK) return rc;
    DeviceGuard g(ctx->device);
    const moara::Attention a{q, k, v, out, rest, lse, q_row, q_head, k_row, k_head, v_row, v_head, tokens, heads, kv_heads, dim,
                             scale, static_cast<const AttentionTile*>(seqs->tiles), seqs->n_pairs, seqs->work, ctx->d_status,
                             moara::tc_wait_limit(ctx->tc)};
    const cudaError_t e = moara::launch_attention(a, static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "attention launch");
    return MOARA_OK;
}

int moara_attention_backward(moara_ctx* ctx, const moara_sequences* seqs, int tokens, int heads, int kv_heads, int dim,
                             float scale, const void* dout, int64_t do_row, int64_t do_head, const void* q, int64_t q_row,
                             int64_t q_head, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row,
                             int64_t v_head, const void* out, const void* rest, const float* lse, float* delta, void* dq,
                             void* dk, void* dv, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    int rc = check_attention(ctx, seqs, tokens, heads, kv_heads, dim, scale);
    if (rc != MOARA_OK || seqs->n_tiles == 0) return rc;
    rc = check_heads(ctx, "dout", dout, do_row, do_head, tokens, heads, dim);
    if (rc == MOARA_OK) rc = check_heads(ctx, "q", q, q_row, q_head, tokens, heads, dim);
    if (rc == MOARA_OK) rc = check_heads(ctx, "k", k, k_row, k_head, tokens, kv_heads, dim);
    if (rc == MOARA_OK) rc = check_heads(ctx, "v", v, v_row, v_head, tokens, kv_heads, dim);
    if (rc == MOARA_OK) rc = check_out(ctx, "out", out);
    if (rc == MOARA_OK && rest != nullptr) rc = check_out(ctx, "rest", rest);
    if (rc == MOARA_OK) rc = check_floats(ctx, "lse", lse);
    if (rc == MOARA_OK) rc = check_floats(ctx, "delta", delta);
    if (rc == MOARA_OK) rc = check_out(ctx, "dq", dq);
    if (rc == MOARA_OK) rc = check_out(ctx, "dk", dk);
    if (rc == MOARA_OK) rc = check_out(ctx, "dv", dv);
    if (rc != MOARA_OK) return rc;
    DeviceGuard g(ctx->device);
    const AttentionTile* tiles = static_cast<const AttentionTile*>(seqs->tiles) + seqs->n_pairs;
    const moara::AttentionGrad a{dout, q, k, v, out, rest, lse, delta, dq, dk, dv, do_row, do_head, q_row, q_head, k_row, k_head,
                                 v_row, v_head, tokens, heads, kv_heads, dim, scale, tiles, seqs->n_tiles,
                                 seqs->longest, seqs->work, ctx->d_status, moara::tc_wait_limit(ctx->tc)};
    const cudaError_t e = moara::launch_attention_backward(a, static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "attention gradient launch");
    return MOARA_OK;
}

int moara_policy_loss_workspace_bytes(int rows, size_t* out) {
    if (out == nullptr) return MOARA_ERR_INVALID_ARG;
    if (rows < 1) return MOARA_ERR_SHAPE;
    *out = moara::policy_loss_workspace(rows);
    return MOARA_OK;
}

int moara_policy_loss(moara_ctx* ctx, int rows, int vocab, const void* Z, int dtype, int64_t ldz, const int64_t* target,
                      const float* old_logp, const float* ref_logp, const float* adv, const float* weight, float low,
                      float high, float kl, float* sums, float* logp, void* dZ, int64_t lddz, void* workspace,
                      size_t workspace_bytes, void* stream) {
    if (ctx == nullptr) return MOARA_ERR_INVALID_ARG;
    if (rows < 1 || vocab < 1) return fail(ctx, MOARA_ERR_SHAPE, "rows and vocab must be >= 1");
    if (rows > INT_MAX / 8 || vocab > INT_MAX - 1024) return fail(ctx, MOARA_ERR_SHAPE, "too many rows or columns");
    int rc = check_rows(ctx, "Z", Z, dtype, vocab, ldz);
    if (rc == MOARA_OK && dZ != nullptr) rc = check_rows(ctx, "dZ", dZ, dtype, vocab, lddz);
    if (rc == MOARA_OK && dZ == Z && lddz != ldz) rc = fail(ctx, MOARA_ERR_SHAPE, "dZ is Z with another pitch");
    if (rc == MOARA_OK) rc = check_apart(ctx, Span("dZ", dZ, dtype, rows, vocab, lddz), Span("Z", Z, dtype, rows, vocab, ldz));
    if (rc == MOARA_OK && target == nullptr) rc = fail(ctx, MOARA_ERR_INVALID_ARG, "target is NULL");
    if (rc == MOARA_OK && !aligned(target, 8)) rc = fail(ctx, MOARA_ERR_ALIGN, "target is not aligned to its type");
    if (rc == MOARA_OK) rc = check_floats(ctx, "old_logp", old_logp);
    if (rc == MOARA_OK && ref_logp != nullptr) rc = check_floats(ctx, "ref_logp", ref_logp);
    if (rc == MOARA_OK) rc = check_floats(ctx, "adv", adv);
    if (rc == MOARA_OK && weight != nullptr) rc = check_floats(ctx, "weight", weight);
    if (rc == MOARA_OK) rc = check_floats(ctx, "sums", sums);
    if (rc == MOARA_OK) rc = check_floats(ctx, "logp", logp);
    if (rc != MOARA_OK) return rc;
    if (!(low >= 0.0f && low <= 1.0f) || !(high >= 1.0f))
        return fail(ctx, MOARA_ERR_INVALID_ARG, "the ratio's bounds must lie in 0 .. 1 and from 1 on");
    if (!(kl >= 0.0f && kl < INFINITY)) return fail(ctx, MOARA_ERR_INVALID_ARG, "kl must be >= 0");
    if (kl > 0.0f && ref_logp == nullptr) return fail(ctx, MOARA_ERR_INVALID_ARG, "a KL term needs ref_logp");
    size_t need = 0;
    moara_policy_loss_workspace_bytes(rows, &need);
    if (workspace == nullptr || workspace_bytes < need)
        return fail(ctx, MOARA_ERR_WORKSPACE, "the loss needs %zu bytes of workspace", need);
    if (!aligned16(workspace)) return fail(ctx, MOARA_ERR_ALIGN, "workspace is not 16-byte aligned");
    DeviceGuard g(ctx->device);
    const moara::PolicyLoss a{rows, vocab, Z, dtype, ldz, target, old_logp, ref_logp, adv, weight, low, high, kl, sums, logp,
                              dZ, lddz, workspace, ctx->d_status, moara::tc_wait_limit(ctx->tc)};
    const cudaError_t e = moara::launch_policy_loss(a, static_cast<cudaStream_t>(stream), &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "policy loss launch");
    return MOARA_OK;
}

}  // extern "C"
