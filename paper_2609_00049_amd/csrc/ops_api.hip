// C ABI of the operators a quantized model is run, scored and differentiated with: token log
// probabilities, packed attention and the 8-bit integer product.  Argument checks and launches only; the
// workspaces are the caller's (a captured graph keeps its own).
#include <cmath>
#include <string>

#include "common.h"
#include "ctx.h"
#include "kernels.h"
#include "../../include/realq.h"

using realq::set_error;
using realq::Timed;

namespace {

// The context's device, for the scope of a call: the caller may have another one current.
struct OnDevice {
    int before = -1;
    bool moved = false;
    hipError_t enter(int device) {
        hipError_t e = hipGetDevice(&before);
        if (e == hipSuccess && before != device) {
            e = hipSetDevice(device);
            moved = e == hipSuccess;
        }
        return e;
    }
    ~OnDevice() {
        if (moved) (void)hipSetDevice(before);
    }
};

constexpr int64_t kMostRows = (int64_t)1 << 40, kMostColumns = INT32_MAX;

bool aligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// Runs an entry point's body; nothing is thrown across the C boundary.
template <class F>
int guarded(realq_ctx* ctx, F&& body) {
    if (!ctx) return REALQ_ERR_INVALID_ARG;
    try {
        return body();
    } catch (...) {
        return REALQ_ERR_OOM;
    }
}

// What a workspace goes by.
int check_logprobs_sizes(realq_ctx* ctx, const realq_logprobs_desc* d, const std::string& w) {
    if (d->dtype != REALQ_BF16 && d->dtype != REALQ_F32)
        return set_error(ctx, REALQ_ERR_INVALID_ARG, w + "dtype must be REALQ_BF16 or REALQ_F32");
    if (d->T < 0 || d->T > kMostRows || d->V < 1 || d->V > kMostColumns)
        return set_error(ctx, REALQ_ERR_SHAPE, w + "need 0 <= T, 1 <= V < 2^31");
    if (d->top < 0 || d->top > REALQ_LOGPROBS_MAX_TOP || d->top > d->V)
        return set_error(ctx, REALQ_ERR_SHAPE, w + "top must be 0 .. min(V, 64)");
    return REALQ_OK;
}

int check_logprobs(realq_ctx* ctx, const realq_logprobs_desc* d, const char* who) {
    const std::string w = std::string(who) + ": ";
    if (!d) return set_error(ctx, REALQ_ERR_INVALID_ARG, w + "NULL descriptor");
    if (const int rc = check_logprobs_sizes(ctx, d, w)) return rc;
    if (d->ld < d->V || d->ld > kMostRows) return set_error(ctx, REALQ_ERR_SHAPE, w + "need ld >= V");
    if (d->T == 0) return REALQ_OK;
    if (!d->logits) return set_error(ctx, REALQ_ERR_INVALID_ARG, w + "NULL logits");
    if (!aligned(d->logits, d->dtype == REALQ_F32 ? 4 : 2) || !aligned(d->targets, 8))
        return set_error(ctx, REALQ_ERR_INVALID_ARG, w + "logits or targets not aligned to their elements");
    return REALQ_OK;
}

realq::LogprobsArgs logprobs_args(const realq_logprobs_desc* d) {
    return {d->logits, d->dtype == REALQ_F32, d->T, d->V, d->ld, d->targets, d->top};
}

int check_attention(realq_ctx* ctx, const realq_attention_desc* d, const char* who) {
    const std::string w = std::string(who) + ": ";
    if (!d) return set_error(ctx, REALQ_ERR_INVALID_ARG, w + "NULL descriptor");
    if (d->T < 0 || d->T > INT32_MAX || d->n_seqs < 0 || d->n_seqs > ((int64_t)1 << 22) || d->T / 32 > ((int64_t)1 << 23))
        return set_error(ctx, REALQ_ERR_SHAPE, w + "need 0 <= T <= 2^28, 0 <= n_seqs <= 2^22");
    if (d->n_heads < 1 || d->n_heads > 65535 || d->n_kv < 1 || d->n_heads % d->n_kv)
        return set_error(ctx, REALQ_ERR_SHAPE, w + "need 1 <= n_heads <= 65535, n_kv >= 1 dividing n_heads");
    if ((d->T / 128 + d->n_seqs) * d->n_heads >= (int64_t)1 << 23)  // blocks of 512 threads, fewer than 2^32
        return set_error(ctx, REALQ_ERR_SHAPE, w + "need (T / 128 + n_seqs) n_heads < 2^23");
    if (d->head_dim < 8 || d->head_dim > 256 || d->head_dim % 8)
        return set_error(ctx, REALQ_ERR_SHAPE, w + "head_dim must be a multiple of 8, 8 .. 256");
    if (!(d->scale >= 0.f) || std::isinf(d->scale))
        return set_error(ctx, REALQ_ERR_INVALID_ARG, w + "scale must be finite and >= 0 (0: 1 / sqrt(head_dim))");
    return REALQ_OK;
}

// A token-major array of heads: rows of `heads` heads on 16 bytes, ld elements apart.
int check_heads(realq_ctx* ctx, const char* who, const char* name, const void* p, int64_t ld, int64_t heads, int hd) {
    const std::string w = std::string(who) + ": " + name;
    if (!p) return set_error(ctx, REALQ_ERR_INVALID_ARG, w + " is NULL");
    if (ld < heads * hd || ld % 8 || ld > ((int64_t)1 << 24))
        return set_error(ctx, REALQ_ERR_SHAPE, w + ": row stride must be a multiple of 8, hold all heads and be at most 2^24");
    if (!aligned(p, 16)) return set_error(ctx, REALQ_ERR_INVALID_ARG, w + " must be aligned to 16 bytes");
    return REALQ_OK;
}

int check_inputs(realq_ctx* ctx, const realq_attention_desc* d, const char* who) {
    if (!d->cu_seqlens || !aligned(d->cu_seqlens, 4))
        return set_error(ctx, REALQ_ERR_INVALID_ARG, std::string(who) + ": cu_seqlens is NULL or not aligned");
    if (const int rc = check_heads(ctx, who, "q", d->q, d->ldq, d->n_heads, d->head_dim)) return rc;
    if (const int rc = check_heads(ctx, who, "k", d->k, d->ldk, d->n_kv, d->head_dim)) return rc;
    return check_heads(ctx, who, "v", d->v, d->ldv, d->n_kv, d->head_dim);
}

realq::AttnArgs attn_args(const realq_attention_desc* d) {
    const float scale = d->scale == 0.f ? (float)(1.0 / std::sqrt((double)d->head_dim)) : d->scale;
    return {d->q, d->k, d->v, d->ldq, d->ldk, d->ldv, d->T, d->n_seqs, d->cu_seqlens, d->n_heads, d->n_kv, d->head_dim,
            scale};
}

}  // namespace

extern "C" {

// ============================================================================ token log probabilities

int realq_token_logprobs_workspace(realq_ctx* ctx, const realq_logprobs_desc* d, size_t* bytes) {
    return guarded(ctx, [&]() -> int {
        if (!bytes) return set_error(ctx, REALQ_ERR_INVALID_ARG, "token_logprobs_workspace: NULL bytes");
        if (!d || d->T < 0 || d->V < 1 || d->top < 0)
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "token_logprobs_workspace: bad descriptor");
        if (const int rc = check_logprobs_sizes(ctx, d, "token_logprobs_workspace: ")) return rc;
        *bytes = realq::logprobs_workspace(d->T, d->V, d->top, d->dtype == REALQ_F32, ctx->cus);
        return REALQ_OK;
    });
}

int realq_token_logprobs(realq_ctx* ctx, const realq_logprobs_desc* d, float* logp, float* lse, float* entropy,
                         int64_t* top_ids, float* top_logp, void* work, size_t work_bytes) {
    return guarded(ctx, [&]() -> int {
        if (const int rc = check_logprobs(ctx, d, "token_logprobs")) return rc;
        if (d->T == 0) return REALQ_OK;
        if (!lse || (logp && !d->targets) || (d->top > 0 && (!top_ids || !top_logp)))
            return set_error(ctx, REALQ_ERR_INVALID_ARG,
                             "token_logprobs: lse is required, logp needs targets, top > 0 needs top_ids and top_logp");
        if (!aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(top_ids, 8) ||
            !aligned(top_logp, 4) || !aligned(work, 16))
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "token_logprobs: an output or the workspace is not aligned");
        const size_t need = realq::logprobs_workspace(d->T, d->V, d->top, d->dtype == REALQ_F32, ctx->cus);
        if (need > 0 && (!work || work_bytes < need))
            return set_error(ctx, REALQ_ERR_INVALID_ARG,
                             "token_logprobs: the workspace needs " + std::to_string(need) + " bytes");
        OnDevice on;
        RQ_HIP(ctx, on.enter(ctx->device));
        Timed tm(ctx, "logprobs");
        RQ_HIP(ctx, realq::logprobs_forward(logprobs_args(d), logp, lse, entropy, top_ids, top_logp, work, ctx->cus,
                                            ctx->stream));
        return REALQ_OK;
    });
}

int realq_token_logprobs_backward(realq_ctx* ctx, const realq_logprobs_desc* d, const float* lse, const float* entropy,
                                  const int64_t* top_ids, const float* dlogp, const float* dentropy, const float* dtop,
                                  void* dlogits, int64_t ldd) {
    return guarded(ctx, [&]() -> int {
        if (const int rc = check_logprobs(ctx, d, "token_logprobs_backward")) return rc;
        if (d->T == 0) return REALQ_OK;
        if (!lse || !dlogits || (dlogp && !d->targets) || (dentropy && !entropy) || (dtop && (d->top < 1 || !top_ids)))
            return set_error(ctx, REALQ_ERR_INVALID_ARG,
                             "token_logprobs_backward: lse and dlogits are required, dlogp needs targets, dentropy "
                             "entropy, dtop top >= 1 and top_ids");
        if (ldd < d->V || ldd > kMostRows) return set_error(ctx, REALQ_ERR_SHAPE, "token_logprobs_backward: ldd < V");
        if (dlogits == d->logits && ldd != d->ld)
            return set_error(ctx, REALQ_ERR_SHAPE, "token_logprobs_backward: in place needs ldd = ld");
        if (!aligned(lse, 4) || !aligned(entropy, 4) || !aligned(top_ids, 8) || !aligned(dlogp, 4) ||
            !aligned(dentropy, 4) || !aligned(dtop, 4) || !aligned(dlogits, d->dtype == REALQ_F32 ? 4 : 2))
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "token_logprobs_backward: an array is not aligned");
        OnDevice on;
        RQ_HIP(ctx, on.enter(ctx->device));
        Timed tm(ctx, "logprobs");
        RQ_HIP(ctx, realq::logprobs_backward(logprobs_args(d), lse, entropy, top_ids, dlogp, dentropy, dtop, dlogits,
                                             ldd, ctx->stream));
        return REALQ_OK;
    });
}

// ============================================================================ packed attention

int realq_packed_attention(realq_ctx* ctx, const realq_attention_desc* d, uint16_t* O, int64_t ldo, float* lse) {
    return guarded(ctx, [&]() -> int {
        const char* who = "packed_attention";
        if (const int rc = check_attention(ctx, d, who)) return rc;
        if (d->T == 0 || d->n_seqs == 0) return REALQ_OK;
        if (const int rc = check_inputs(ctx, d, who)) return rc;
        if (const int rc = check_heads(ctx, who, "O", O, ldo, d->n_heads, d->head_dim)) return rc;
        if (!aligned(lse, 4)) return set_error(ctx, REALQ_ERR_INVALID_ARG, "packed_attention: lse is not aligned");
        OnDevice on;
        RQ_HIP(ctx, on.enter(ctx->device));
        Timed tm(ctx, "packed_attention");
        RQ_HIP(ctx, realq::attn_packed_forward(attn_args(d), O, ldo, lse, ctx->stream));
        return REALQ_OK;
    });
}

int realq_packed_attention_workspace(realq_ctx* ctx, const realq_attention_desc* d, size_t* bytes) {
    return guarded(ctx, [&]() -> int {
        if (const int rc = check_attention(ctx, d, "packed_attention_workspace")) return rc;
        if (!bytes) return set_error(ctx, REALQ_ERR_INVALID_ARG, "packed_attention_workspace: NULL bytes");
        *bytes = d->T == 0 || d->n_seqs == 0 ? 0 : realq::attn_packed_workspace(attn_args(d));
        return REALQ_OK;
    });
}

int realq_packed_attention_backward(realq_ctx* ctx, const realq_attention_desc* d, const uint16_t* O, int64_t ldo,
                                    const float* lse, const uint16_t* dO, int64_t lddo, void* work,
                                    size_t work_bytes, uint16_t* dQ, int64_t lddq, uint16_t* dK, int64_t lddk,
                                    uint16_t* dV, int64_t lddv) {
    return guarded(ctx, [&]() -> int {
        const char* who = "packed_attention_backward";
        if (const int rc = check_attention(ctx, d, who)) return rc;
        if (d->T == 0 || d->n_seqs == 0) return REALQ_OK;
        if (const int rc = check_inputs(ctx, d, who)) return rc;
        const int H = d->n_heads, G = d->n_kv, hd = d->head_dim;
        if (const int rc = check_heads(ctx, who, "O", O, ldo, H, hd)) return rc;
        if (const int rc = check_heads(ctx, who, "dO", dO, lddo, H, hd)) return rc;
        if (const int rc = check_heads(ctx, who, "dQ", dQ, lddq, H, hd)) return rc;
        if (const int rc = check_heads(ctx, who, "dK", dK, lddk, G, hd)) return rc;
        if (const int rc = check_heads(ctx, who, "dV", dV, lddv, G, hd)) return rc;
        if (!lse || !aligned(lse, 4))
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "packed_attention_backward: lse is NULL or not aligned");
        const size_t need = realq::attn_packed_workspace(attn_args(d));
        if (!work || !aligned(work, 16) || work_bytes < need)
            return set_error(ctx, REALQ_ERR_INVALID_ARG,
                             "packed_attention_backward: the workspace needs " + std::to_string(need) + " bytes on 16");
        OnDevice on;
        RQ_HIP(ctx, on.enter(ctx->device));
        Timed tm(ctx, "packed_attention");
        RQ_HIP(ctx, realq::attn_packed_backward(attn_args(d), O, ldo, lse, dO, lddo, work, dQ, lddq, dK, lddk, dV,
                                                lddv, ctx->stream));
        return REALQ_OK;
    });
}

// ============================================================================ 8-bit integer product

int realq_quantize_rows_i8(realq_ctx* ctx, const void* X, int32_t dtype, int64_t T, int64_t n, int64_t ldx, int8_t* Q,
                           int64_t ldq, float* scale) {
    return guarded(ctx, [&]() -> int {
        if (dtype != REALQ_BF16 && dtype != REALQ_F32)
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "quantize_rows_i8: dtype must be REALQ_BF16 or REALQ_F32");
        if (T < 0 || T > kMostRows || n < 1 || n > kMostColumns || ldx < n || ldq < n || ldx > kMostRows || ldq > kMostRows)
            return set_error(ctx, REALQ_ERR_SHAPE, "quantize_rows_i8: need T >= 0, 1 <= n < 2^31, ldx >= n, ldq >= n");
        if (T == 0) return REALQ_OK;
        if (!X || !Q || !scale || !aligned(X, dtype == REALQ_F32 ? 4 : 2) || !aligned(scale, 4))
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "quantize_rows_i8: X, Q or scale is NULL or not aligned");
        OnDevice on;
        RQ_HIP(ctx, on.enter(ctx->device));
        Timed tm(ctx, "linear_i8");
        RQ_HIP(ctx, realq::quantize_rows_i8(X, dtype == REALQ_F32, T, n, ldx, Q, ldq, scale, ctx->stream));
        return REALQ_OK;
    });
}

int realq_linear_i8(realq_ctx* ctx, const int8_t* X, int64_t ldx, const float* sx, const int8_t* W, int64_t ldw,
                    const float* sw, const float* bias, int64_t T, int64_t n, int64_t m, void* Y, int32_t dtype,
                    int64_t ldy) {
    return guarded(ctx, [&]() -> int {
        if (dtype != REALQ_BF16 && dtype != REALQ_F32)
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "linear_i8: dtype must be REALQ_BF16 or REALQ_F32");
        if (T < 0 || T > ((int64_t)1 << 30) || m < 1 || m > ((int64_t)1 << 30) || n < 1 || n > REALQ_I8_MAX_COLUMNS)
            return set_error(ctx, REALQ_ERR_SHAPE, "linear_i8: need 0 <= T <= 2^30, 1 <= m <= 2^30, 1 <= n <= 131071");
        if (ldx < n || ldw < n || ldy < m || ldx > kMostRows || ldw > kMostRows || ldy > kMostRows)
            return set_error(ctx, REALQ_ERR_SHAPE, "linear_i8: need ldx >= n, ldw >= n, ldy >= m");
        if (T == 0) return REALQ_OK;
        if (!X || !sx || !W || !sw || !Y || !aligned(sx, 4) || !aligned(sw, 4) || !aligned(bias, 4) ||
            !aligned(Y, dtype == REALQ_F32 ? 4 : 2))
            return set_error(ctx, REALQ_ERR_INVALID_ARG, "linear_i8: X, sx, W, sw or Y is NULL or an array not aligned");
        if (((T + 127) / 128) * ((m + 127) / 128) > ((int64_t)1 << 22))
            return set_error(ctx, REALQ_ERR_SHAPE, "linear_i8: more than 2^22 tiles of 128 x 128 outputs");
        OnDevice on;
        RQ_HIP(ctx, on.enter(ctx->device));
        Timed tm(ctx, "linear_i8");
        RQ_HIP(ctx, realq::linear_i8({X, W, T, n, m, ldx, ldw, ldy, sx, sw, bias, Y, dtype == REALQ_F32}, ctx->stream));
        return REALQ_OK;
    });
}

}  // extern "C"
