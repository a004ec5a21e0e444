// C ABI of the operators at the two ends of a language model (declared in include/ef21.h): argument checks and launches.
#include <cmath>

#include "../../include/ef21.h"
#include "lm.h"

namespace {

using ef21::report_error;

static_assert((int)ef21::kF32 == (int)EF21_F32 && (int)ef21::kBF16 == (int)EF21_BF16 && (int)ef21::kF16 == (int)EF21_F16,
              "value types of lm.h and ef21.h must agree");

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1;

int invalid(const char *text) { return report_error(EF21_EINVAL, text); }

bool aligned(const void *p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }

bool value_type(int type) { return type == EF21_F32 || type == EF21_BF16 || type == EF21_F16; }

// A two-dimensional array: its pointer may be NULL where it has no rows.
int check_rows(const void *p, int type, int64_t rows, int64_t width, int64_t stride, const char *null, const char *strided) {
    if (stride < width || (rows > 0 && stride > (INT64_MAX >> 3) / rows)) return invalid(strided);
    if (rows > 0 && (!p || !aligned(p, ef21::value_bytes(type)))) return invalid(null);
    return EF21_OK;
}

int check_tokens(const void *tokens, int token_type, int64_t count) {
    if (token_type != EF21_I32 && token_type != EF21_I64) return invalid("unknown type of the tokens or labels");
    if (count > 0 && (!tokens || !aligned(tokens, token_type == EF21_I64 ? 8 : 4))) return invalid("tokens or labels are NULL or misaligned");
    return EF21_OK;
}

int check_vectors(int64_t rows, std::initializer_list<const void *> arrays) {
    for (const void *p : arrays)
        if (rows > 0 && (!p || !aligned(p, 4))) return invalid("an array with one entry per row is NULL or misaligned");
    return EF21_OK;
}

int check_logits(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels, int label_type,
                 ef21::LogitRows *out) {
    if (!value_type(type)) return invalid("unknown type of the logits");
    if (rows < 0 || rows > kMostRows) return invalid("rows must be in [0, 2^31)");
    if (vocab < 1 || vocab > kMostRows) return invalid("vocab must be in [1, 2^31)");
    if (int rc = check_rows(logits, type, rows, vocab, stride, "logits are NULL or misaligned", "the logits' stride is too small or too large")) return rc;
    if (int rc = check_tokens(labels, label_type, rows)) return rc;
    *out = ef21::LogitRows{logits, type, rows, vocab, stride, {labels, label_type}};
    return EF21_OK;
}

int check_grad(const ef21::LogitRows &in, const void *grad, int64_t grad_stride) {
    if (int rc = check_rows(grad, in.type, in.rows, in.vocab, grad_stride, "grad_logits is NULL or misaligned",
                            "the gradient's stride is too small or too large"))
        return rc;
    if (grad == in.x && grad_stride != in.stride && in.rows > 1) return invalid("a gradient written over the logits must have their stride");
    return EF21_OK;
}

int check_workspace(const void *workspace, int64_t have, size_t need) {
    if (need == 0) return EF21_OK;
    if (!workspace || !aligned(workspace, 256)) return invalid("workspace is NULL or not 256-byte aligned");
    if (have < 0 || (size_t)have < need) return invalid("workspace is too small");
    return EF21_OK;
}

int launched(hipError_t st, const char *what) { return st == hipSuccess ? EF21_OK : ef21::report_hip_error(st, what); }

int check_embed_grad_sizes(int32_t n, int64_t count, int64_t vocab, int64_t width) {
    if (n < 1 || n > 65535) return invalid("n must be in [1, 65535]");
    if (count < 0 || count > kMostRows || count > ((int64_t)1 << 40) / n) return invalid("count must be in [0, 2^31), and n count at most 2^40");
    if (vocab < 1 || vocab > kMostRows - 1) return invalid("vocab must be in [1, 2^31 - 1)");
    if (width < 1 || width > kMostRows) return invalid("width must be in [1, 2^31)");
    if (width > ((int64_t)1 << 60) / n / vocab) return invalid("the gradient is too large");
    return EF21_OK;
}

}  // namespace

extern "C" {

int ef21_embed(const void *table, int table_type, int64_t vocab, int64_t width, int64_t table_stride, const void *tokens,
               int token_type, int64_t count, float scale, void *out, int out_type, int64_t out_stride, void *hip_stream) {
    if (!value_type(table_type) || !value_type(out_type)) return invalid("unknown type of the table or of out");
    if (count < 0 || count > kMostRows) return invalid("count must be in [0, 2^31)");
    if (vocab < 1 || vocab > kMostRows) return invalid("vocab must be in [1, 2^31)");
    if (width < 1 || width > kMostRows) return invalid("width must be in [1, 2^31)");
    if (!std::isfinite(scale)) return invalid("scale must be finite");
    if (int rc = check_tokens(tokens, token_type, count)) return rc;
    if (int rc = check_rows(table, table_type, vocab, width, table_stride, "table is NULL or misaligned", "the table's stride is too small or too large"))
        return rc;
    if (int rc = check_rows(out, out_type, count, width, out_stride, "out is NULL or misaligned", "the stride of out is too small or too large")) return rc;
    const ef21::EmbedArgs p{table, table_type, vocab, width, table_stride, {tokens, token_type}, count, scale, out, out_type, out_stride};
    return launched(ef21::launch_embed(p, (hipStream_t)hip_stream), "embedding kernel launch");
}

int ef21_embed_grad_workspace(int32_t n, int64_t count, int64_t vocab, int64_t width, int64_t *bytes) {
    if (int rc = check_embed_grad_sizes(n, count, vocab, width)) return rc;
    if (!bytes) return invalid("bytes is NULL");
    *bytes = (int64_t)ef21::embed_grad_workspace_bytes(n, count, vocab, width);
    return EF21_OK;
}

int ef21_embed_grad(const void *grad_out, int type, int64_t grad_stride, const void *tokens, int token_type, int32_t n,
                    int64_t count, int64_t vocab, int64_t width, float scale, float *table_grad, int64_t worker_stride,
                    int accumulate, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (!value_type(type)) return invalid("unknown type of grad_out");
    if (int rc = check_embed_grad_sizes(n, count, vocab, width)) return rc;
    if (!std::isfinite(scale)) return invalid("scale must be finite");
    if (int rc = check_tokens(tokens, token_type, n * count)) return rc;
    if (int rc = check_rows(grad_out, type, n * count, width, grad_stride, "grad_out is NULL or misaligned", "the stride of grad_out is too small or too large"))
        return rc;
    if (int rc = check_vectors(1, {table_grad})) return rc;
    if (n > 1 && (worker_stride < vocab * width || worker_stride > (INT64_MAX >> 3) / n)) return invalid("worker_stride is too small or too large");
    if (int rc = check_workspace(workspace, workspace_bytes, ef21::embed_grad_workspace_bytes(n, count, vocab, width))) return rc;
    const ef21::EmbedGradArgs p{grad_out, type, grad_stride, {tokens, token_type}, n, count, vocab, width, scale, table_grad, worker_stride, accumulate};
    return launched(ef21::launch_embed_grad(p, workspace, (hipStream_t)hip_stream), "embedding gradient launch");
}

int ef21_token_logps(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                     int label_type, float *logp, float *lse, void *hip_stream) {
    ef21::LogitRows in;
    if (int rc = check_logits(logits, type, rows, vocab, stride, labels, label_type, &in)) return rc;
    if (int rc = check_vectors(rows, {logp, lse})) return rc;
    return launched(ef21::launch_token_logps(in, logp, lse, (hipStream_t)hip_stream), "log-probability kernel launch");
}

int ef21_token_logps_grad(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                          int label_type, const float *lse, const float *grad_logp, void *grad_logits, int64_t grad_stride,
                          void *hip_stream) {
    ef21::LogitRows in;
    if (int rc = check_logits(logits, type, rows, vocab, stride, labels, label_type, &in)) return rc;
    if (int rc = check_vectors(rows, {lse, grad_logp})) return rc;
    if (int rc = check_grad(in, grad_logits, grad_stride)) return rc;
    return launched(ef21::launch_token_grad(in, lse, grad_logp, {grad_logits, grad_stride}, (hipStream_t)hip_stream), "logit gradient launch");
}

int ef21_preference_loss_workspace(int64_t rows, int32_t pairs, int64_t *bytes) {
    if (rows < 0 || rows > kMostRows) return invalid("rows must be in [0, 2^31)");
    if (pairs < 1) return invalid("pairs must be at least 1");
    if (!bytes) return invalid("bytes is NULL");
    *bytes = (int64_t)ef21::preference_workspace_bytes(rows);
    return EF21_OK;
}

int ef21_preference_loss(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                         int label_type, const int64_t *seq_start, int32_t pairs, const float *ref_logp, float beta,
                         float smoothing, int loss, int mean, const float *pair_weight, float *out_loss, float *logp,
                         void *grad_logits, int64_t grad_stride, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    ef21::LogitRows in;
    if (int rc = check_logits(logits, type, rows, vocab, stride, labels, label_type, &in)) return rc;
    if (int rc = check_vectors(rows, {ref_logp, logp})) return rc;
    if (grad_logits)
        if (int rc = check_grad(in, grad_logits, grad_stride)) return rc;
    if (pairs < 1) return invalid("pairs must be at least 1");
    if (!seq_start || !aligned(seq_start, 8)) return invalid("seq_start is NULL or misaligned");
    if (!out_loss || !aligned(out_loss, 4) || !aligned(pair_weight, 4)) return invalid("out_loss is NULL, or it or pair_weight misaligned");
    if (!(beta > 0.f) || !std::isfinite(beta)) return invalid("beta must be finite and > 0");
    if (!(smoothing >= 0.f && smoothing < 1.f)) return invalid("smoothing must be in [0, 1)");
    if (loss != EF21_LOSS_LOGISTIC && loss != EF21_LOSS_LEAST_SQUARES) return invalid("unknown loss");
    if (int rc = check_workspace(workspace, workspace_bytes, ef21::preference_workspace_bytes(rows))) return rc;
    const ef21::PairArgs p{seq_start, pairs, rows, logp, ref_logp, in.labels, vocab, beta, smoothing, loss, mean, pair_weight, out_loss, nullptr};
    return launched(ef21::launch_preference(in, p, {grad_logits, grad_stride}, workspace, (hipStream_t)hip_stream), "preference loss launch");
}

int ef21_policy_loss_workspace(int64_t rows, int64_t *bytes) {
    if (rows < 0 || rows > kMostRows) return invalid("rows must be in [0, 2^31)");
    if (!bytes) return invalid("bytes is NULL");
    *bytes = (int64_t)ef21::policy_workspace_bytes(rows);
    return EF21_OK;
}

int ef21_policy_loss(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                     int label_type, const float *old_logp, const float *advantages, const float *ref_logp,
                     const float *weight, float clip_low, float clip_high, float kl, float *out_loss, float *token_loss,
                     float *logp, void *grad_logits, int64_t grad_stride, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    ef21::LogitRows in;
    if (int rc = check_logits(logits, type, rows, vocab, stride, labels, label_type, &in)) return rc;
    if (int rc = check_vectors(rows, {old_logp, advantages, token_loss, logp})) return rc;
    if (grad_logits)
        if (int rc = check_grad(in, grad_logits, grad_stride)) return rc;
    if (!out_loss || !aligned(out_loss, 4) || !aligned(ref_logp, 4) || !aligned(weight, 4))
        return invalid("out_loss is NULL, or it, ref_logp or weight misaligned");
    if (!(clip_low >= 0.f && clip_low <= 1.f)) return invalid("clip_low must be in [0, 1]");
    if (!(clip_high >= 0.f) || !std::isfinite(clip_high)) return invalid("clip_high must be finite and >= 0");
    if (!(kl >= 0.f) || !std::isfinite(kl)) return invalid("kl must be finite and >= 0");
    if (kl > 0.f && rows > 0 && !ref_logp) return invalid("a KL term needs ref_logp");
    if (int rc = check_workspace(workspace, workspace_bytes, ef21::policy_workspace_bytes(rows))) return rc;
    const ef21::PolicyArgs p{old_logp, kl > 0.f ? ref_logp : nullptr, advantages, weight, clip_low, clip_high, kl, out_loss, token_loss, logp};
    return launched(ef21::launch_policy(in, p, {grad_logits, grad_stride}, workspace, (hipStream_t)hip_stream), "policy loss launch");
}

}  // extern "C"
