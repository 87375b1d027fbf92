// extern "C" entry points of the vocabulary operators (embedding.hip, distill.hip, logits.hip): argument checks.
#include "spmm_internal.h"

#include <cmath>

namespace scorch {

// embedding.hip
scorch_status_t launch_lookup(int32_t tokens, int32_t vocab, int32_t d, const int32_t *ids, const void *E, int32_t e_type, int64_t lde,
                              float scale, void *out, int32_t out_type, int64_t ldo, hipStream_t stream);
uint64_t gradient_workspace_bytes(int32_t tokens, int32_t d);
scorch_status_t launch_gradient(int32_t tokens, int32_t vocab, int32_t d, const int32_t *ids, const void *dout, int32_t dout_type,
                                int64_t lddo, float scale, int32_t accumulate, void *dE, int32_t de_type, int64_t ldde,
                                char *workspace, hipStream_t stream);
// distill.hip
scorch_status_t launch_distill(int what, int32_t rows, int32_t vocab, const void *Z, int32_t z_type, int64_t ldz, const int32_t *rowptr,
                               const int32_t *colidx, const float *vals, float x, const float *dloss, float *loss, float *stats,
                               void *dZ, int64_t lddz, hipStream_t stream);
// logits.hip
scorch_status_t launch_logits(int32_t rows, int32_t vocab, const void *in, int32_t type, int64_t ldi, const scorch_logits_rules_t &rules,
                              void *out, int32_t out_type, int64_t ldo, hipStream_t stream);

constexpr int32_t kEmbeddingColumnsMax = 1 << 22;  // tiles of columns are the slow dimension of a launch

static int type_bytes(int32_t type) { return type == SCORCH_TYPE_F32 ? 4 : type == SCORCH_TYPE_BF16 || type == SCORCH_TYPE_F16 ? 2 : 0; }

// A dense operand of rows x cols elements; `name` for the message.
static scorch_status_t check_dense(const char *call, const char *name, const void *p, int32_t type, int64_t rows, int64_t cols, int64_t ld) {
    if (!type_bytes(type)) {
        set_error("%s: unknown type %d of %s", call, type, name);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (rows == 0 || cols == 0) return SCORCH_OK;
    if (!p) {
        set_error("%s: %s must not be NULL", call, name);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (ld < cols) {
        set_error("%s: row stride %lld of %s is smaller than its %lld columns", call, (long long)ld, name, (long long)cols);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (reinterpret_cast<uintptr_t>(p) % type_bytes(type) != 0) {
        set_error("%s: %s is not aligned to its elements", call, name);
        return SCORCH_ERR_INVALID_ARG;
    }
    return SCORCH_OK;
}

static scorch_status_t check_embedding(const char *call, int32_t tokens, int32_t vocab, int32_t d) {
    if (tokens < 0 || vocab < 0 || d < 0) {
        set_error("%s: negative dimension (tokens=%d vocab=%d d=%d)", call, tokens, vocab, d);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (d > kEmbeddingColumnsMax) {
        set_error("%s: d = %d exceeds %d", call, d, kEmbeddingColumnsMax);
        return SCORCH_ERR_UNSUPPORTED;
    }
    return SCORCH_OK;
}

static scorch_status_t check_distill(const char *call, int32_t rows, int32_t vocab, const void *Z, int32_t z_type, int64_t ldz,
                                     const int32_t *rowptr, float x) {
    if (rows < 0 || vocab < 0) {
        set_error("%s: negative dimension (rows=%d vocab=%d)", call, rows, vocab);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (!(x > 0.f) || !std::isfinite(x * 1.44269504f)) {  // times log2(e): the kernels' powers are of two
        set_error("%s: inv_temperature = %g must be positive and no more than 2.35e38", call, (double)x);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (rows > 0 && !rowptr) {
        set_error("%s: rowptr must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    return check_dense(call, "Z", Z, z_type, rows, vocab, ldz);
}

static scorch_status_t check_distill_gradient(const char *call, int32_t rows, int32_t vocab, const void *Z, int64_t ldz, int32_t z_type,
                                              void *dZ, int64_t lddz) {
    scorch_status_t st = check_dense(call, "dZ", dZ, z_type, rows, vocab, lddz);
    if (st != SCORCH_OK) return st;
    if (dZ == Z && rows > 1 && lddz != ldz && vocab > 0) {
        set_error("%s: dZ is Z with another row stride", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (vocab > SCORCH_DISTILL_VOCAB_MAX) {
        set_error("%s: vocab = %d exceeds the %d columns whose marks fit LDS", call, vocab, SCORCH_DISTILL_VOCAB_MAX);
        return SCORCH_ERR_UNSUPPORTED;
    }
    return SCORCH_OK;
}

}  // namespace scorch

using namespace scorch;

extern "C" {

scorch_status_t scorch_embedding_lookup(int32_t tokens, int32_t vocab, int32_t d, const int32_t *ids, const void *E, int32_t e_type,
                                        int64_t lde, float scale, void *out, int32_t out_type, int64_t ldo, void *stream) {
    const char *call = "embedding lookup";
    scorch_status_t st = check_embedding(call, tokens, vocab, d);
    if (st == SCORCH_OK) st = check_dense(call, "E", E, e_type, vocab, d, lde);
    if (st == SCORCH_OK) st = check_dense(call, "out", out, out_type, tokens, d, ldo);
    if (st != SCORCH_OK || tokens == 0 || d == 0) return st;
    if (!ids) {
        set_error("%s: ids must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    return launch_lookup(tokens, vocab, d, ids, E, e_type, lde, scale, out, out_type, ldo, static_cast<hipStream_t>(stream));
}

scorch_status_t scorch_embedding_gradient_workspace_bytes(int32_t tokens, int32_t vocab, int32_t d, size_t *bytes_out) {
    const char *call = "embedding gradient workspace";
    if (!bytes_out) {
        set_error("%s: bytes_out must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    scorch_status_t st = check_embedding(call, tokens, vocab, d);
    if (st == SCORCH_OK) *bytes_out = (size_t)gradient_workspace_bytes(tokens, d);
    return st;
}

scorch_status_t scorch_embedding_gradient(int32_t tokens, int32_t vocab, int32_t d, const int32_t *ids, const void *dout,
                                          int32_t dout_type, int64_t lddo, float scale, int32_t accumulate, void *dE, int32_t de_type,
                                          int64_t ldde, void *workspace, size_t workspace_bytes, void *stream) {
    const char *call = "embedding gradient";
    scorch_status_t st = check_embedding(call, tokens, vocab, d);
    if (st == SCORCH_OK) st = check_dense(call, "dout", dout, dout_type, tokens, d, lddo);
    if (st == SCORCH_OK) st = check_dense(call, "dE", dE, de_type, vocab, d, ldde);
    if (st != SCORCH_OK || vocab == 0 || d == 0 || (tokens == 0 && accumulate)) return st;
    if (tokens > 0 && !ids) {
        set_error("%s: ids must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) {
        set_error("%s: workspace must be a 256-byte aligned device pointer", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (workspace_bytes < gradient_workspace_bytes(tokens, d)) {
        set_error("%s: workspace of %zu bytes is smaller than the %llu needed", call, workspace_bytes,
                  (unsigned long long)gradient_workspace_bytes(tokens, d));
        return SCORCH_ERR_WORKSPACE_TOO_SMALL;
    }
    return launch_gradient(tokens, vocab, d, ids, dout, dout_type, lddo, scale, accumulate != 0, dE, de_type, ldde,
                           static_cast<char *>(workspace), static_cast<hipStream_t>(stream));
}

scorch_status_t scorch_distill_loss(int32_t rows, int32_t vocab, const void *Z, int32_t z_type, int64_t ldz, const int32_t *rowptr,
                                    const int32_t *colidx, const float *vals, float inv_temperature, float *loss, float *stats,
                                    void *stream) {
    const char *call = "distillation loss";
    scorch_status_t st = check_distill(call, rows, vocab, Z, z_type, ldz, rowptr, inv_temperature);
    if (st != SCORCH_OK || rows == 0) return st;
    if (!loss || !stats) {
        set_error("%s: loss and stats must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    return launch_distill(1, rows, vocab, Z, z_type, ldz, rowptr, colidx, vals, inv_temperature, nullptr, loss, stats, nullptr, 0,
                          static_cast<hipStream_t>(stream));
}

scorch_status_t scorch_distill_gradient(int32_t rows, int32_t vocab, const void *Z, int32_t z_type, int64_t ldz, const int32_t *rowptr,
                                        const int32_t *colidx, const float *vals, float inv_temperature, const float *stats,
                                        const float *dloss, void *dZ, int64_t lddz, void *stream) {
    const char *call = "distillation gradient";
    scorch_status_t st = check_distill(call, rows, vocab, Z, z_type, ldz, rowptr, inv_temperature);
    if (st == SCORCH_OK) st = check_distill_gradient(call, rows, vocab, Z, ldz, z_type, dZ, lddz);
    if (st != SCORCH_OK || rows == 0 || vocab == 0) return st;
    if (!stats) {
        set_error("%s: stats must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    return launch_distill(2, rows, vocab, Z, z_type, ldz, rowptr, colidx, vals, inv_temperature, dloss, nullptr, const_cast<float *>(stats),
                          dZ, lddz, static_cast<hipStream_t>(stream));
}

scorch_status_t scorch_distill_loss_gradient(int32_t rows, int32_t vocab, const void *Z, int32_t z_type, int64_t ldz,
                                             const int32_t *rowptr, const int32_t *colidx, const float *vals, float inv_temperature,
                                             const float *dloss, float *loss, void *dZ, int64_t lddz, void *stream) {
    const char *call = "distillation loss and gradient";
    scorch_status_t st = check_distill(call, rows, vocab, Z, z_type, ldz, rowptr, inv_temperature);
    if (st == SCORCH_OK) st = check_distill_gradient(call, rows, vocab, Z, ldz, z_type, dZ, lddz);
    if (st != SCORCH_OK || rows == 0) return st;
    if (!loss) {
        set_error("%s: loss must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    return launch_distill(3, rows, vocab, Z, z_type, ldz, rowptr, colidx, vals, inv_temperature, dloss, loss, nullptr, dZ, lddz,
                          static_cast<hipStream_t>(stream));
}

scorch_status_t scorch_logits_process(int32_t rows, int32_t vocab, const void *logits, int32_t type, int64_t ldl,
                                      const scorch_logits_rules_t *rules, void *out, int32_t out_type, int64_t ldo, void *stream) {
    const char *call = "logits";
    if (rows < 0 || vocab < 0) {
        set_error("%s: negative dimension (rows=%d vocab=%d)", call, rows, vocab);
        return SCORCH_ERR_INVALID_ARG;
    }
    scorch_status_t st = check_dense(call, "logits", logits, type, rows, vocab, ldl);
    if (st == SCORCH_OK) st = check_dense(call, "out", out, out_type, rows, vocab, ldo);
    if (st != SCORCH_OK || rows == 0 || vocab == 0) return st;
    if (!rules) {
        set_error("%s: rules must not be NULL", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (out == logits && (out_type != type || (rows > 1 && ldo != ldl))) {
        set_error("%s: out is logits with another type or row stride", call);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (rules->mask && rules->ldm < ((int64_t)vocab + 31) / 32) {
        set_error("%s: mask rows of %lld words are shorter than the %lld of %d columns", call, (long long)rules->ldm,
                  (long long)(((int64_t)vocab + 31) / 32), vocab);
        return SCORCH_ERR_INVALID_ARG;
    }
    return launch_logits(rows, vocab, logits, type, ldl, *rules, out, out_type, ldo, static_cast<hipStream_t>(stream));
}

}  // extern "C"
