// C ABI of the operators on rows of learned vectors (declared in include/avq.h): argument checking and launches. They hold
// no state: whatever they need beside their arguments is the caller's scratch.
#include <cmath>

#include "avq_internal.h"
#include "probs.h"
#include "row_types.h"

using namespace avq;

namespace {

constexpr int64_t kMaxCount = (int64_t)1 << 28;
constexpr int kMaxRowDim = 16384;
constexpr int kMaxQueries = 1 << 19, kMaxGiven = 4096;

int refuse(const char *what) { set_error("%s", what); return AVQ_EINVAL; }

int check_type(int32_t type)
{
    return type == AVQ_F32 || type == AVQ_BF16 || type == AVQ_F16 ? AVQ_OK : refuse("type must be AVQ_F32, AVQ_BF16 or AVQ_F16");
}

int check_dim(int32_t d)
{
    if (d >= 1 && d <= kMaxRowDim) return AVQ_OK;
    set_error("d must be 1 .. %d, got %d", kMaxRowDim, d);
    return AVQ_EINVAL;
}

// A matrix of `rows` rows: its pointer (needed where there are rows) on a whole element, its rows not over one another.
int check_rows(const void *p, int64_t rows, int32_t d, int64_t ld, int32_t type, const char *what)
{
    if (rows > 0 && !p) { set_error("%s is NULL", what); return AVQ_EINVAL; }
    if (ld < d) { set_error("%s: rows of %d elements, %lld apart", what, d, (long long)ld); return AVQ_EINVAL; }
    if ((uintptr_t)p % type_bytes(type)) { set_error("%s is not aligned to its elements", what); return AVQ_EINVAL; }
    return AVQ_OK;
}

int check_n(int64_t n)
{
    if (n >= 1 && n < ((int64_t)1 << 31)) return AVQ_OK;
    set_error("n must be 1 .. 2^31 - 1, got %lld", (long long)n);
    return AVQ_EINVAL;
}

int check_count(int64_t count)
{
    if (count >= 0 && count <= kMaxCount) return AVQ_OK;
    set_error("count must be 0 .. 2^28, got %lld", (long long)count);
    return AVQ_EINVAL;
}

int check_scratch(const void *scratch, int64_t have, size_t need)
{
    if (need == 0) return AVQ_OK;
    if (!scratch || have < 0 || (uint64_t)have < need) {
        set_error("scratch of %zu bytes needed, got %lld", need, (long long)(scratch ? have : 0));
        return AVQ_EINVAL;
    }
    return (uintptr_t)scratch % 256 ? refuse("scratch must be aligned to 256 bytes") : AVQ_OK;
}

int check_probs(int32_t type, int64_t n, int32_t d, int32_t nq, int32_t given, float scale)
{
    AVQ_TRY(check_type(type));
    AVQ_TRY(check_dim(d));
    AVQ_TRY(check_n(n));
    if (nq < 0 || nq > kMaxQueries) { set_error("nq must be 0 .. %d, got %d", kMaxQueries, nq); return AVQ_EINVAL; }
    if (given < 0 || given > kMaxGiven) { set_error("m must be 0 .. %d, got %d", kMaxGiven, given); return AVQ_EINVAL; }
    if ((int64_t)nq * given > kMaxCount) { set_error("nq x m must be at most 2^28"); return AVQ_EINVAL; }
    if (!std::isfinite(scale) || scale == 0.0f) return refuse("scale must be finite and not 0");
    return AVQ_OK;
}

int check_k(int64_t n, int32_t d, int32_t k)
{
    if (k < 0 || k > AVQ_MAX_SELECT || k > n) { set_error("k must be 0 .. min(n, %d), got %d", AVQ_MAX_SELECT, k); return AVQ_EINVAL; }
    if (finish_lds(d, k) > kFinishLds) { set_error("k = %d alternatives in %d dimensions exceed what a workgroup holds", k, d); return AVQ_EINVAL; }
    return AVQ_OK;
}

} // namespace

namespace avq {

int check_log_probs(const ProbParams &p)
{
    AVQ_TRY(check_probs(p.type, p.n, p.d, p.nq, p.given, p.scale));
    AVQ_TRY(check_k(p.n, p.d, p.k));
    AVQ_TRY(check_rows(p.points, p.n, p.d, p.ld_points, p.type, "points"));
    AVQ_TRY(check_rows(p.queries, p.nq, p.d, p.ld_queries, p.type, "queries"));
    if (p.nq == 0) return AVQ_OK;
    if (!p.lse) return refuse("lse_out is NULL");
    if (p.given > 0 && (!p.ids || !p.logp)) return refuse("ids and logp_out are needed for m > 0");
    if (p.k > 0 && (!p.alt_ids || !p.alt_logp)) return refuse("alt_ids_out and alt_logp_out are needed for k > 0");
    return AVQ_OK;
}

} // namespace avq

extern "C" int avq_embed(const void *table, int32_t type, int64_t n, int32_t d, int64_t ld_table, const int32_t *ids, int64_t count, float scale, void *out, int64_t ld_out,
                         void *hip_stream)
{
    AVQ_TRY(check_type(type));
    AVQ_TRY(check_dim(d));
    AVQ_TRY(check_n(n));
    AVQ_TRY(check_count(count));
    AVQ_TRY(check_rows(table, n, d, ld_table, type, "table"));
    AVQ_TRY(check_rows(out, count, d, ld_out, type, "out"));
    if (count > 0 && !ids) return refuse("ids is NULL");
    return launch_embed(EmbedParams{table, type, n, d, ld_table, ids, count, scale, out, ld_out}, (hipStream_t)hip_stream);
}

extern "C" int64_t avq_embed_grad_scratch(int64_t n, int32_t d, int64_t count)
{
    if (check_dim(d) != AVQ_OK || check_n(n) != AVQ_OK || check_count(count) != AVQ_OK) return AVQ_EINVAL;
    return count == 0 ? 0 : (int64_t)embed_grad_scratch_bytes(n, d, count);
}

extern "C" int avq_embed_grad(const void *grad, int32_t type, int64_t ld_grad, const int32_t *ids, int64_t count, float scale, void *out, int64_t n, int32_t d, int64_t ld_out,
                              int32_t accumulate, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    AVQ_TRY(check_type(type));
    AVQ_TRY(check_dim(d));
    AVQ_TRY(check_n(n));
    AVQ_TRY(check_count(count));
    AVQ_TRY(check_rows(grad, count, d, ld_grad, type, "grad"));
    AVQ_TRY(check_rows(out, n, d, ld_out, type, "out"));
    if (count > 0 && !ids) return refuse("ids is NULL");
    AVQ_TRY(check_scratch(scratch, scratch_bytes, count == 0 ? 0 : embed_grad_scratch_bytes(n, d, count)));
    return launch_embed_grad(EmbedGradParams{grad, type, ld_grad, ids, count, scale, out, n, d, ld_out, accumulate != 0, scratch}, (hipStream_t)hip_stream);
}

extern "C" int avq_layer_norm(const void *x, int32_t type, int64_t rows, int32_t d, int64_t ld_x, const void *weight, const void *bias, float eps, void *y, int64_t ld_y,
                              float *mean, float *rstd, void *hip_stream)
{
    AVQ_TRY(check_type(type));
    AVQ_TRY(check_dim(d));
    AVQ_TRY(check_count(rows));
    AVQ_TRY(check_rows(x, rows, d, ld_x, type, "x"));
    AVQ_TRY(check_rows(y, rows, d, ld_y, type, "y"));
    AVQ_TRY(check_rows(weight, 0, d, d, type, "weight"));
    AVQ_TRY(check_rows(bias, 0, d, d, type, "bias"));
    if (!std::isfinite(eps) || eps < 0.0f) return refuse("eps must be finite and not negative");
    return launch_norm(NormParams{x, type, rows, d, ld_x, weight, bias, eps, y, ld_y, mean, rstd}, (hipStream_t)hip_stream);
}

extern "C" int64_t avq_layer_norm_grad_scratch(int64_t rows, int32_t d)
{
    if (check_dim(d) != AVQ_OK || check_count(rows) != AVQ_OK) return AVQ_EINVAL;
    return (int64_t)norm_grad_scratch_bytes(rows, d);
}

extern "C" int avq_layer_norm_grad(const void *grad, int32_t type, int64_t ld_grad, const void *x, int64_t ld_x, int64_t rows, int32_t d, const float *mean, const float *rstd,
                                   const void *weight, void *dx, int64_t ld_dx, void *dweight, void *dbias, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    AVQ_TRY(check_type(type));
    AVQ_TRY(check_dim(d));
    AVQ_TRY(check_count(rows));
    AVQ_TRY(check_rows(grad, rows, d, ld_grad, type, "grad"));
    AVQ_TRY(check_rows(x, rows, d, ld_x, type, "x"));
    AVQ_TRY(check_rows(dx, rows, d, ld_dx, type, "dx"));
    AVQ_TRY(check_rows(weight, 0, d, d, type, "weight"));
    AVQ_TRY(check_rows(dweight, 0, d, d, type, "dweight"));
    AVQ_TRY(check_rows(dbias, 0, d, d, type, "dbias"));
    if (rows > 0 && (!mean || !rstd)) return refuse("mean and rstd of the forward pass are needed");
    AVQ_TRY(check_scratch(scratch, scratch_bytes, norm_grad_scratch_bytes(rows, d)));
    return launch_norm_grad(NormGradParams{grad, type, ld_grad, x, ld_x, rows, d, mean, rstd, weight, dx, ld_dx, dweight, dbias, scratch}, (hipStream_t)hip_stream);
}

extern "C" int64_t avq_log_probs_scratch(int32_t type, int64_t n, int32_t d, int32_t nq, int32_t m, int32_t k)
{
    if (check_probs(type, n, d, nq, m, 1.0f) != AVQ_OK || check_k(n, d, k) != AVQ_OK) return AVQ_EINVAL;
    return (int64_t)log_probs_scratch_bytes(type, n, d, nq, m, k);
}

extern "C" int avq_log_probs(const void *points, int32_t type, int64_t n, int32_t d, int64_t ld_points, const void *queries, int32_t nq, int64_t ld_queries, float scale,
                             const int32_t *ids, int32_t m, float *logp_out, float *lse_out, float *entropy_out, int32_t k, int32_t *alt_ids_out, float *alt_logp_out,
                             void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    const ProbParams p{points, type, n, d, ld_points, queries, nq, ld_queries, scale, ids, m, logp_out, lse_out, entropy_out, k, alt_ids_out, alt_logp_out, scratch};
    AVQ_TRY(check_log_probs(p));
    AVQ_TRY(check_scratch(scratch, scratch_bytes, log_probs_scratch_bytes(type, n, d, nq, m, k)));
    return launch_log_probs(p, (hipStream_t)hip_stream);
}

extern "C" int64_t avq_log_probs_grad_scratch(int32_t type, int64_t n, int32_t d, int32_t nq, int32_t m)
{
    if (check_probs(type, n, d, nq, m, 1.0f) != AVQ_OK) return AVQ_EINVAL;
    return (int64_t)log_probs_grad_scratch_bytes(type, n, d, nq, m);
}

extern "C" int avq_log_probs_grad(const void *points, int32_t type, int64_t n, int32_t d, int64_t ld_points, const void *queries, int32_t nq, int64_t ld_queries, float scale,
                                  const int32_t *ids, int32_t m, const float *lse, const float *entropy, const float *grad_logp, const float *grad_entropy, const float *grad_lse,
                                  void *dqueries, int64_t ld_dqueries, void *dpoints, int64_t ld_dpoints, int32_t accumulate, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    AVQ_TRY(check_probs(type, n, d, nq, m, scale));
    AVQ_TRY(check_rows(points, n, d, ld_points, type, "points"));
    AVQ_TRY(check_rows(queries, nq, d, ld_queries, type, "queries"));
    if (dqueries) AVQ_TRY(check_rows(dqueries, nq, d, ld_dqueries, type, "dqueries"));
    if (dpoints) AVQ_TRY(check_rows(dpoints, n, d, ld_dpoints, type, "dpoints"));
    if (nq > 0) {
        if (!lse) return refuse("lse of the forward pass is needed");
        if (m > 0 && (!ids || !grad_logp)) return refuse("ids and grad_logp are needed for m > 0");
        if (grad_entropy && !entropy) return refuse("entropy of the forward pass is needed with its gradient");
    }
    AVQ_TRY(check_scratch(scratch, scratch_bytes, log_probs_grad_scratch_bytes(type, n, d, nq, m)));
    return launch_log_probs_grad(ProbGradParams{points, type, n, d, ld_points, queries, nq, ld_queries, scale, ids, m, lse, entropy, grad_logp, grad_entropy, grad_lse, dqueries,
                                                ld_dqueries, dpoints, ld_dpoints, accumulate != 0, scratch},
                                 (hipStream_t)hip_stream);
}
