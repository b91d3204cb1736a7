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

extern "C" int avq_list_log_probs(const void *points, int32_t type, int64_t n, int32_t d, int64_t ld_points, const void *queries, int32_t nq, int64_t ld_queries, float scale,
                                  const int32_t *ids, int32_t m, const float *offset, float *logp_out, float *lse_out, void *hip_stream)
{
    AVQ_TRY(check_probs(type, n, d, nq, m, scale));
    AVQ_TRY(check_rows(points, n, d, ld_points, type, "points"));
    AVQ_TRY(check_rows(queries, nq, d, ld_queries, type, "queries"));
    if (nq > 0) {
        if (!lse_out) return refuse("lse_out is NULL");
        if (m > 0 && (!ids || !logp_out)) return refuse("ids and logp_out are needed for m > 0");
    }
    return launch_list_probs(ListParams{points, type, n, d, ld_points, queries, nq, ld_queries, scale, ids, m, offset, logp_out, lse_out}, (hipStream_t)hip_stream);
}

extern "C" int64_t avq_list_log_probs_grad_scratch(int64_t n, int32_t d, int32_t nq, int32_t m)
{
    if (check_probs(AVQ_F32, n, d, nq, m, 1.0f) != AVQ_OK) return AVQ_EINVAL;
    return (int64_t)list_grad_scratch_bytes(n, d, nq, m);
}

extern "C" int avq_list_log_probs_grad(const void *points, int32_t type, int64_t n, int32_t d, int64_t ld_points, const void *queries, int32_t nq, int64_t ld_queries, float scale,
                                       const int32_t *ids, int32_t m, const float *logp, const float *grad_logp, const float *grad_lse, float *doffset, void *dqueries,
                                       int64_t ld_dqueries, void *dpoints, int64_t ld_dpoints, int32_t accumulate, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    AVQ_TRY(check_probs(type, n, d, nq, m, scale));
    AVQ_TRY(check_rows(points, n, d, ld_points, type, "points"));
    AVQ_TRY(check_rows(queries, nq, d, ld_queries, type, "queries"));
    if (dqueries) AVQ_TRY(check_rows(dqueries, nq, d, ld_dqueries, type, "dqueries"));
    if (dpoints) AVQ_TRY(check_rows(dpoints, n, d, ld_dpoints, type, "dpoints"));
    if (nq > 0 && m > 0 && (!ids || !logp || !grad_logp || !doffset)) return refuse("ids, logp, grad_logp and doffset are needed for m > 0");
    AVQ_TRY(check_scratch(scratch, scratch_bytes, list_grad_scratch_bytes(n, d, nq, m)));
    return launch_list_grad(ListGradParams{points, type, n, d, ld_points, queries, nq, ld_queries, scale, ids, m, logp, grad_logp, grad_lse, doffset, dqueries, ld_dqueries, dpoints,
                                           ld_dpoints, accumulate != 0, scratch},
                            (hipStream_t)hip_stream);
}

namespace {

int check_distill(const DistillParams &p)
{
    AVQ_TRY(check_type(p.type));
    AVQ_TRY(check_count(p.rows));
    if (p.m < 0 || p.m > kMaxGiven) { set_error("m must be 0 .. %d, got %d", kMaxGiven, p.m); return AVQ_EINVAL; }
    AVQ_TRY(check_rows(p.teacher, p.m > 0 ? p.rows : 0, p.m, p.ld_teacher, p.type, "teacher"));
    if (!(p.temperature >= 1e-6 && p.temperature <= 1e6)) return refuse("temperature must be 1e-6 .. 1e6");
    if (p.rows > 0 && p.m > 0 && !p.logp) return refuse("logp is NULL");
    return AVQ_OK;
}

constexpr int kMaxSequences = 1 << 23;

int check_sequences(const float *logp, int64_t tokens, const int32_t *offsets, int32_t sequences)
{
    AVQ_TRY(check_count(tokens));
    if (sequences < 0 || sequences > kMaxSequences) { set_error("sequences must be 0 .. %d, got %d", kMaxSequences, sequences); return AVQ_EINVAL; }
    if (tokens > 0 && !logp) return refuse("logp is NULL");
    if (sequences > 0 && !offsets) return refuse("offsets is NULL");
    return AVQ_OK;
}

// the gradient's part of the arguments
int check_upstream(const float *grad_loss, const float *grad_logp, int64_t losses, int64_t tokens)
{
    if (losses > 0 && !grad_loss) return refuse("grad_loss is NULL");
    return tokens > 0 && !grad_logp ? refuse("grad_logp is NULL") : AVQ_OK;
}

int check_preference(const PreferenceParams &p)
{
    if (p.pairs < 0 || p.pairs > kMaxSequences / 2) { set_error("pairs must be 0 .. %d, got %d", kMaxSequences / 2, p.pairs); return AVQ_EINVAL; }
    AVQ_TRY(check_sequences(p.logp, p.tokens, p.offsets, 2 * p.pairs));
    if (!std::isfinite(p.beta) || !std::isfinite(p.margin)) return refuse("beta and margin must be finite");
    if (!(p.smoothing >= 0.0 && p.smoothing <= 1.0)) return refuse("smoothing must be 0 .. 1");
    return p.pairs > 0 && (!p.loss || !p.logit) ? refuse("loss_out and logit_out are needed") : AVQ_OK;
}

int check_policy(const PolicyParams &p)
{
    AVQ_TRY(check_sequences(p.logp, p.tokens, p.offsets, p.sequences));
    if (p.tokens > 0 && !p.old) return refuse("old is NULL");
    if (!p.advantage && (p.each ? p.tokens : p.sequences) > 0) return refuse("advantage is NULL");
    if (!(p.clip_low >= 0.0 && p.clip_low <= 1.0)) return refuse("clip_low must be 0 .. 1");
    if (!(std::isfinite(p.clip_high) && p.clip_high >= 0.0)) return refuse("clip_high must be finite and not negative");
    if (!(std::isfinite(p.kl_weight) && p.kl_weight >= 0.0)) return refuse("kl_weight must be finite and not negative");
    if (p.kl_weight != 0.0 && !p.ref && p.tokens > 0) return refuse("kl_weight needs ref");
    return p.sequences > 0 && !p.loss ? refuse("loss_out is NULL") : AVQ_OK;
}

} // namespace

extern "C" int avq_distill_loss(const float *logp, const void *teacher, int32_t type, int64_t rows, int32_t m, int64_t ld_teacher, const float *teacher_lse, double temperature,
                                float *loss_out, void *hip_stream)
{
    const DistillParams p{logp, teacher, type, ld_teacher, teacher_lse, temperature, rows, m, loss_out, nullptr, nullptr};
    AVQ_TRY(check_distill(p));
    if (rows > 0 && !loss_out) return refuse("loss_out is NULL");
    return launch_distill(p, (hipStream_t)hip_stream);
}

extern "C" int avq_distill_loss_grad(const float *logp, const void *teacher, int32_t type, int64_t rows, int32_t m, int64_t ld_teacher, const float *teacher_lse, double temperature,
                                     const float *grad_loss, float *loss_out, float *grad_logp, void *hip_stream)
{
    const DistillParams p{logp, teacher, type, ld_teacher, teacher_lse, temperature, rows, m, loss_out, grad_loss, grad_logp};
    AVQ_TRY(check_distill(p));
    AVQ_TRY(check_upstream(grad_loss, grad_logp, rows, rows * m));
    return launch_distill(p, (hipStream_t)hip_stream);
}

extern "C" int64_t avq_preference_loss_scratch(int64_t tokens, int32_t pairs)
{
    if (check_count(tokens) != AVQ_OK || pairs < 0 || pairs > kMaxSequences / 2) return refuse("tokens must be 0 .. 2^28 and pairs 0 .. 2^22");
    return (int64_t)preference_scratch_bytes(tokens, pairs);
}

extern "C" int avq_preference_loss(const float *logp, const float *ref, const uint8_t *mask, int64_t tokens, const int32_t *offsets, int32_t pairs, double beta, double margin,
                                   double smoothing, int32_t average, float *loss_out, float *logit_out, float *reward_out, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    const PreferenceParams p{logp, ref, mask, tokens, offsets, pairs, beta, margin, smoothing, average != 0, loss_out, logit_out, reward_out, nullptr, nullptr, scratch};
    AVQ_TRY(check_preference(p));
    AVQ_TRY(check_scratch(scratch, scratch_bytes, preference_scratch_bytes(tokens, pairs)));
    return launch_preference(p, (hipStream_t)hip_stream);
}

extern "C" int avq_preference_loss_grad(const float *logp, const float *ref, const uint8_t *mask, int64_t tokens, const int32_t *offsets, int32_t pairs, double beta, double margin,
                                        double smoothing, int32_t average, const float *grad_loss, float *loss_out, float *logit_out, float *reward_out, float *grad_logp, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    const PreferenceParams p{logp, ref, mask, tokens, offsets, pairs, beta, margin, smoothing, average != 0, loss_out, logit_out, reward_out, grad_loss, grad_logp, scratch};
    AVQ_TRY(check_preference(p));
    AVQ_TRY(check_upstream(grad_loss, grad_logp, pairs, tokens));
    AVQ_TRY(check_scratch(scratch, scratch_bytes, preference_scratch_bytes(tokens, pairs)));
    return tokens == 0 && pairs == 0 ? AVQ_OK : launch_preference(p, (hipStream_t)hip_stream);
}

extern "C" int64_t avq_policy_loss_scratch(int64_t tokens, int32_t sequences)
{
    if (check_count(tokens) != AVQ_OK || sequences < 0 || sequences > kMaxSequences) return refuse("tokens must be 0 .. 2^28 and sequences 0 .. 2^23");
    return (int64_t)policy_scratch_bytes(tokens, sequences);
}

extern "C" int avq_policy_loss(const float *logp, const float *old, const float *ref, const float *advantage, int32_t each, const uint8_t *mask, int64_t tokens,
                               const int32_t *offsets, int32_t sequences, double clip_low, double clip_high, double kl_weight, int32_t average, float *loss_out, float *kl_out,
                               float *clipped_out, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    const PolicyParams p{logp, old, ref, advantage, each != 0, mask, tokens, offsets, sequences, clip_low, clip_high, kl_weight, average != 0, loss_out, kl_out, clipped_out, nullptr,
                         nullptr, scratch};
    AVQ_TRY(check_policy(p));
    AVQ_TRY(check_scratch(scratch, scratch_bytes, policy_scratch_bytes(tokens, sequences)));
    return launch_policy(p, (hipStream_t)hip_stream);
}

extern "C" int avq_policy_loss_grad(const float *logp, const float *old, const float *ref, const float *advantage, int32_t each, const uint8_t *mask, int64_t tokens,
                                    const int32_t *offsets, int32_t sequences, double clip_low, double clip_high, double kl_weight, int32_t average, const float *grad_loss,
                                    float *loss_out, float *kl_out, float *clipped_out, float *grad_logp, void *scratch, int64_t scratch_bytes, void *hip_stream)
{
    const PolicyParams p{logp, old, ref, advantage, each != 0, mask, tokens, offsets, sequences, clip_low, clip_high, kl_weight, average != 0, loss_out, kl_out, clipped_out, grad_loss,
                         grad_logp, scratch};
    AVQ_TRY(check_policy(p));
    AVQ_TRY(check_upstream(grad_loss, grad_logp, sequences, tokens));
    AVQ_TRY(check_scratch(scratch, scratch_bytes, policy_scratch_bytes(tokens, sequences)));
    return tokens == 0 && sequences == 0 ? AVQ_OK : launch_policy(p, (hipStream_t)hip_stream);
}
