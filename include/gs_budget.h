/*
 * gs_budget.h - a field held to a budget of Gaussians. The field (gs.h) is
 * attention of the query p over the Gaussians: Phi = sum p_i v_i with the
 * attention weights p_i = a_i / I, a_i = w_i G_i, I = sum a_i. Here the weight
 * that every Gaussian gets is accumulated over the batches of training
 * (gs_shares), a set is cut down to the Gaussians that got most of it
 * (gs_evict), Gaussians - or the samples of the next batch - are drawn by
 * given random numbers (gs_draw), and drawn Gaussians are copied, their weight
 * shared between the copies, which leaves the field as it was (gs_split; the
 * paper's Sec. 4.2.1 describes such copies). Same library and conventions as
 * gs.h: device pointers the caller owns, work enqueued on the caller's stream
 * (nothing here waits), gs_status codes with gs_last_error(), no device memory
 * allocated by the library. Every call may be captured into a HIP graph, and
 * the same inputs give bit-identical results. Calls that share a workspace
 * follow each other. Outputs and the workspace overlap neither inputs nor each
 * other; a call whose arrays do is refused (GS_ERR_INVALID_ARGUMENT).
 */
#ifndef GS_BUDGET_H
#define GS_BUDGET_H

#include "gs_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of workspace of gs_shares for an index (built) and a query; (size_t)-1
 * for invalid arguments. */
size_t gs_shares_work_bytes(const gs_index *index, const gs_query *query);

/*
 * The attention weight that the Gaussians get from a batch of queries, added
 * to their decaying scores:
 *   score[i] <- decay score[i] + w_i sum_t f_t G_i(p_t)   over Q_i(p_t) <= 2 ln(1/tau)
 *   f_t = gain[t] / influence[t] where influence[t] > 0, and 0 elsewhere
 * with gain null: 1 for every query. influence is I as gs_sample wrote it for
 * this index and query (0 where the field is undefined); a caller may set
 * elements to 0 to leave queries out. Queries outside the domain count for
 * nothing, whatever their influence. gain may hold any finite numbers (the
 * error of a sample, say). With gain null the new weights of all Gaussians add
 * up to the number of defined queries, up to rounding and to the pairs at the
 * cutoff (below). For VOXELS, POINTS and JITTER queries
 * plan must be the one that gs_sample (or gs_plan_queries and
 * gs_sample_planned) filled for this index and query; influence is read from
 * the caller's array, not from the plan. gauss must be the Gaussians that the
 * index was built from, unchanged. decay = 0 overwrites score without reading
 * it (0 <= decay, finite). score and work overlap no input (the Gaussians, the
 * index's arrays, the query's, the plan, influence and gain).
 * The sums are float32, those of a Gaussian that very many queries reach joined
 * in float64, in an order that the inputs alone fix. Pairs whose Q
 * is so near the cutoff that float32 cannot tell are decided in float64 from
 * gauss (the sampler decides them in float32: of a pair that the two take
 * differently, tau w_i / I is missing in the sum or too much).
 */
gs_status gs_shares(const gs_gaussians *gauss, const gs_index *index, const gs_query *query, const void *plan,
                    size_t plan_bytes, const float *influence, const float *gain, float decay, float *score,
                    void *work, size_t work_bytes, hipStream_t stream);

/* Bytes of workspace of gs_evict for n Gaussians (-1 cast to size_t for n out
 * of range). */
size_t gs_evict_work_bytes(int64_t n);

/*
 * Cuts a set of n Gaussians down to the first min(budget, n) in this order:
 * those with pinned[i] != 0 before all others (null: none; the newest ones,
 * say, whose score has not had time to grow), then by score from largest to
 * smallest (a NaN is the least score, -0 equals 0), then by index. The kept
 * ones stand in out in the order of their indices: source[j] is the input
 * index of row j, rising with j, as gs_adamw_carry takes it, and score_out[j]
 * its score (null: not wanted). out, source and score_out have room for
 * min(budget, n) rows. 0 <= n, budget < 2^31.
 */
gs_status gs_evict(const gs_params *in, int64_t n, const float *score, const uint8_t *pinned, int64_t budget,
                   const gs_params *out, int32_t *source, float *score_out, void *work, size_t work_bytes,
                   hipStream_t stream);

/* Settings of gs_draw. */
typedef struct gs_draw_params {
    double temperature; /* finite, >= 0; 0: the best candidate, always */
    double top_p;       /* in [0, 1]; 1: off */
    double min_p;       /* in [0, 1]; 0: off */
    int64_t top_k;      /* >= 0; 0: off */
    int32_t logits;     /* 0: scores are weights >= 0, otherwise logits */
    int32_t type;       /* GS_SCORE_F32 or GS_SCORE_BF16 */
} gs_draw_params;
enum { GS_SCORE_F32 = 0, GS_SCORE_BF16 = 1 };

/* Bytes of workspace of gs_draw for any settings (-1 cast to size_t for sizes
 * out of range). */
size_t gs_draw_work_bytes(int64_t rows, int64_t n, int64_t draws);

/*
 * Draws from rows of n candidates, with replacement, by given random numbers:
 * draw d of row r is ids[r draws + d], a function of the row and of
 * uniform[r draws + d] alone. scores[r stride + j], j < n, is the score of
 * candidate j, as a weight x (mass x^(1/T); one that is not > 0 is never
 * drawn) or as a logit x (mass exp(x / T)); NaN is never drawn. lengths (null:
 * n for every row) cuts row r to its first lengths[r] candidates. The masses
 * are held as whole numbers against the row's best candidate, formed in
 * float64:
 *   q_j = (x_j / max)^(1/T) or exp((x_j - max) / T), times 2^k, rounded to the nearest,
 *   k = min(52, 62 - ceil(log2 n))
 * (where max is infinite: 2^k for those that equal it, 0 for the others; a
 * candidate of less than 2^-(k+1) of the best one's mass is never drawn).
 * Then, with candidates ordered by score from largest to smallest and equal
 * ones by index:
 *   top_k: the first top_k stay;
 *   top_p: of these, those stay before which there is at most
 *          floor(top_p 2^53) M / 2^53 (rounded down) of mass, M the mass of
 *          all of these: the shortest beginning with more than top_p of it;
 *   min_p: of these, those stay with q_j >= min_p 2^k.
 * With U = floor(uniform 2^53) (uniform below 0 or NaN counts as 0, from 1 on
 * as 1 - 2^-53) and M the mass of those that stay, the draw is the first j,
 * in the order of the row, with sum_{i <= j} q_i > U M / 2^53 (rounded down),
 * and prob (null: not wanted) q_j / M. All sums are exact, so the draws do
 * not depend on how the work is cut. temperature 0 draws the first of the
 * largest scores, with prob 1. A row in which nothing can be drawn (no
 * candidates, or none with mass) gives id -1 and prob 0. Numbers in rising
 * order draw ids in rising order, which reads memory line by line, here and
 * where gs_split copies what was drawn (419430 of 2 M Gaussians: 65 -> 55 us
 * and 78 -> 37).
 * A row of up to 16384 candidates, or one of which top_k leaves up to 1024, is
 * drawn by one workgroup: many draws from it take 1 to 4 ns each.
 * 0 <= rows, n < 2^31, 0 <= draws < 2^31, rows n and rows draws below 2^40.
 */
gs_status gs_draw(int64_t rows, int64_t n, const void *scores, int64_t stride, const int32_t *lengths,
                  const gs_draw_params *params, int64_t draws, const double *uniform, int32_t *ids, float *prob,
                  void *work, size_t work_bytes, hipStream_t stream);

/* Bytes of workspace of gs_split for n Gaussians (-1 cast to size_t for n out
 * of range). */
size_t gs_split_work_bytes(int64_t n);

/*
 * Copies of drawn Gaussians, in place: set has room for n + count rows, and
 * row n + j becomes a copy of row ids[j] < n. With c = 1 + the number of
 * times a Gaussian is in ids, it and its copies get its activated weight
 * over c, w / c, as weight logit -ln((c - 1) + c e^-logit) (float64, rounded
 * once), so the field is unchanged (up to that rounding); c = 1 leaves it
 * alone. score[n + count] (null: none) is shared the same way: score / c.
 * source[n + j] = -1 - ids[j] (null: not wanted): a new Gaussian for
 * gs_adamw_carry, so its moments start at 0; source[0 .. n) is left alone.
 * An id outside [0, n) makes a Gaussian that contributes nothing: its mean is
 * NaN, its log-scale 0, its rotation (1, 0, 0, 0), its value logit 0, its
 * weight logit -infinity, its score 0, and source is -1 - id (-1 for a negative
 * id). n + count < 2^31. No two of the set's arrays, ids, source, score and
 * work overlap.
 */
gs_status gs_split(const gs_params *set, int64_t n, const int32_t *ids, int64_t count, int32_t *source, float *score,
                   void *work, size_t work_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GS_BUDGET_H */
