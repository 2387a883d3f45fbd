/*
 * Float64 CPU oracle for the speculative-decoding verify step
 * (appending the draft block to the paged cache, attention of the draft block,
 * accept / resample, GammaTune controller, GammaTune+ early stop of drafting).
 *
 * TEST INFRASTRUCTURE ONLY.  This file is the slow, plain definition that the
 * CUDA library is checked against.  It shares no code with the CUDA path and
 * must never be called from it; only the tests, the smoke check and the
 * benchmark's CPU-baseline leg may load it.
 *
 * Every routine is written as the definition (attention) or as the steps of
 * the procedure in the order the paper and the speculative-sampling rule state
 * them (accept / resample, Algorithm 1): no blocking, no fusion, no
 * reordering.  The only parallelism is an OpenMP loop over independent
 * sequences / query rows, which does not change any arithmetic.
 *
 * Compile with -ffp-contract=off so that (1-eta)*gbar + eta*A is two
 * multiplications and one addition, each rounded once (IEEE binary64).
 */
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

/* ------------------------------------------------------------------------- */
/* bf16 storage format: the upper 16 bits of an IEEE binary32 value.          */
static double bf16_bits_to_f64(uint16_t h)
{
    uint32_t u = ((uint32_t)h) << 16;
    float f;
    memcpy(&f, &u, sizeof f);
    return (double)f;
}

/* =========================================================================
 * 1. Attention of the draft block against the paged KV cache.
 *
 * Paper, Section 3 ("Background"): the target model verifies the gamma drafted
 * tokens in one parallel forward; with KV caching (Section 5) the part of that
 * forward that grows with context is causal softmax attention of the
 * gamma+1 new positions against the cache.  This is the textbook definition:
 *
 *   s_j = scale * sum_d q[d] k_j[d]          j = 0 .. n_keys-1
 *   m   = max_j s_j ;  Z = sum_j exp(s_j - m)
 *   o[d] = sum_j exp(s_j - m) v_j[d] / Z ;   lse = m + ln Z
 *
 * KV token j of a sequence lives in physical page block_table[j / page_size],
 * slot j % page_size.  kv_strides = element strides of the pool for
 * (page, kv head, slot, dim).
 * ========================================================================= */
void oracle_attn_row(const uint16_t *q_row, const uint16_t *k_pool, const uint16_t *v_pool,
                     const int64_t *kv_strides, const int32_t *block_table_row, int page_size,
                     int kv_head, int head_dim, int n_keys, double scale, double *o, double *lse)
{
    double *s = (double *)malloc(sizeof(double) * (size_t)(n_keys > 0 ? n_keys : 1));
    double m = -INFINITY;
    for (int j = 0; j < n_keys; ++j) {
        int64_t page = block_table_row[j / page_size];
        int64_t slot = j % page_size;
        const uint16_t *k = k_pool + page * kv_strides[0] + (int64_t)kv_head * kv_strides[1] +
                            slot * kv_strides[2];
        double dot = 0.0;
        for (int d = 0; d < head_dim; ++d)
            dot += bf16_bits_to_f64(q_row[d]) * bf16_bits_to_f64(k[(int64_t)d * kv_strides[3]]);
        s[j] = dot * scale;
        if (s[j] > m) m = s[j];
    }
    double Z = 0.0;
    for (int d = 0; d < head_dim; ++d) o[d] = 0.0;
    for (int j = 0; j < n_keys; ++j) {
        int64_t page = block_table_row[j / page_size];
        int64_t slot = j % page_size;
        const uint16_t *v = v_pool + page * kv_strides[0] + (int64_t)kv_head * kv_strides[1] +
                            slot * kv_strides[2];
        double e = exp(s[j] - m);
        Z += e;
        for (int d = 0; d < head_dim; ++d)
            o[d] += e * bf16_bits_to_f64(v[(int64_t)d * kv_strides[3]]);
    }
    for (int d = 0; d < head_dim; ++d) o[d] /= Z;
    if (lse) *lse = m + log(Z);
    free(s);
}

/*
 * All rows of a ragged batch.  Sequence b has gamma[b]+1 query rows, stored at
 * rows cu_q[b] .. cu_q[b+1]-1 of q [sum R, hq, head_dim]; they are the LAST
 * gamma[b]+1 positions of the sequence (seq_len[b] counts them), so row i sees
 * keys 0 .. seq_len[b]-(gamma[b]+1)+i inclusive.  Query head h reads kv head
 * h / (hq / hkv).
 */
void oracle_verify_attn(const uint16_t *q, const uint16_t *k_pool, const uint16_t *v_pool,
                        const int64_t *kv_strides, const int32_t *block_table,
                        int64_t block_table_stride, const int32_t *seq_len, const int32_t *gamma,
                        const int32_t *cu_q, int batch, int hq, int hkv, int head_dim,
                        int page_size, double scale, double *o, double *lse)
{
    int group = hq / hkv;
    for (int b = 0; b < batch; ++b) {
        int R = gamma[b] + 1;
        int L = seq_len[b];
        int64_t n_items = (int64_t)R * hq;
#pragma omp parallel for schedule(dynamic, 1)
        for (int64_t it = 0; it < n_items; ++it) {
            int i = (int)(it / hq);
            int h = (int)(it % hq);
            int pos = L - R + i;
            int64_t row = (int64_t)cu_q[b] + i;
            oracle_attn_row(q + (row * hq + h) * head_dim, k_pool, v_pool, kv_strides,
                            block_table + (int64_t)b * block_table_stride, page_size, h / group,
                            head_dim, pos + 1, scale, o + (row * hq + h) * head_dim,
                            lse ? lse + row * hq + h : NULL);
        }
    }
}

/* -------------------------------------------------------------------------
 * 1b. Appending the draft block to the cache (KV caching, paper Section 5,
 *     experimental setup).  Before the verify attention runs, the keys and
 *     values of the gamma[b]+1 new positions are written behind the context:
 *     new row i of sequence b is token  pos = seq_len[b] - (gamma[b]+1) + i
 *     (seq_len already counts the block), which lives in physical page
 *     block_table[b][pos / page_size], slot pos % page_size.  A plain copy of
 *     bf16 bit patterns; every other element of the pools is left alone.
 *     k_new, v_new: [sum R, hkv, head_dim].
 * ------------------------------------------------------------------------- */
void oracle_kv_append(const uint16_t *k_new, const uint16_t *v_new, uint16_t *k_pool, uint16_t *v_pool,
                      const int64_t *kv_strides, const int32_t *block_table, int64_t block_table_stride,
                      const int32_t *seq_len, const int32_t *gamma, const int32_t *cu_q, int batch,
                      int hkv, int head_dim, int page_size)
{
    for (int b = 0; b < batch; ++b) {
        int R = gamma[b] + 1;
        for (int i = 0; i < R; ++i) {
            int pos = seq_len[b] - R + i;
            int64_t page = block_table[(int64_t)b * block_table_stride + pos / page_size];
            int64_t slot = pos % page_size;
            for (int g = 0; g < hkv; ++g) {
                int64_t dst = page * kv_strides[0] + (int64_t)g * kv_strides[1] + slot * kv_strides[2];
                int64_t src = (((int64_t)cu_q[b] + i) * hkv + g) * head_dim;
                for (int d = 0; d < head_dim; ++d) {
                    k_pool[dst + (int64_t)d * kv_strides[3]] = k_new[src + d];
                    v_pool[dst + (int64_t)d * kv_strides[3]] = v_new[src + d];
                }
            }
        }
    }
}

/* =========================================================================
 * 2. Accept / resample (speculative sampling, paper Section 3, first
 *    paragraph, by reference to Leviathan et al. and Chen et al.).
 * ========================================================================= */

/* softmax of x/T in float64: p_k = exp(x_k/T - m) / sum_j exp(x_j/T - m).
 * Returns ln sum_j exp(x_j / T). */
static double softmax_f64(const float *x, int V, double T, double *p)
{
    double m = -INFINITY;
    for (int k = 0; k < V; ++k) {
        double z = (double)x[k] / T;
        if (z > m) m = z;
    }
    double Z = 0.0;
    for (int k = 0; k < V; ++k) {
        p[k] = exp((double)x[k] / T - m);
        Z += p[k];
    }
    for (int k = 0; k < V; ++k) p[k] /= Z;
    return m + log(Z);
}

/* index of the largest element, lowest index on ties */
static int argmax_lowest(const float *x, int V)
{
    int best = 0;
    for (int k = 1; k < V; ++k)
        if (x[k] > x[best]) best = k;
    return best;
}

/*
 * Inverse CDF in vocabulary order: smallest k with sum_{j<=k} w_j > u * W,
 * W = sum_j w_j.  Zero-weight tokens are never chosen; if rounding leaves no
 * such k the last token with positive weight is taken.
 * Near-edge report: if u*W lies within tol*W of the lower (upper) CDF edge of
 * the chosen token, *alt is the previous (next) token with positive weight
 * and *flag is set; both tokens are then legal answers for a float32 device.
 */
static int inv_cdf(const double *w, int V, double u, double tol, int *alt, uint8_t *flag)
{
    double W = 0.0;
    for (int k = 0; k < V; ++k) W += w[k];
    double target = u * W;
    double c = 0.0, lower = 0.0, upper = 0.0;
    int y = -1;
    for (int k = 0; k < V; ++k) {
        double c_next = c + w[k];
        if (w[k] > 0.0 && c_next > target) {
            y = k;
            lower = c;
            upper = c_next;
            break;
        }
        c = c_next;
    }
    if (y < 0) {
        for (int k = V - 1; k >= 0; --k)
            if (w[k] > 0.0) { y = k; break; }
        lower = W - (y >= 0 ? w[y] : 0.0);
        upper = W;
    }
    *alt = -1;
    *flag = 0;
    if (y >= 0) {
        if (target - lower < tol * W) {
            for (int k = y - 1; k >= 0; --k)
                if (w[k] > 0.0) { *alt = k; *flag = 1; break; }
        } else if (upper - target < tol * W) {
            for (int k = y + 1; k < V; ++k)
                if (w[k] > 0.0) { *alt = k; *flag = 1; break; }
        }
    }
    return y;
}

/*
 * One verify step for a ragged batch.
 *
 * Row layout: sequence b owns target rows cu_q[b] .. cu_q[b]+gamma[b]
 * (row i is the target distribution for draft position i; row gamma[b] is the
 * bonus position) and draft rows / tokens / uniforms cu_d[b] .. cu_d[b]+gamma[b]-1.
 *
 * T > 0, for i = 0 .. gamma-1 in order:
 *     p_i = softmax(t_i / T), q_i = softmax(d_i / T)
 *     ratio_i = min(1, p_i[x_i] / q_i[x_i])            (1 if q_i[x_i] == 0)
 *     accept iff u_i < ratio_i ; the first rejection ends the scan: n = i
 *   n < gamma : next token ~ normalise(max(0, p_n - q_n))   (p_n if that mass is 0)
 *   n = gamma : next token ~ p_gamma                         (bonus token)
 *   both by inverse CDF with u_sample[b].
 * T == 0: n = first i with argmax(t_i) != x_i, next token = argmax(t_n).
 *
 * force (nullable, one per draft position): -1 = decide by the rule,
 * 0 / 1 = take this decision instead.  A comparison harness uses it to follow
 * the device through a position the oracle itself reports as a near tie.
 *
 * Outputs: n_accepted[b] (accepted draft tokens, 0..gamma, the extra token not
 * counted); out_tokens[b, 0..n-1] = accepted drafts, [n] = next token, rest -1;
 * ratio / accept_flag per draft position (NaN / 0 where the scan never got);
 * logZ_p per target row, logZ_q per draft row (ln sum exp(x/T); NaN if T == 0);
 * alt_token / sample_flag / resid_mass per sequence.
 */
void oracle_accept_sample(const float *target_logits, const float *draft_logits, int64_t row_stride,
                          int V, const int32_t *draft_tokens, const float *u_accept,
                          const float *u_sample, const float *temperature, const int32_t *gamma,
                          const int32_t *cu_q, const int32_t *cu_d, int batch, int gamma_max,
                          const int8_t *force, double accept_tol, double sample_tol,
                          int32_t *n_accepted, int32_t *out_tokens, double *ratio, double *logZ_p,
                          double *logZ_q, uint8_t *accept_flag, int32_t *alt_token,
                          uint8_t *sample_flag, double *resid_mass)
{
#pragma omp parallel for schedule(dynamic, 1)
    for (int b = 0; b < batch; ++b) {
        int g = gamma[b];
        double T = (double)temperature[b];
        const float *t_rows = target_logits + (int64_t)cu_q[b] * row_stride;
        const float *d_rows = draft_logits + (int64_t)cu_d[b] * row_stride;
        const int32_t *x = draft_tokens + cu_d[b];
        int32_t *out = out_tokens + (int64_t)b * (gamma_max + 1);
        for (int i = 0; i <= gamma_max; ++i) out[i] = -1;
        for (int i = 0; i < g; ++i) {
            ratio[cu_d[b] + i] = NAN;
            accept_flag[cu_d[b] + i] = 0;
            logZ_q[cu_d[b] + i] = NAN;
        }
        for (int i = 0; i <= g; ++i) logZ_p[cu_q[b] + i] = NAN;
        alt_token[b] = -1;
        sample_flag[b] = 0;
        resid_mass[b] = NAN;

        int n = g;
        int y;
        if (T == 0.0) {
            for (int i = 0; i < g; ++i) {
                int top = argmax_lowest(t_rows + (int64_t)i * row_stride, V);
                int ok = (top == x[i]);
                if (force && force[cu_d[b] + i] >= 0) ok = force[cu_d[b] + i];
                if (!ok) { n = i; break; }
            }
            y = argmax_lowest(t_rows + (int64_t)n * row_stride, V);
        } else {
            double *p = (double *)malloc(sizeof(double) * (size_t)V);
            double *q = (double *)malloc(sizeof(double) * (size_t)V);
            double *w = (double *)malloc(sizeof(double) * (size_t)V);
            for (int i = 0; i < g; ++i) {
                logZ_p[cu_q[b] + i] = softmax_f64(t_rows + (int64_t)i * row_stride, V, T, p);
                logZ_q[cu_d[b] + i] = softmax_f64(d_rows + (int64_t)i * row_stride, V, T, q);
                double r = 1.0;
                if (q[x[i]] > 0.0) {
                    r = p[x[i]] / q[x[i]];
                    if (r > 1.0) r = 1.0;
                }
                double u = (double)u_accept[cu_d[b] + i];
                ratio[cu_d[b] + i] = r;
                accept_flag[cu_d[b] + i] = (fabs(u - r) < accept_tol) ? 1 : 0;
                int ok = (u < r);
                if (force && force[cu_d[b] + i] >= 0) ok = force[cu_d[b] + i];
                if (!ok) { n = i; break; }
            }
            /* p, q still hold rows n when the scan stopped at a rejection */
            if (n < g) {
                double W = 0.0;
                for (int k = 0; k < V; ++k) {
                    w[k] = p[k] - q[k];
                    if (w[k] < 0.0) w[k] = 0.0;
                    W += w[k];
                }
                resid_mass[b] = W;
                if (!(W > 0.0))
                    for (int k = 0; k < V; ++k) w[k] = p[k];
            } else {
                logZ_p[cu_q[b] + g] = softmax_f64(t_rows + (int64_t)g * row_stride, V, T, w);
            }
            int alt;
            uint8_t fl;
            y = inv_cdf(w, V, (double)u_sample[b], sample_tol, &alt, &fl);
            alt_token[b] = alt;
            sample_flag[b] = fl;
            free(p);
            free(q);
            free(w);
        }
        n_accepted[b] = n;
        for (int i = 0; i < n; ++i) out[i] = x[i];
        out[n] = y;
    }
}

/* =========================================================================
 * 3. GammaTune controller, paper Section 4.1, Algorithm 1, per sequence.
 *
 *   mode 1 (reading "proposed"): the expansion rule of Eq. 7 raises the
 *       acceptance count that feeds the moving average, as the prose of the
 *       "Adaptive Expansion" paragraph says:
 *           A' = A + delta  if A == gamma  else A
 *           gbar <- min(gmax, max(gmin, (1-eta)*gbar + eta*A'))      (Eq. 8)
 *           gamma <- ceil(gbar)
 *   mode 2 (reading "literal"): Algorithm 1 exactly as printed, where the
 *       assignment gamma <- A + delta is overwritten by the last line, so
 *       the average is fed A itself.
 *   mode 0: fixed gamma (plain speculative decoding); state is left alone.
 *
 * Bookkeeping around it (implied by KV caching): the block just verified had
 * gamma+1 positions appended; A+1 of them stay; the next block appends
 * gamma_next+1:  seq_len <- seq_len - (gamma+1) + (A+1) + (gamma_next+1).
 * cu_q / cu_d are rebuilt as prefix sums of gamma_next+1 / gamma_next (packed
 * rows), or as b*(gamma_max+1) / b*gamma_max when padded_rows is set (every
 * sequence owns a fixed slab of rows, of which it uses the first gamma+1).
 * ========================================================================= */
void oracle_gamma_tune_update(const int32_t *n_accepted, double *gamma_bar, int32_t *gamma,
                              int32_t *seq_len, int32_t *cu_q, int32_t *cu_d, int batch,
                              double eta, double delta, int gamma_min, int gamma_max, int mode,
                              int padded_rows, const int32_t *n_drafted)
{
    /* n_drafted (GammaTune+, Section 4.2; NULL for plain GammaTune): the draft stopped after
     * n_drafted[b] <= gamma[b] tokens, so that many rows (+1) were appended to the cache; the
     * comparison "A = gamma" still uses the gamma the controller issued. */
    cu_q[0] = 0;
    cu_d[0] = 0;
    for (int b = 0; b < batch; ++b) {
        int A = n_accepted[b];
        int g_old = gamma[b];
        int rows_old = (n_drafted != NULL ? n_drafted[b] : g_old) + 1;
        int g_new = g_old;
        if (mode == 1 || mode == 2) {
            double a_eff = (double)A;
            if (A == g_old) {
                if (mode == 1) a_eff = (double)A + delta;
                /* mode 2: gamma <- A + delta here, but it is overwritten below */
            }
            double t1 = (1.0 - eta) * gamma_bar[b];
            double t2 = eta * a_eff;
            double s = t1 + t2;
            if (s < (double)gamma_min) s = (double)gamma_min;
            if (s > (double)gamma_max) s = (double)gamma_max;
            gamma_bar[b] = s;
            g_new = (int)ceil(s);
        }
        gamma[b] = g_new;
        seq_len[b] = seq_len[b] - rows_old + (A + 1) + (g_new + 1);
        cu_q[b + 1] = padded_rows ? (b + 1) * (gamma_max + 1) : cu_q[b] + g_new + 1;
        cu_d[b + 1] = padded_rows ? (b + 1) * gamma_max : cu_d[b] + g_new;
    }
}

/*
 * GammaTune+ (Section 4.2): confidence-guided early stop of drafting.  The draft's confidence
 * at position i is its top probability c_i = max_k softmax(d_i / T)_k.  The paper only says
 * that drafting stops when it falls below tau; the reading taken here: the token drafted at
 * the first such position is still part of the block, nothing is drafted after it, so
 *     n_drafted = min(gamma, 1 + first i with c_i < tau)      (gamma if there is none).
 * T = 0 (greedy draft): c_i = 1, never below tau <= 1.
 * flag[row] = 1 when |c_i - tau| < tol (either decision is legal there).
 */
void oracle_draft_stop(const float *draft_logits, int64_t row_stride, int vocab, const float *temperature,
                       double tau, const int32_t *gamma, const int32_t *cu_d, int batch, double tol,
                       int32_t *n_drafted, double *top_prob, uint8_t *flag)
{
    for (int b = 0; b < batch; ++b) {
        const int g = gamma[b];
        const double T = (double)temperature[b];
        int n = g;
        for (int i = 0; i < g; ++i) {
            const float *d = draft_logits + (int64_t)(cu_d[b] + i) * row_stride;
            double c = 1.0;
            if (T > 0.0) {
                double m = -INFINITY;
                for (int k = 0; k < vocab; ++k)
                    if ((double)d[k] > m) m = (double)d[k];
                double z = 0.0;
                for (int k = 0; k < vocab; ++k) z += exp(((double)d[k] - m) / T);
                c = 1.0 / z;
            }
            top_prob[cu_d[b] + i] = c;
            flag[cu_d[b] + i] = fabs(c - tau) < tol ? 1 : 0;
            if (n == g && c < tau) n = i + 1 < g ? i + 1 : g;
        }
        n_drafted[b] = n;
    }
}

/*
 * One drafting step with the confidence stop (paper Section 4.2: the draft model's top
 * probability is looked at while it drafts, and drafting ends once it falls below tau).
 *
 * Row b of draft_logits holds sequence b's draft logits for its next position.  For every
 * sequence with active[b] != 0 (and n_drafted[b] < gamma[b]):
 *     q = softmax(d / T);  token ~ q by inverse CDF with u[b]  (T == 0: token = argmax d, lowest index)
 *     c = max_k q_k                                                (T == 0: c = 1)
 *     draft_tokens[cu_d[b] + n_drafted[b]] = token, top_prob[same] = c, n_drafted[b] += 1
 *     active[b] = (c >= tau) && (n_drafted[b] < gamma[b])
 * The token drawn at a position whose confidence is below tau is kept (it is the last one
 * drafted), as in oracle_draft_stop.  Sequences that are not active are left untouched.
 * alt_token / sample_flag report a draw within tol of a CDF edge (see inv_cdf); conf_flag[b] = 1
 * when |c - tau| < conf_tol (either decision is legal there).
 */
void oracle_draft_step(const float *draft_logits, int64_t row_stride, int vocab, const float *temperature,
                       double tau, const float *u, const int32_t *gamma, const int32_t *cu_d, int batch,
                       double tol, double conf_tol, int32_t *n_drafted, int32_t *active,
                       int32_t *draft_tokens, double *top_prob, int32_t *alt_token, uint8_t *sample_flag,
                       uint8_t *conf_flag)
{
    double *q = (double *)malloc((size_t)(vocab > 0 ? vocab : 1) * sizeof(double));
    for (int b = 0; b < batch; ++b) {
        alt_token[b] = -1;
        sample_flag[b] = 0;
        conf_flag[b] = 0;
        if (!active[b]) continue;
        if (n_drafted[b] >= gamma[b]) { active[b] = 0; continue; }
        const float *d = draft_logits + (int64_t)b * row_stride;
        const double T = (double)temperature[b];
        int token;
        double c = 1.0;
        if (T > 0.0) {
            softmax_f64(d, vocab, T, q);
            int alt; uint8_t fl;
            token = inv_cdf(q, vocab, (double)u[b], tol, &alt, &fl);
            alt_token[b] = alt;
            sample_flag[b] = fl;
            c = 0.0;
            for (int k = 0; k < vocab; ++k)
                if (q[k] > c) c = q[k];
        } else {
            token = argmax_lowest(d, vocab);
        }
        const int pos = cu_d[b] + n_drafted[b];
        draft_tokens[pos] = token;
        top_prob[pos] = c;
        conf_flag[b] = fabs(c - tau) < conf_tol ? 1 : 0;
        n_drafted[b] += 1;
        active[b] = (c >= tau) && (n_drafted[b] < gamma[b]);
    }
    free(q);
}

/* gamma = gamma0, gbar = gamma0 for every sequence, plus the prefix sums. */
void oracle_gamma_tune_init(double *gamma_bar, int32_t *gamma, int32_t *cu_q, int32_t *cu_d,
                            int batch, int gamma0, int gamma_max, int padded_rows)
{
    cu_q[0] = 0;
    cu_d[0] = 0;
    for (int b = 0; b < batch; ++b) {
        gamma_bar[b] = (double)gamma0;
        gamma[b] = gamma0;
        cu_q[b + 1] = padded_rows ? (b + 1) * (gamma_max + 1) : cu_q[b] + gamma0 + 1;
        cu_d[b + 1] = padded_rows ? (b + 1) * gamma_max : cu_d[b] + gamma0;
    }
}

/* =========================================================================
 * 4. Cost model of paper Section 3 (Eq. 2-6), in units of T_draft:
 *    cost = N / (alpha*gamma + 1) * (c + gamma).  Analysis only.
 * ========================================================================= */
double oracle_cost_model(double n_tokens, double alpha, double gamma, double c)
{
    double n_steps = n_tokens / (alpha * gamma + 1.0);      /* Eq. 3 */
    double calls_target = n_steps;                          /* Eq. 4 */
    double calls_draft = gamma * n_steps;                   /* Eq. 5 */
    return c * calls_target + 1.0 * calls_draft;            /* Eq. 2 with T_draft = 1, T_target = c */
}

/* =========================================================================
 * 6. Block tables and slot maps from the sequences' lengths (KV caching, paper
 *    Section 5): the sequential walk over the batch.  Pages given back are
 *    pushed on the free stack first, then pages asked for are popped, both in
 *    the order of the batch; the first sequence that does not get all its pages
 *    gets none and neither does any behind it.  Returns the condition bits
 *    (1 bad gamma, 2 bad page / count, 32 bad length, 64 out of pages).
 * ========================================================================= */
int oracle_kv_pages_update(const int32_t *seq_len, int batch, int32_t *block_table, int64_t stride,
                           int32_t *n_held, int32_t *free_list, int32_t *n_free, int64_t n_pages,
                           const int32_t *gamma, const int32_t *cu_q, int gamma_max, int64_t *slot_map,
                           int32_t *positions, int64_t n_rows)
{
    int cond = 0;
    int64_t top = *n_free;
    if (top < 0) { top = 0; cond |= 2; }
    if (top > n_pages) { top = n_pages; cond |= 2; }
    uint8_t *ok = (uint8_t *)malloc((size_t)batch);
    uint8_t *has = (uint8_t *)malloc((size_t)batch);
    for (int b = 0; b < batch; ++b) {
        int64_t need = ((int64_t)seq_len[b] + 15) / 16;
        ok[b] = seq_len[b] >= 0 && need <= stride && n_held[b] >= 0 && n_held[b] <= stride;
        has[b] = ok[b];
        if (!ok[b]) { cond |= 32; continue; }
        int64_t held = n_held[b];
        for (int64_t c = need; c < held; ++c) {
            int32_t *e = block_table + b * stride + c;
            if (*e < 0 || *e >= n_pages) cond |= 2;
            if (top < n_pages) free_list[top++] = *e;
            else cond |= 2;
            *e = -1;
        }
        if (need < held) n_held[b] = (int32_t)need;
    }
    int out = 0;
    for (int b = 0; b < batch; ++b) {
        if (!ok[b]) continue;
        int64_t need = ((int64_t)seq_len[b] + 15) / 16;
        int64_t want = need - n_held[b];
        if (want <= 0) continue;
        if (out || want > top) { out = 1; has[b] = 0; cond |= 64; continue; }
        while (n_held[b] < need) block_table[b * stride + n_held[b]++] = free_list[--top];
    }
    *n_free = (int32_t)top;
    for (int64_t r = 0; r < n_rows; ++r) {
        if (slot_map) slot_map[r] = -1;
        if (positions) positions[r] = -1;
    }
    for (int b = 0; b < batch && (slot_map || positions); ++b) {
        int g = gamma[b];
        if (g < 0 || g > gamma_max) { cond |= 1; g = g < 0 ? 0 : gamma_max; }
        if (!ok[b] || seq_len[b] == 0) continue;
        if (seq_len[b] < g + 1) { cond |= 32; continue; }
        if (!has[b]) continue;
        for (int i = 0; i <= g; ++i) {
            int64_t r = (int64_t)cu_q[b] + i;
            if (r >= cu_q[b + 1] || r >= n_rows) break;
            int pos = seq_len[b] - (g + 1) + i;
            int32_t page = block_table[b * stride + pos / 16];
            if (page < 0 || page >= n_pages) { cond |= 2; continue; }
            if (slot_map) slot_map[r] = (int64_t)page * 16 + pos % 16;
            if (positions) positions[r] = pos;
        }
    }
    free(ok);
    free(has);
    return cond;
}

/* =========================================================================
 * 7. Norm, rotation and append of one row's heads (KV caching, paper Section 5).
 *    One head of D bf16 values: y = x * w / sqrt(mean x^2 + eps) (y = x without
 *    weights), then each pair (a, b) turned by pos * inv_freq and scaled.
 *    z: the result in float64 (not rounded); mag: scale * (|y_a| + |y_b|) of the
 *    element's pair (|y_d| outside the rotated dims), the scale that rounding
 *    errors of the result are measured against.
 * ========================================================================= */
void oracle_norm_rotate(const uint16_t *x, int D, const double *weight, double eps, const double *angle, int rot_dim,
                        int interleaved, double scale, double *z, double *mag)
{
    double ss = 0.0;
    for (int d = 0; d < D; ++d) {
        z[d] = bf16_bits_to_f64(x[d]);
        ss += z[d] * z[d];
    }
    if (weight)
        for (int d = 0; d < D; ++d) z[d] = z[d] * weight[d] / sqrt(ss / D + eps);
    for (int d = 0; d < D; ++d) mag[d] = fabs(z[d]);
    for (int f = 0; f < rot_dim / 2; ++f) {
        int a = interleaved ? 2 * f : f, b = interleaved ? 2 * f + 1 : f + rot_dim / 2;
        double ya = z[a], yb = z[b], c = cos(angle[f]), s = sin(angle[f]);
        z[a] = scale * (ya * c - yb * s);
        z[b] = scale * (yb * c + ya * s);
        mag[a] = mag[b] = fabs(scale) * (fabs(ya) + fabs(yb));
    }
}

/* rows [n, heads, D] (row r starts at r * stride): heads of every row through oracle_norm_rotate */
void oracle_norm_rotate_rows(const uint16_t *x, int64_t stride, int n, int heads, int D, const double *weight, double eps,
                             const int32_t *positions, const uint8_t *freq_axis, const double *inv_freq, int rot_dim,
                             int interleaved, double scale, double *z, double *mag)
{
#pragma omp parallel for schedule(static)
    for (int r = 0; r < n; ++r) {
        double angle[1024];
        for (int f = 0; f < rot_dim / 2; ++f)
            angle[f] = (double)positions[(freq_axis ? (int64_t)freq_axis[f] * n : 0) + r] * inv_freq[f];
        for (int h = 0; h < heads; ++h) {
            int64_t o = ((int64_t)r * heads + h) * D;
            oracle_norm_rotate(x + r * stride + (int64_t)h * D, D, weight, eps, angle, rot_dim, interleaved, scale, z + o, mag + o);
        }
    }
}

/* =========================================================================
 * 8. Penalties, biases and grammar masks on logit rows, and the token counts
 *    behind the penalties: the definition, element by element in float64.
 *    out: the unrounded result; mag: sum of the magnitudes of its terms (the
 *    scale of float32 rounding errors).  Rows that belong to no sequence are left.
 * ========================================================================= */
static void adjust_row(const float *x, int V, const int16_t *counts, const int32_t *drafts, int n_before, double rep, double freq,
                       double pres, const int32_t *bias_tokens, const float *bias_values, int n_bias, const uint32_t *mask,
                       double *out, double *mag)
{
    int32_t *c = (int32_t *)calloc((size_t)V, sizeof(int32_t));
    double *bias = (double *)calloc((size_t)V, sizeof(double));
    for (int j = 0; j < n_before; ++j)
        if (drafts[j] >= 0 && drafts[j] < V) c[drafts[j]] += 1;
    for (int e = 0; e < n_bias; ++e)                     /* the later entry counts */
        if (bias_tokens[e] >= 0 && bias_tokens[e] < V) bias[bias_tokens[e]] = bias_values[e];
    for (int k = 0; k < V; ++k) {
        double v = x[k];
        uint16_t h = counts ? (uint16_t)counts[k] : 0;
        int n = c[k] + (h & 0x7fff);
        if (counts) {
            if (n > 0 || (h & 0x8000)) v = v > 0 ? v / rep : v * rep;
            mag[k] = fabs(v) + fabs(freq * n) + (n > 0 ? fabs(pres) : 0.0) + fabs(bias[k]);
            v -= freq * n + (n > 0 ? pres : 0.0);
        } else {
            mag[k] = fabs(v) + fabs(bias[k]);
        }
        v += bias[k];
        if (mask && !((mask[k / 32] >> (k % 32)) & 1u)) {
            v = -INFINITY;
            mag[k] = 0.0;
        }
        out[k] = v;
    }
    free(c);
    free(bias);
}

void oracle_logits_adjust(const float *logits, int64_t stride, int V, int batch, const int32_t *gamma, const int32_t *cu_q,
                          const int32_t *cu_d, const int32_t *n_drafted, const int32_t *draft_tokens, const int16_t *counts,
                          int64_t count_stride, const float *rep, const float *freq, const float *pres, const int32_t *bias_tokens,
                          const float *bias_values, const int32_t *n_bias, int bias_stride, const uint32_t *mask,
                          int64_t mask_stride, double *out, double *mag)
{
    int penal = rep || freq || pres;
#pragma omp parallel for schedule(dynamic)
    for (int b = 0; b < batch; ++b) {
        int rows = n_drafted ? 1 : gamma[b] + 1;
        for (int i = 0; i < rows; ++i) {
            int64_t r = n_drafted ? b : (int64_t)cu_q[b] + i;
            adjust_row(logits + r * stride, V, penal ? counts + b * count_stride : NULL, draft_tokens + (cu_d ? cu_d[b] : 0),
                       penal ? (n_drafted ? n_drafted[b] : i) : 0, rep ? rep[b] : 1.0, freq ? freq[b] : 0.0, pres ? pres[b] : 0.0,
                       bias_tokens + (int64_t)b * bias_stride, bias_values + (int64_t)b * bias_stride, n_bias ? n_bias[b] : 0,
                       mask ? mask + r * mask_stride : NULL, out + r * V, mag + r * V);
        }
    }
}

/* tokens of b: tokens[first[b]] .. tokens[first[b] + n[b] - 1]; entries outside [0, V) are skipped */
void oracle_token_counts_update(int16_t *counts, int64_t stride, int V, int batch, const int32_t *tokens, const int64_t *first,
                                const int32_t *n, const int32_t *reset, int prompt)
{
    for (int b = 0; b < batch; ++b) {
        int16_t *row = counts + b * stride;
        if (reset && reset[b])
            for (int k = 0; k < V; ++k) row[k] = 0;
        for (int j = 0; j < n[b]; ++j) {
            int32_t t = tokens[first[b] + j];
            if (t < 0 || t >= V) continue;
            uint16_t h = (uint16_t)row[t];
            if (prompt) h |= 0x8000;
            else if ((h & 0x7fff) < 0x7fff) h += 1;
            row[t] = (int16_t)h;
        }
    }
}

/* -------------------------------------------------------------------------
 * Long contexts (KV caching, paper Section 5): a summary of every page's keys,
 * the pages that a row reads by a score on it, attention over listed pages.
 * The summary and the score are defined in float32, every operation rounded
 * once, so that whole numbers and choices can be compared for equality.
 * ------------------------------------------------------------------------- */
static float bf16_bits_to_f32(uint16_t h)
{
    union { uint32_t u; float f; } x;
    x.u = (uint32_t)h << 16;
    return x.f;
}

static int whole(float x, float scale)
{
    if (!(scale > 0.f) || isinf(scale)) return 0;        /* NaN too */
    float n = rintf(x / scale);                          /* half to even: the default rounding mode */
    return n > 127.f ? 127 : n < -127.f ? -127 : (int)n;
}

/* pages first[b] / 16 .. of positions first[b] .. seq_len[b] - 1 of every sequence */
void oracle_page_bounds_update(const uint16_t *k_pool, const int64_t *kv_strides, const int32_t *block_table, int64_t stride,
                               const int32_t *seq_len, const int32_t *first, int batch, int hkv, int D, int page_size,
                               int8_t *bounds, float *scales)
{
    for (int b = 0; b < batch; ++b)
        for (int lp = first[b] / page_size; first[b] < seq_len[b] && lp * page_size < seq_len[b]; ++lp) {
            int64_t page = block_table[b * stride + lp];
            int n = seq_len[b] - lp * page_size < page_size ? seq_len[b] - lp * page_size : page_size;
            for (int h = 0; h < hkv; ++h) {
                float hi[256], lo[256], big = 0.f;
                for (int d = 0; d < D; ++d) {
                    hi[d] = -INFINITY;
                    lo[d] = INFINITY;
                    for (int s = 0; s < n; ++s) {
                        float k = bf16_bits_to_f32(k_pool[page * kv_strides[0] + h * kv_strides[1] + s * kv_strides[2] + d * kv_strides[3]]);
                        if (k > hi[d] || isnan(k)) hi[d] = k;        /* a NaN stays */
                        if (k < lo[d] || isnan(k)) lo[d] = k;
                    }
                    if (fabsf(hi[d]) > big || isnan(hi[d])) big = fabsf(hi[d]);
                    if (fabsf(lo[d]) > big) big = fabsf(lo[d]);
                }
                float scale = big * (1.f / 127.f);
                int8_t *out = bounds + (page * hkv + h) * 2 * D;
                for (int d = 0; d < D; ++d) {
                    out[d] = (int8_t)whole(hi[d], scale);
                    out[D + d] = (int8_t)whole(lo[d], scale);
                }
                scales[page * hkv + h] = scale;
            }
        }
}

/* chosen [n_seen]: 1 for the pages that one row and kv head reads; q: the group's heads [G, D] */
void oracle_page_choice(const uint16_t *q, int G, int D, const int8_t *bounds, const float *scales, int hkv, int head,
                        const int32_t *table, int n_seen, int n_select, int n_first, int n_last, float *score, uint8_t *chosen)
{
    float big = 0.f;
    for (int e = 0; e < G * D; ++e)                      /* a query that is no number leaves none */
        if (fabsf(bf16_bits_to_f32(q[e])) > big || isnan(bf16_bits_to_f32(q[e]))) big = fabsf(bf16_bits_to_f32(q[e]));
    float scale = big * (1.f / 127.f);
    for (int p = 0; p < n_seen; ++p) {
        const int8_t *bd = bounds + ((int64_t)table[p] * hkv + head) * 2 * D;
        int best = 0;
        for (int g = 0; g < G; ++g) {
            int sum = 0;
            for (int d = 0; d < D; ++d) {
                int x = whole(bf16_bits_to_f32(q[g * D + d]), scale), u = x * bd[d], v = x * bd[D + d];
                sum += u > v ? u : v;
            }
            if (g == 0 || sum > best) best = sum;
        }
        score[p] = (float)best * scales[(int64_t)table[p] * hkv + head];
        if (isnan(score[p])) score[p] = INFINITY;            /* no number counts as the highest */
        chosen[p] = (uint8_t)(p < n_first || p >= n_seen - n_last || n_seen <= n_select);
    }
    for (int left = n_select - n_first - n_last; n_seen > n_select && left > 0; --left) {
        int at = -1;
        for (int p = 0; p < n_seen; ++p)
            if (!chosen[p] && (at < 0 || score[p] > score[at])) at = p;      /* the lower page on ties */
        chosen[at] = 1;
    }
}

/* attention of one query row over the given positions; mag[d]: the weighted sum of |v_d|, what rounded weights err by */
void oracle_attn_positions(const uint16_t *q_row, const uint16_t *k_pool, const uint16_t *v_pool, const int64_t *kv_strides,
                           const int32_t *table, int page_size, int kv_head, int D, const int32_t *positions, int n, double scale,
                           double *o, double *mag, double *lse)
{
    double *s = (double *)malloc(sizeof(double) * (size_t)(n > 0 ? n : 1)), m = -INFINITY, Z = 0.0;
    for (int d = 0; d < D; ++d) o[d] = mag[d] = 0.0;
    for (int j = 0; j < n; ++j) {
        const uint16_t *k = k_pool + table[positions[j] / page_size] * kv_strides[0] + kv_head * kv_strides[1] +
                            positions[j] % page_size * kv_strides[2];
        double dot = 0.0;
        for (int d = 0; d < D; ++d) dot += bf16_bits_to_f64(q_row[d]) * bf16_bits_to_f64(k[d * kv_strides[3]]);
        s[j] = dot * scale;
        if (s[j] > m) m = s[j];
    }
    for (int j = 0; j < n; ++j) {
        const uint16_t *v = v_pool + table[positions[j] / page_size] * kv_strides[0] + kv_head * kv_strides[1] +
                            positions[j] % page_size * kv_strides[2];
        double e = exp(s[j] - m);
        Z += e;
        for (int d = 0; d < D; ++d) {
            double x = bf16_bits_to_f64(v[d * kv_strides[3]]);
            o[d] += e * x;
            mag[d] += e * fabs(x);
        }
    }
    for (int d = 0; d < D && n > 0; ++d) {
        o[d] /= Z;
        mag[d] /= Z;
    }
    *lse = n > 0 ? m + log(Z) : -INFINITY;
    free(s);
}

/* listed pages with row masks; n_list NULL: every row reads all of its positions */
void oracle_attn_pages(const uint16_t *q, const uint16_t *k_pool, const uint16_t *v_pool, const int64_t *kv_strides,
                       const int32_t *block_table, int64_t stride, const int32_t *seq_len, const int32_t *gamma, const int32_t *cu_q,
                       int batch, int hq, int hkv, int D, int page_size, const int32_t *page_list, const uint64_t *row_mask,
                       const int32_t *n_list, int64_t list_stride, double scale, double *o, double *mag, double *lse)
{
    int G = hq / hkv;
    for (int b = 0; b < batch; ++b) {
        int R = gamma[b] + 1;
#pragma omp parallel for schedule(dynamic)
        for (int64_t it = 0; it < (int64_t)R * hq; ++it) {
            int i = (int)(it / hq), h = (int)(it % hq), g = h / G, pos = seq_len[b] - R + i, n = 0;
            int32_t *at = (int32_t *)malloc(sizeof(int32_t) * (size_t)(pos + 1));
            if (n_list == NULL) {
                for (n = 0; n <= pos; ++n) at[n] = n;
            } else {
                int64_t base = ((int64_t)b * hkv + g) * list_stride;
                for (int e = 0; e < n_list[b * hkv + g]; ++e) {
                    if (!((row_mask[base + e] >> i) & 1u)) continue;
                    for (int s = 0; s < page_size; ++s) {
                        int t = page_list[base + e] * page_size + s;
                        if (t <= pos) at[n++] = t;
                    }
                }
            }
            int64_t row = ((int64_t)cu_q[b] + i) * hq + h;
            oracle_attn_positions(q + row * D, k_pool, v_pool, kv_strides, block_table + b * stride, page_size, g, D, at, n, scale,
                                  o + row * D, mag + row * D, lse + row);
            free(at);
        }
    }
}
