/*
 * libstreamindex -- dense attention of whole prompts, or of the next part of them, packed one behind the other.  Same library, same
 * conventions as streamindex.h: caller-owned device pointers, contiguous row-major, 16-byte aligned (offsets, first and lse 4-byte; other
 * alignments are refused); work is enqueued on `stream` and the call returns without synchronising; nothing is allocated; only
 * a kernel launch is enqueued, so a call can be captured into a HIP graph; argument errors are reported before anything is launched.  What
 * a call writes must not overlap what it reads in memory, or what another call reads or writes at the same time.
 *
 * Sequence b has the queries q_offsets[b] .. q_offsets[b+1] - 1 and the rows k_offsets[b] .. k_offsets[b+1] - 1 of keys and values.  With
 *   t           = first[b] + i           position of its query i
 *   rows        = k_offsets[b+1] - k_offsets[b]
 *   legal(t)    = rows for SI_MASK_NONE, min(rows, floor((t+1)/m)) for the causal mode (no row where t < 0)
 *   seen(t)     = the last min(n_win, legal(t)) legal rows
 *   x_s         = scale * <q[i,g,:], K[s,h,:]>,  h = g / (H / H_kv): H / H_kv heads of the query share one of keys and values
 *   out[i,g,:]  = sum_{s in seen(t)} exp(x_s - lse) V[s,h,:],   lse[i,g] = ln sum_{s in seen(t)} exp(x_s);
 *   out = 0 and lse = -inf where nothing is seen.
 * m = 1 is causal attention, m > 1 attention over compressed rows, one per m positions (legal(t) of streamindex.h).  A prompt's next
 * part has first = the number of positions before it and the rows of all of them.  (A part of few queries behind many rows is faster by
 * si_paged_attention, which splits the rows over the chip: 128 queries behind 8,192 rows, 64 heads of 128 on 8: 52 us against 137.)
 */
#ifndef STREAMINDEX_PROMPT_H
#define STREAMINDEX_PROMPT_H

#include "streamindex.h"

#ifdef __cplusplus
extern "C" {
#endif

#ifndef SI_ALL_ROWS
#define SI_ALL_ROWS 0x7FFFFFFF /* n_win of a position that sees all its legal rows */
#endif

typedef struct {
    int32_t B;     /* sequences                           */
    int32_t N_q;   /* packed queries                      */
    int32_t N_k;   /* packed rows of keys and values      */
    int32_t H;     /* heads of the queries                */
    int32_t H_kv;  /* heads of keys and values, H a multiple of it */
    int32_t D;     /* 64 or 128                           */
} si_packed_dims;

/*   q          device [N_q,H,D] bf16
 *   K, V       device [N_k,H_kv,D] bf16;  V NULL: a row's keys are its values
 *   q_offsets  device [B + 1] int32, not decreasing, in 0 .. N_q;  NULL: N_q / B queries a sequence (N_q a multiple of B);  k_offsets likewise
 *   first      device [B] int32;  NULL = 0
 *   n_win      >= 0; SI_ALL_ROWS: no window
 *   out        device [N_q,H,D] bf16;  lse device [N_q,H] f32 or NULL.  Queries that belong to no sequence are left as they were.
 * fp32 products, statistics and sums: a logit is infinite where <q,K>, or that times scale * log2(e), passes fp32's range, and finite values give
 * finite results where the number of rows seen times the largest value is at most 2^117, as sums are divided by that of their weights at the end.  A
 * weight exp(x_s - reference) is rounded to bf16 once, as an operand of the second product; lse is made of the weights before that.  A head whose
 * query is not finite, or one of whose logits is NaN or +infinity, gets NaN in out and lse, and no other head does.  A logit of -infinity is a weight of
 * 0 (a finite query with no other logits gets out = 0 and lse = -inf); infinite or NaN values of a row that is seen make infinities or NaN of out where
 * they stand.  What rows hold
 * that a query does not see (later positions, before the window, other sequences) never reaches its result, NaN and infinities included.
 * scale has to be finite, scale * log2(e) too (SI_ERR_INVALID_ARG).  No workspace.  The same call gives the same bits, and no bit of a head's
 * result depends on the queries of other heads or positions.
 * There is at least one query and one row (SI_ERR_INVALID_ARG): where no sequence has a row yet, one that belongs to none.
 * Limits, SI_ERR_UNSUPPORTED_SHAPE beyond them: D = 64 or 128, H <= 1024, N_q, N_k <= 2^30, B <= 2^20, N_q H + 128 B H_kv < 2^30. */
si_status si_prompt_attention(const void* q, const void* K, const void* V, const si_packed_dims* dims, const int32_t* q_offsets,
                              const int32_t* k_offsets, const int32_t* first, int32_t m, si_mask_mode mask_mode, int32_t n_win, float scale,
                              void* out, float* lse, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* STREAMINDEX_PROMPT_H */
