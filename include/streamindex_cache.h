/*
 * libstreamindex -- a compressed cache that is held in 4 bits and bounded in length, for serving.
 * Same library, same conventions as streamindex.h: caller-owned device pointers, contiguous row-major,
 * 16-byte aligned (start, lengths and new_lengths 4-byte; other alignments are refused); work is enqueued on `stream` and the call returns
 * without synchronising; nothing is allocated; only kernel launches are enqueued, so a call can be
 * captured into a HIP graph; argument errors are reported before anything is launched.  Two calls
 * that share a workspace, or of which one writes what the other reads or writes, must not overlap in time.
 *
 * The format.  A row of D values is D codes of 4 bits and D / 32 scale bytes:
 *   code   1 sign bit, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives;
 *          value i is in byte i / 2 of the row, in the low half where i is even;
 *   scale  byte e + 127 of the power 2^e that values 32 j .. 32 j + 31 are multiples of, -13 <= e <= 13.
 * The cache is codes [B,T,D/2] and scales [B,T,D/32] bytes: 68 bytes a row of 128 in place of 256 in bf16.
 * What a row's codes stand for is exact in bf16 and in fp16.  Scale bytes outside 114 .. 140 make no sense; no call writes them.
 */
#ifndef STREAMINDEX_CACHE_H
#define STREAMINDEX_CACHE_H

#include "streamindex.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits, SI_ERR_UNSUPPORTED_SHAPE beyond them: D as stated at each call; for the attention and its weights H <= 64, k <= 4096,
 * n_win <= 4096, B S <= 2^24 - 8, T <= 2^30; for the eviction T <= 2^30, B < 2^22, and
 * B times T / 256 (rounded up) below 2^24. */

/* Rows into the cache: row n of batch b becomes cache row start[b] + n.
 *   rows   device [B,S,D] bf16     S new rows a batch (dims->S; dims->H_I is not used); D = 32, 64 or 128
 *   start  device [B] int32        NULL = 0.  Rows that would fall outside 0 .. T-1 are not stored.
 *   codes  device [B,T,D/2] bytes, scales device [B,T,D/32] bytes; other rows stay as they are
 * e is the least exponent for which no value of the block exceeds 7 * 2^e (6 is the largest code and 7 is off by
 * as much as 5 is: half a step), at least -13, at most 13; values go to the nearest code, ties to the even one,
 * beyond 6 to 6.  So a value is off by at most 2^e (0.25 2^e below 2^(e+1)), one smaller than 2^-15 may become 0, and
 * 6 * 2^13 is the largest value there is: larger ones and infinities become it.  A NaN becomes a number of its block's
 * largest code and does not count for e. */
si_status si_quantize_rows(const void* rows, const int32_t* start, const si_dims* dims, void* codes, void* scales,
                           void* stream);

/* Rows out of the cache, as the values the codes stand for: row n of batch b is cache row start[b] + n,
 * zeros where that is outside 0 .. T-1.
 *   rows  device [B,S,D] bf16;  the rest as above. */
si_status si_dequantize_rows(const void* codes, const void* scales, const int32_t* start, const si_dims* dims, void* rows,
                             void* stream);

/* si_sparse_attention (streamindex_attention.h) on a cache held in 4 bits, whose batches may hold different numbers of rows:
 *   legal(t)  = min(lengths[b], T) for SI_MASK_NONE, min(lengths[b], T, floor((t+1)/m)) for the causal mode;
 *   Window(t) = the last min(n_win, legal(t)) legal rows;
 *   U(t)      = entries of the query's list in 0 .. min(lengths[b], T) - 1, and Window(t), as a set (the list's
 *               entries must be distinct; others than these, such as the pad -1, are skipped);
 *   out[b,t,h,:] = sum_{s in U(t)} p_s V[b,s,:],  p = softmax over U(t) of scale * <qa[b,t,h,:], V[b,s,:]>,
 *   lse[b,t,h]   = ln sum_{s in U(t)} exp(scale * <qa[b,t,h,:], V[b,s,:]>)
 * with V the values of the cache's rows; out = 0 and lse = -inf where U(t) is empty.
 *   qa       device [B,S,H,D] bf16  (dims->H_I carries H, 1..64; D = 64 or 128)
 *   lengths  device [B] int32       rows that a batch holds; NULL = T
 *   idx      device [B,S,k] int32   0 <= k <= 4096; may be NULL with k = 0
 *   out      device [B,S,H,D] f32,  lse device [B,S,H] f32 or NULL
 * fp32 products, statistics and sums; the weights enter the second product with 22 mantissa bits, or to 2^-32 of their sum where that
 * is more.  A head's values and scale may be as far apart as they like: what is lost is what fp32 loses of the logits.
 * Lists that si_indexer_topk makes are of all T rows: where batches hold fewer, rows behind lengths[b] take places in them, which are skipped here.
 * A caller keeps such rows from being chosen by a call of si_indexer_topk a batch, with that batch's rows as T; otherwise a list holds that many fewer.
 * A head whose query is not finite, or whose logits are not, gets NaN in out and lse, and no other head does.  scale has to be finite,
 * scale * log2(e) too (SI_ERR_INVALID_ARG).
 * No workspace.  The same call gives the same bits; calls of other numbers of queries may differ in a query's last places. */
si_status si_quantized_attention(const void* qa, const void* codes, const void* scales, const int32_t* lengths,
                                 const int32_t* idx, const si_dims* dims, int32_t m, int32_t k, si_mask_mode mask_mode,
                                 int32_t n_win, float scale, float* out, float* lse, void* stream);

/* What the rows of the cache receive of the softmax of a call of si_quantized_attention:
 *   weights[b,s] += sum over t with s in U(t) and over h of exp(scale * <qa[b,t,h,:], V[b,s,:]> - lse[b,t,h])
 * Arguments as of that call, and
 *   lse        device [B,S,H] f32    as that call wrote it
 *   weights    device [B,T] f32      rows that are in no U(t) stay as they are
 *   workspace  device, si_accumulate_workspace_bytes(dims) bytes: none with S = 1 (may be NULL then), else 8 B T
 * A query with a head whose lse is NaN adds nothing; no other adds more than H to a row.
 * A query's heads are summed in fp32, queries in 64-bit fixed point, in units of the power of two at or above S H over 2^63, so that the same
 * call gives the same bits: what a query gives a row is off by half a unit beside fp32's rounding, and S = 1 has no units.  An lse is as good as
 * fp32, so a weight is off by about |lse| 2^-23 relative to itself. */
size_t si_accumulate_workspace_bytes(const si_dims* dims);
si_status si_accumulate_weights(const void* qa, const void* codes, const void* scales, const int32_t* lengths,
                                const int32_t* idx, const si_dims* dims, int32_t m, int32_t k, si_mask_mode mask_mode,
                                int32_t n_win, float scale, const float* lse, float* weights, void* workspace,
                                size_t workspace_bytes, void* stream);

/* An array whose rows belong to the cache's rows: row_bytes bytes each, src [B,T,row_bytes] -> dst [B,n_keep,row_bytes]. */
typedef struct {
    const void* src;
    void* dst;
    int32_t row_bytes;
} si_row_move;
#define SI_MAX_ROW_MOVES 8

/* Eviction.  Of the n = min(lengths[b], T) rows that batch b holds, min(n, n_keep) stay: the first n_sink, the last n_recent, and
 * of the others those with the largest weights (ties: the smaller row; NaN is the smallest weight).
 *   weights      device [B,T] f32
 *   lengths      device [B] int32, NULL = T
 *   moves        host array of n_moves <= SI_MAX_ROW_MOVES: the rows that stay are copied from src to dst, in the order they had;
 *                rows of dst behind them stay as they are.  dst must overlap neither another array of the call nor src.
 *                row_bytes >= 1; src and dst aligned to 16 bytes.
 *   kept         device [B,n_keep] int32: the rows that stay, ascending, then -1
 *   new_lengths  device [B] int32 or NULL: how many stay (may be `lengths` itself; small calls then take two launches in place of one)
 *   workspace    device, si_evict_workspace_bytes(B, T) bytes
 * 1 <= n_keep <= T; n_sink, n_recent >= 0, n_sink + n_recent <= n_keep. */
size_t si_evict_workspace_bytes(int32_t B, int32_t T);
si_status si_evict_rows(const float* weights, const int32_t* lengths, int32_t B, int32_t T, int32_t n_keep, int32_t n_sink,
                        int32_t n_recent, const si_row_move* moves, int32_t n_moves, int32_t* kept, int32_t* new_lengths,
                        void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* STREAMINDEX_CACHE_H */
