/*
 * libstreamindex -- dense attention over a paged cache, for serving: rows of keys and values enter the pages of a cache that all
 * requests share, in 16 or 8 bits, and the newest positions of each request attend to all rows it holds, or to a window of them.
 * Same library, same conventions as streamindex.h: caller-owned device pointers, contiguous row-major, 16-byte aligned (offsets, start,
 * lengths, first, table and lse 4-byte; other alignments are refused); work is enqueued on `stream` and the call returns without
 * synchronising; nothing is allocated; only kernel launches are enqueued, so a call can be captured into a HIP graph; argument errors are
 * reported before anything is launched.  Two calls that share a workspace, or of which one writes what the other reads or writes, must not
 * overlap in time; what a call writes must not overlap what it reads in memory.
 *
 * The cache.  n_pages pages of page_rows rows of H_kv heads of D values, keys and values apart: K and V [n_pages, H_kv, page_rows, D].
 * Row s of sequence b is row s % page_rows of page table[b, s / page_rows].  A number outside 0 .. n_pages - 1 (such as -1) says that the
 * page is not there: its rows are not stored, come back as zeros, and no position sees them.  A page may be in several tables.
 *   bits = 16  rows are bf16 as they are.
 *   bits = 8   a row is D codes of 8 bits (1 sign, 4 exponent, 3 mantissa bits; bias 7, no infinities, largest 448, 0x7F and 0xFF are NaN)
 *              and one scale byte e + 127: the row's values are codes * 2^e, -64 <= e <= 63.  129 bytes a row of 128 in place of 256.
 *              What a row's codes stand for is exact in bf16.  Scale bytes outside 63 .. 190 make no sense; no call writes them.
 */
#ifndef STREAMINDEX_PAGES_H
#define STREAMINDEX_PAGES_H

#include "streamindex.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SI_ALL_ROWS 0x7FFFFFFF /* n_win of a position that sees all its legal rows */

typedef struct {
    void* K;                /* device [n_pages, H_kv, page_rows, D] bf16, or bytes of codes                              */
    void* V;                /* the same; NULL: a row's keys are its values (the compressed cache of si_sparse_attention) */
    void* K_scales;         /* device [n_pages, H_kv, page_rows] bytes with bits = 8, not used with 16                   */
    void* V_scales;
    const int32_t* table;   /* device [B, table_pages]                                                                   */
    int32_t B;              /* sequences                                                                                 */
    int32_t table_pages;
    int32_t n_pages;
    int32_t page_rows;      /* 16, 32, 64, .. 1024                                                                       */
    int32_t H_kv;           /* heads                                                                                     */
    int32_t D;              /* 64 or 128                                                                                 */
    int32_t bits;           /* 16 or 8                                                                                   */
} si_paged_cache;

/* Limits, SI_ERR_UNSUPPORTED_SHAPE beyond them: D and page_rows as stated, H and H_kv <= 1024, table_pages * page_rows <= 2^30, B <= 2^20,
 * N <= 2^27 and N * H_kv * D <= 2^36 for rows in and out; B <= 2^14 and B S H <= 2^22 for the attention. */

/* Rows into the cache.  Packed rows offsets[b] .. offsets[b+1] - 1 become rows start[b], start[b] + 1, .. of sequence b; what would fall
 * outside the table is not stored, and what packed rows hold that belong to no sequence does not matter.
 *   k_rows, v_rows  device [N, H_kv, D] bf16    (v_rows is not used where the cache's V is NULL, and may be NULL)
 *   offsets         device [B + 1] int32, not decreasing, in 0 .. N;  NULL: N / B rows a sequence (N a multiple of B)
 *   start           device [B] int32, >= 0;  NULL = 0
 * No row may be stored twice by a call.  bits = 8: e is the least exponent for which no value of the row exceeds 448 * 2^e, at least -64, at
 * most 63; values go to the nearest code, ties to the even one.  So a value is off by at most 2^-4 of itself, or by 2^(e - 10) where it is below
 * 2^(e - 6); 448 * 2^63 is the largest value there is: larger ones and infinities become it.  A NaN stays one and does not count for e. */
si_status si_store_pages(const void* k_rows, const void* v_rows, int32_t N, const int32_t* offsets, const int32_t* start,
                         const si_paged_cache* cache, void* stream);

/* Rows out of the cache, as the values that are held: the way back.  Zeros where the sequence has no such row in its table; packed rows that belong to
 * no sequence stay as they are.
 *   k_rows, v_rows  device [N, H_kv, D] bf16;  either may be NULL, v_rows has to be where the cache's V is. */
si_status si_load_pages(const si_paged_cache* cache, int32_t N, const int32_t* offsets, const int32_t* start, void* k_rows, void* v_rows,
                        void* stream);

/* Attention of S positions of each sequence (1 or a few: the newest token, drafted ones) over the rows that the sequence holds.  With
 *   held        = min(lengths[b], table_pages * page_rows)
 *   t           = first[b] + i           position of query i of 0 .. S - 1
 *   legal(t)    = held for SI_MASK_NONE, min(held, floor((t+1)/m)) for the causal mode (no row where t < 0)
 *   seen(t)     = the last min(n_win, legal(t)) legal rows, without those whose page is not there
 *   x_s         = scale * <q[b,i,g,:], K[s,h,:]>,  h = g / (H / H_kv): H / H_kv heads of the query share one of the cache
 *   out[b,i,g,:] = sum_{s in seen(t)} exp(x_s - lse) V[s,h,:],   lse[b,i,g] = ln sum_{s in seen(t)} exp(x_s);
 *   out = 0 and lse = -inf where nothing is seen.
 *   q          device [B,S,H,D] bf16   (H a multiple of H_kv)
 *   lengths    device [B] int32        NULL = table_pages * page_rows
 *   first      device [B] int32        NULL = 0
 *   n_win      >= 0; SI_ALL_ROWS: no window
 *   out        device [B,S,H,D] bf16;  lse device [B,S,H] f32 or NULL
 *   workspace  device, si_paged_workspace_bytes(B, S, H, H_kv, D) bytes: room for the parts of sequences that are split, whatever the lengths are.  The size
 *              knows neither the table's width nor n_win: a call whose table or window leaves every sequence few rows asks for as much, and uses 8 B bytes at most
 * fp32 products, statistics and sums: a logit is infinite where <q,K>, or that times scale * log2(e), passes fp32's range, and finite values give
 * finite results where the number of rows seen times the largest value is at most 2^117, as sums are divided by that of their weights at the end.  A
 * weight exp(x_s - reference) is rounded to bf16 once, as an operand of the second product; lse is made of the weights before that.  A head whose
 * query is not finite, or one of whose logits is NaN or +infinity, gets NaN in out and lse, and no other head does.  A logit of -infinity is a weight of
 * 0 (a finite query with no other logits gets out = 0 and lse = -inf); infinite or NaN values of a row that is seen make infinities or NaN of out where
 * they stand.  What rows hold
 * that a position does not see (behind the length, before the window, later positions' rows) never reaches its result, NaN and infinities included.
 * scale has to be finite, scale * log2(e) too (SI_ERR_INVALID_ARG).  The same call gives the same bits, and no bit of a head's
 * result depends on the queries of other heads or positions. */
size_t si_paged_workspace_bytes(int32_t B, int32_t S, int32_t H, int32_t H_kv, int32_t D);
si_status si_paged_attention(const void* q, const si_paged_cache* cache, int32_t S, int32_t H, const int32_t* lengths, const int32_t* first,
                             int32_t m, si_mask_mode mask_mode, int32_t n_win, float scale, void* out, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* STREAMINDEX_PAGES_H */
