/*
 * libelastic_cache -- several new tokens of a sequence at a time over paged caches: a prompt's chunk, drafted tokens, chunks beside single tokens.
 * The conventions, statuses and what a paged cache is are those of ec.h.
 */
#ifndef EC_TOKENS_H_
#define EC_TOKENS_H_

#include "ec.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Three calls: pages and slots for the tokens (once for all layers), then in every layer their queries and keys turned by their positions and stored, and
 * their attention.  Tokens are packed: those of sequence b are token_start[b] .. token_start[b+1] - 1 of T, sequence after sequence; tokens behind the
 * last sequence's are padding.
 */

/*
 * Pages for new rows, on the device: page table, a stack of free pages, and where every new token goes.  With L = len_b[b] the rows of sequence b that
 * stay (below 0: the place holds no sequence, and all its pages are given back), n = max(new_b[b], 0) its new tokens, h = held_b[b] the pages that it
 * holds, entries 0 .. h-1 of its row of the table:
 *   1. a sequence fits if L >= 0, its tokens end at or before T and ceil((L + n) / page) <= max_pages.  It wants ceil((L + n) / page) pages, one that
 *      does not fit ceil(L / page) and none beyond those it holds
 *   2. pages beyond what a sequence wants are given back: sequence after sequence, each from its last entry down, onto the stack; their entries become -1
 *   3. sequences take the pages that they miss from the top of the stack, in order; the first for which they are too few and all behind it that miss
 *      some get none
 *   4. start_b[b] = L and the table holds slots 0 .. L + n - 1 of a sequence that fits and has its pages.  Of all others start_b[b] = -1: the calls
 *      that take it as the rows before the step leave such a place out
 *   len_b,new_b     DEVICE [B] int32, read only
 *   seen_b          DEVICE [B] int32, tokens seen before the step; may be NULL, seen_after_b then too
 *   page_table      DEVICE [B,max_pages] int32, updated
 *   held_b          DEVICE [B] int32, updated (taken as 0 .. max_pages)
 *   free_pages      DEVICE [n_pages] int32, the stack; entries from n_free on keep what they hold
 *   n_free          DEVICE [1] int32, updated (taken as 0 .. n_pages)
 *   start_b         DEVICE [B] int32, written
 *   len_after_b     DEVICE [B] int32, written: L + n, L where start_b is -1, -1 without a sequence; may be len_b
 *   seen_after_b    DEVICE [B] int32, written: seen_b + n, seen_b where start_b is -1; may be seen_b
 *   token_start     DEVICE [B+1] int32, written: sums of n, of all sequences alike, T where they are larger
 *   rows            DEVICE [T] int64, written: a token's row of the pools, page id * page + row of the page; -1 for padding, for tokens of sequences
 *                   that start at -1 and where the table names no page; may be NULL
 *   pos             DEVICE [T] int32, written: seen_b[b] + i of the i-th token of b (L + i without seen_b), 0 where it has none; may be NULL
 * Requires 1 <= B <= 8192, 1 <= T <= 2^24; no two arrays may overlap but those named.  A table, stack or held_b that names a page twice
 * gives unspecified pages (nothing outside the arrays is touched).  Results are deterministic.
 */
int ec_paged_plan(const int32_t* len_b, const int32_t* new_b, const int32_t* seen_b, int32_t* page_table, int32_t* held_b, int32_t* free_pages,
                  int32_t* n_free, int B, int T, int page, int n_pages, int max_pages, int32_t* start_b, int32_t* len_after_b,
                  int32_t* seen_after_b, int32_t* token_start, int64_t* rows, int32_t* pos, void* stream);

/*
 * Rotary positions, and rows into pages.  With a = pos[t] * freq[i] (formed and brought below a turn in 64 bits) pair i of a query's or key's head, (x, y),
 * becomes mscale * (x cos a - y sin a, y cos a + x sin a); pair i is elements i and i + rot / 2 (pairing EC_ROTARY_HALVES) or 2 i and 2 i + 1
 * (EC_ROTARY_NEIGHBOURS), elements from rot on stay as they are.  Long contexts are a matter of freq and mscale.
 *   q               DEVICE [T,H,D] dt, tokens q_step elements apart (k, v likewise), so that parts of one projection's output can be given; read only
 *   k,v             DEVICE [T,Hkv,D] dt, read only
 *   pos             DEVICE [T] int32
 *   rows            DEVICE [T] int64, a row of the pools each (see ec_paged_plan); what lies outside the pools is no token: nothing is read or written for it
 *   freq            DEVICE [rot/2] float, radians per position
 *   q_out           DEVICE [T,H,D] dt, dense, written; must not overlap q, k or v (EC_EINVAL)
 *   k_pages,v_pages rows written: the turned key, the value as it is
 *   pos_pages       written: pos; may be NULL
 *   mass_pages      written: 0, what the frequency policy's rows start from; may be NULL
 * Requires rot even, 2 <= rot <= D, a finite mscale, steps of at least a token's elements, T <= 2^24, T * H <= 2^30.  q, k, v, q_out, the pools and the
 * steps lie on 16-byte boundaries (else EC_EUNSUPPORTED).  Two tokens of one row leave a mixture of them there.  Arithmetic is in fp32, rounded once.
 */
typedef enum { EC_ROTARY_HALVES = 0, EC_ROTARY_NEIGHBOURS = 1 } ec_rotary_pairing;
int ec_paged_rotary_store(const void* q, const void* k, const void* v, int64_t q_step, int64_t k_step, int64_t v_step, const int32_t* pos,
                          const int64_t* rows, const float* freq, float mscale, int rot, int pairing, int T, int H, int Hkv, int G, int D,
                          int page, int n_pages, int dt, void* q_out, void* k_pages, void* v_pages, int32_t* pos_pages, float* mass_pages,
                          void* stream);

/*
 * Attention of the new tokens over paged caches that hold their rows already.  For token i of sequence b, L = start_b[b]:
 *     out = softmax_j(scale * <q, k_j>) . v_j,   lse = log sum_j exp(scale * <q, k_j>)   over slots j = 0 .. L + i
 * of the query head's key/value head.  Slots behind the table's last and on no page weigh nothing.  A token that sees no row, or only scores of -inf,
 * gets zeros and an lse of -inf; so do all tokens of a place whose L is outside 0 .. max_pages * page - 1.  Rows of out and lse behind the last
 * sequence's tokens are left as they are.
 *   q,out           DEVICE [T,H,D] dt; out must not overlap q (EC_EINVAL)
 *   lse             DEVICE [T,H] float, written; may be NULL; must not overlap q or out (EC_EINVAL)
 *   start_b         DEVICE [B] int32, token_start DEVICE [B+1] int32 (taken as 0 .. T; what overlaps or falls is unspecified)
 *   ws              DEVICE scratch, ec_workspace_bytes(EC_FN_PAGED_CHUNK_STEP, B,H,T,D,dt), of one call at a time
 * Requires T <= 2^24, T * H <= 2^30.  Products are formed on the matrix cores with fp32 accumulation, sums and the softmax in fp32.  Where a sequence of bf16
 * brings more than 32 tokens times query heads of a key/value head, its weights enter the product with V rounded to bf16 (their sum does not); with
 * fewer, and in fp32, they enter with all 24 bits.  A weight below the range of normal fp32 numbers, 2^-126 of the largest, may count as 0, and an infinite V
 * with it gives NaN then.  An infinite or NaN row of V reaches the tokens that see it, and no others.  ws needs no contents.  Results are deterministic: a row's sum is formed in an order that depends on
 * the lengths of the whole batch and on T, not on time.
 */
int ec_paged_chunk_step(const void* q, const void* k_pages, const void* v_pages, const int32_t* page_table, const int32_t* start_b,
                        const int32_t* token_start, int B, int T, int H, int Hkv, int D, int page, int n_pages, int max_pages, float scale,
                        int dt, void* out, float* lse, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EC_TOKENS_H_ */
