/*
 * mds_cache.h -- the target model's key/value cache around the verification
 * of draft trees (part of libmds.so; return codes and mds_dtype are mds.h's).
 *
 * A step of multi-draft decoding on a batch of sequences is
 *
 *   mds_cache_reserve    room for the n = 1 + K * L tokens of a draft tree
 *   per model layer:
 *     mds_cache_append   their keys and values, quantised to 8 bits
 *     mds_cache_attend   attention of every tree node over the cache
 *   mds_verify           the target logits of the nodes against the drafts
 *   mds_cache_commit     the root and the accepted branch stay, packed; the
 *                        other tokens and the pages behind them go
 *
 * and mds_cache_fork / _truncate / _free share, shorten and drop sequences.
 *
 * Tree.  Node 0 is the root: the last emitted token, which is not in the
 * cache yet.  Node 1 + k * L + j is branch k's draft token j (depth j + 1).
 * Node i is held in slot len + i, len being the sequence's committed tokens.
 * It sees the committed tokens, the root, and its own branch up to itself.
 * Its position is len + depth.  K = 1 is a chain: one token (n = 1), or a
 * chunk of a prompt.
 *
 * Storage.  Keys and values are e4m3 numbers with a power-of-two scale for
 * every block of 16 tokens, head, and key or value.  The block quantiser Q
 * takes a = max|x| over the block's live tokens, the least integer e in
 * [-117, 119] with a <= 448 * 2^e, and stores e4m3(x / 2^e), rounded to the
 * nearest (ties to even); numbers above 448 * 2^119 (3.0e38) are stored as
 * that, so that every stored value is finite in 32 bits.  A power-of-two scale gives up none of e4m3's
 * relative precision, and a change of scale is a shift of exponents: exact
 * but for numbers that become subnormal (below 2^-14.8 of the block's
 * maximum).  A call that adds tokens to a block, or moves tokens into it,
 * applies Q to the values that all its live tokens stand for.  NaN is stored
 * as 0 and an infinity as the block's largest number, and MDS_ST_NONFINITE is
 * set: a masked token can therefore never reach another row's output.
 *
 * Pages.  A page holds page_tokens tokens of one sequence in every layer.  A
 * page that several sequences share is copied for the one that writes behind
 * it (mds_cache_reserve).  New pages are the lowest-numbered free ones, given
 * in the order of the call's list of sequences and their tokens: the state
 * depends on the calls alone, not on the order of threads.
 *
 * Everything is device-resident: lengths, page tables and the free pages are
 * read and written by the kernels, no call copies to the host (but
 * mds_cache_status), and a step can be captured in a CUDA graph.
 *
 * seqs lists the batch's sequences, ids in [0, max_seqs), no id twice in one
 * call (but in the src of mds_cache_fork).  An id below 0 marks an unused place of the batch: nothing is done
 * for it, and its outputs are zeros.  An id of max_seqs or more is treated
 * the same and sets MDS_ST_BADSEQ.
 *
 * counts (NULL: n for all) gives the live tokens of each sequence of the
 * call, clamped to [0, n]; rows of tokens beyond it are not read, and their
 * outputs are zeros.
 *
 * Threading: a cache may be used from one host thread at a time and its calls
 * must not overlap on the GPU (they share pages, counters and workspace).
 * All device work is issued on the caller's stream; only mds_cache_status
 * synchronises.
 */
#ifndef MDS_CACHE_H
#define MDS_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "mds.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Status bits of a cache, beside MDS_ST_NONFINITE (a key or value was NaN or
 * infinite), MDS_ST_BADTOKEN (emitted tokens of no branch) and
 * MDS_ST_TIMEOUT. */
#define MDS_ST_NOPAGES 128u /* too few free pages, or a page table too short: the
                               sequence was given none, and tokens that were
                               not reserved before are not stored              */
#define MDS_ST_BADSEQ 256u  /* a sequence id of max_seqs or more; a fork onto a
                               sequence that holds pages; tokens appended,
                               attended to or committed that were not reserved */

#define MDS_CACHE_BLOCK 16        /* tokens per scale                         */
#define MDS_CACHE_MAX_BATCH 1024  /* sequences in one call                    */
#define MDS_CACHE_MAX_TOKENS (1 << 20) /* n of one call, and tokens a sequence may hold
                                     (page_tokens * max_pages)                */
#define MDS_CACHE_MAX_NODES 16384 /* nodes of one attend call                 */
#define MDS_CACHE_MAX_GROUP 64    /* query heads per key/value head           */

typedef struct mds_cache mds_cache;

typedef struct {
  int layers;      /* 1..1024                                                  */
  int pages;       /* pages of the pool, 1..2^24                               */
  int page_tokens; /* tokens per page: 16, 32, 64 or 128                       */
  int kv_heads;    /* 1..1024                                                  */
  int head_dim;    /* 64 or 128                                                */
  int max_seqs;    /* sequences the cache may hold, 1..2^20                    */
  int max_pages;   /* pages one sequence may hold, 1..2^16                     */
  mds_dtype dtype; /* type of keys, values, queries and outputs                */
} mds_cache_config;

/* Bytes of device memory a cache of this configuration needs (0: the
 * configuration is outside the limits above). */
size_t mds_cache_bytes(const mds_cache_config* cfg);

/* A cache on CUDA device `device` in `memory`: mds_cache_bytes(cfg) bytes of
 * device memory aligned to 1024, owned by the caller, who keeps them for the
 * cache's lifetime and does not write to them.  The memory is cleared on
 * `stream`; every sequence is empty and every page free.  Nothing is
 * allocated on the device. */
int mds_cache_create(mds_cache** out, const mds_cache_config* cfg, int device, void* memory, void* stream);

/* Device addresses inside the cache's memory, for reading: *lens is
 * [max_seqs] int32, the committed tokens; *table is [max_seqs][max_pages]
 * int32, the page ids of each sequence, -1 behind them.  Either may be NULL. */
int mds_cache_state(const mds_cache* cache, const int32_t** lens, const int32_t** table);

/* Make room for counts[b] (n) tokens behind the committed ones of every
 * sequence: pages for them, and pages of its own in place of shared ones
 * from the page that holds slot len on (their tokens in front of slot
 * len + counts[b] are copied).  A sequence that the free pages do not reach,
 * counting those before it in the list, or whose page table is too short,
 * gets none (MDS_ST_NOPAGES).
 * Only reserved slots are stored to, attended to and committed.  They stay
 * reserved until commit, truncate or free gives back their page (truncate and
 * free: any slot behind the length).  A fork has what its source has reserved.
 * Where pages are shared, a call that copies any ends what is reserved at
 * len + counts[b], and one that gives none ends it in front of the first. */
int mds_cache_reserve(mds_cache* cache, const int32_t* seqs, const int32_t* counts, int n, int B, void* stream);

/* Store keys and values of layer `layer` in the slots len .. len + counts[b]
 * of each sequence, as far as they are reserved (MDS_ST_BADSEQ where not, or
 * where their page is shared).  k and v are dtype: the element of
 * sequence b of the list, token i, head h and dimension d is at
 * b * strides[0] + i * strides[1] + h * strides[2] + d, strides in elements,
 * multiples of 16 bytes, the bases aligned to 16 bytes (MDS_EINVAL
 * otherwise). */
int mds_cache_append(mds_cache* cache, int layer, const int32_t* seqs, const int32_t* counts, const void* k,
                     const int64_t* k_strides, const void* v, const int64_t* v_strides, int n, int B, void* stream);

/* Attention of the n = 1 + branches * L nodes of each sequence's tree over
 * layer `layer` of the cache (their own keys and values appended before):
 * out[b][i][h] = sum_t softmax_t(scale * q[b][i][h] . k_t) v_t over the slots
 * t that node i sees, k and v those of head h / (q_heads / kv_heads).
 * With window > 0 a key at position p is seen from position x only if
 * p < sinks or p > x - window.  q has strides like k above; out is
 * [B][n][q_heads][head_dim] dtype, contiguous, aligned to 16 bytes.
 * q_heads is kv_heads * g, 1 <= g <= MDS_CACHE_MAX_GROUP.  Products of
 * queries with keys are exact for 16-bit queries (but for elements below 2^-28
 * of their row's maximum) and taken with 22 bits of a 32-bit query; sums and
 * softmax statistics are 32-bit; the softmax weights
 * are rounded to the query's precision before they meet the values, and the
 * normaliser sums the rounded weights.  Weights are held relative to a
 * reference that the largest may pass by 2^48 or miss by 2^20, so sums over
 * values beyond about 2^60 can overflow and values below about 2^-100 lose
 * bits.  Scores beyond 2^127 overflow. */
int mds_cache_attend(mds_cache* cache, int layer, const int32_t* seqs, const int32_t* counts, const void* q,
                     const int64_t* q_strides, void* out, int q_heads, int n, int branches, int window, int sinks,
                     float scale, int B, void* stream);

/* Keep, of the 1 + K * L tokens behind the committed ones, the root and the
 * first accept_len[b] tokens of one branch (accept_len clamped to [-1, L];
 * -1 keeps nothing): they are packed behind the committed tokens in every
 * layer, len grows by 1 + accept_len[b], and the pages behind it are given
 * back.  The branch is the lowest one whose first accept_len[b] draft_tokens
 * ([B][K][L] int32) equal out_tokens ([B][L+1] int32), the arrays that
 * mds_verify read and wrote; both NULL: branch 0.  Tokens of no branch keep
 * branch 0 (MDS_ST_BADTOKEN); tokens that were not reserved, or would be
 * moved into a page that is shared when the call begins, are not kept
 * (MDS_ST_BADSEQ), whichever of the call's sequences share it and keep what. */
int mds_cache_commit(mds_cache* cache, const int32_t* seqs, const int32_t* accept_len, const int32_t* draft_tokens,
                     const int32_t* out_tokens, int K, int L, int B, void* stream);

/* Let dst[b], which must be empty, share all of src[b]'s pages, tokens
 * behind the committed ones included.  src may name a sequence several times;
 * no id of dst may be in src. */
int mds_cache_fork(mds_cache* cache, const int32_t* src, const int32_t* dst, int B, void* stream);

/* Shorten each sequence to lens[b] tokens (to its length where it has fewer)
 * and give back what is behind: pages, and the slots that were reserved. */
int mds_cache_truncate(mds_cache* cache, const int32_t* seqs, const int32_t* lens, int B, void* stream);

/* Empty the sequences and give back their pages. */
int mds_cache_free(mds_cache* cache, const int32_t* seqs, int B, void* stream);

/* The values of n tokens from slot start[b] (NULL: 0) on, of layer `layer`
 * (-1: of all): k and v are [B][n][kv_heads][head_dim] dtype ([layers] in
 * front for layer -1), contiguous, aligned to 16 bytes.  Tokens beyond
 * counts[b] or what the sequence holds are zeros. */
int mds_cache_read(mds_cache* cache, int layer, const int32_t* seqs, const int32_t* start, const int32_t* counts,
                   void* k, void* v, int n, int B, void* stream);

/* Synchronise the device, read and clear the status word: its MDS_ST_* bits
 * (>= 0) or a negative code; *msg (if not NULL) receives a static description
 * of the highest set bit. */
int mds_cache_status(mds_cache* cache, const char** msg);

/* Free the handle (the memory is the caller's). */
void mds_cache_destroy(mds_cache* cache);

#ifdef __cplusplus
}
#endif

#endif /* MDS_CACHE_H */
