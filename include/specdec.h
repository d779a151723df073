/*
 * specdec.h -- C ABI of the B200 (sm_100a) SpecDec draft -> verify -> commit library.
 *
 * The library implements the hot path of Speculative Decoding for seq2seq
 * generation: the Spec-Drafter's parallel pass over k [MASK] queries
 * (Section 3.1.3, inference equation), the verification pass in which the
 * autoregressive encoder-decoder Transformer scores all k drafts of every
 * sequence at once (Section 2, Eq. 1-3), the Spec-Verification acceptance rule
 * (Section 3.2, Eq. 7-9) and the loop that repeats draft -> verify -> commit
 * until [EOS] (Section 2, last sentence; Appendix "Case Study").
 *
 * Conventions
 *   - Pointers named d_* are DEVICE pointers, h_* are HOST pointers.  The caller
 *     owns every buffer it passes; the library owns its arena (repacked weights,
 *     paged KV cache, workspaces) from specdec_create to specdec_destroy.
 *   - `stream` is a cudaStream_t passed as void*.  Calls are asynchronous on it
 *     unless stated otherwise; buffers must stay valid until the stream reaches
 *     the end of the call.
 *   - Every function returns SPECDEC_OK (0) or a negative error code; a message
 *     is kept in the handle (specdec_last_error).  Nothing throws, exits or prints.
 *   - One decoding session per handle at a time: specdec_encode starts it.
 *   - Token ids are int32.  Row-major everywhere.
 *   - There is no CPU fallback: without a CUDA device every compute call fails
 *     with SPECDEC_ERR_CUDA.
 */
#ifndef SPECDEC_H
#define SPECDEC_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPECDEC_OK                 0
#define SPECDEC_ERR_INVALID_ARG   -1
#define SPECDEC_ERR_SHAPE         -2   /* weight manifest does not match the dims        */
#define SPECDEC_ERR_CAPACITY      -3   /* B / S / k / max_tgt beyond create-time limits  */
#define SPECDEC_ERR_NOT_ENCODED   -4
#define SPECDEC_ERR_CUDA          -5
#define SPECDEC_ERR_TIMEOUT       -6   /* a bounded device-side wait gave up.  specdec_generate reports it itself;
                                          the asynchronous step calls report it one call late: specdec_commit and
                                          specdec_get_output fetch the device's error word, and the next call on the
                                          handle that finds it set returns this code and clears it.  The handle stays
                                          usable: start over with specdec_encode                                      */
#define SPECDEC_ERR_UNSUPPORTED   -7
#define SPECDEC_ERR_CORRUPT       -8   /* an integrity check (option "debug_checks") found a damaged red zone behind an
                                          arena block or a non-finite activation; specdec_last_error names it        */

#define SPECDEC_DTYPE_F32   0
#define SPECDEC_DTYPE_BF16  1
#define SPECDEC_DTYPE_F16   2      /* operators on the caller's tensors only: handles take the first two */
#define SPECDEC_DTYPE_FP4   3      /* specdec_packed_cache only */

#define SPECDEC_ACT_RELU    0
#define SPECDEC_ACT_GELU    1

typedef struct specdec_handle specdec_handle;

/* One encoder-decoder Transformer (pre-LN, shared embedding table; position tables are weights, so
 * sinusoidal and learned positions are both just data). */
typedef struct {
    int d_model, n_heads, d_ffn, vocab;
    int enc_layers, dec_layers;
    int max_pos;                       /* rows of the position tables */
} specdec_model_dims;

typedef struct {
    specdec_model_dims verifier, drafter;
    int k_max;                         /* largest draft block                                  */
    int max_batch, max_src, max_tgt;   /* capacity limits of a session                         */
    int page_tokens;                   /* tokens per KV-cache page (power of two)              */
    int pad_id, bos_id, eos_id, mask_id;
    int compute_dtype;                 /* SPECDEC_DTYPE_F32: fp32 operands (SIMT kernels);
                                          SPECDEC_DTYPE_BF16: bf16 operands, fp32 accumulation
                                          (tcgen05 tensor-core GEMMs)                          */
    int ffn_activation;                /* SPECDEC_ACT_RELU (Transformer-base, Section 4.1) or SPECDEC_ACT_GELU:
                                          the exact GELU x * Phi(x), for the BART-base-shaped pair of the
                                          summarisation experiment (Section 5.2); both models use it    */
} specdec_config;

/* One named weight.  `d_ptr` is a DEVICE pointer to fp32 data, row-major.
 * Names, per model prefix "verifier." / "drafter." (y = x W^T + b, W is [out,in]):
 *   embed [V,d]   pos_enc, pos_dec [max_pos,d]
 *   enc.{l}.ln1.{g,b}  enc.{l}.self.{q,k,v,o}.{w,b}  enc.{l}.ln2.{g,b}
 *   enc.{l}.ffn.{w1,b1,w2,b2}   enc.ln_f.{g,b}
 *   dec.{l}.ln1  dec.{l}.self.*  dec.{l}.ln_cross.{g,b}  dec.{l}.cross.{q,k,v,o}.{w,b}
 *   dec.{l}.ln2  dec.{l}.ffn.*   dec.ln_f.{g,b}                                        */
typedef struct {
    const char* name;
    const void* d_ptr;
    int         dtype;                 /* SPECDEC_DTYPE_F32 only */
    int         ndim;
    long long   shape[4];
} specdec_tensor;

/* Counters of specdec_generate.  Tok. of the paper's latency model (Eq. 4) is
 * accepted / seq_iterations (or emitted / seq_iterations counting the
 * bifurcation token); t_d, t_v are ms_draft, ms_verify per iteration. */
typedef struct {
    long long iterations;              /* draft->verify->commit rounds that ran               */
    long long seq_iterations;          /* sum over rounds of sequences still decoding         */
    long long drafted, accepted, emitted;
    double    ms_encode, ms_draft, ms_verify, ms_commit, ms_total;   /* draft / verify / commit: option "stats_timing" only */
    int       status;
} specdec_stats;

/* Builds a handle: validates the manifest against the dims, allocates the arena
 * (the only device allocation the library makes), copies and repacks the weights
 * (bf16 for SPECDEC_DTYPE_BF16).  Synchronises `stream` before returning, so the
 * caller may free its weight buffers afterwards.  *out is NULL on failure; the
 * reason is then available from specdec_last_error(NULL). */
int specdec_create(const specdec_config* cfg, const specdec_tensor* weights, int n_weights,
                   void* stream, specdec_handle** out);
int specdec_destroy(specdec_handle* h);

/* Starts a session: runs both encoders over the right-padded sources and caches
 * the per-decoder-layer cross-attention K/V of both models ("the encoder is
 * forwarded only once", Section 3.1.2).  All sequences start with no committed
 * target token.  d_src [B,S_max] int32, d_src_len [B] (1..S_max), d_max_tgt [B]
 * (0..max_tgt; NULL = max_tgt for all). */
int specdec_encode(specdec_handle* h, const int32_t* d_src, const int32_t* d_src_len,
                   const int32_t* d_max_tgt, int B, int S_max, void* stream);

/* Spec-Drafter pass (Section 3.1.3): for every unfinished sequence, the decoder
 * runs without a causal mask over [BOS, committed tokens, MASK x k] and the
 * argmax (lowest id on ties) at each mask row becomes a draft.
 * d_draft [B,k] int32 out; rows of finished sequences are left untouched. */
int specdec_draft(specdec_handle* h, int k, int32_t* d_draft, void* stream);

/* Verification pass (Section 2 Eq. 1-3, Section 3.2 Eq. 7-9): the verifier
 * decoder scores the block [last committed token, k drafts] causally over the
 * paged KV cache; draft i is accepted iff all earlier ones are, fewer than
 * `beta` vocabulary entries score strictly higher (Eq. 7) and top-1 score minus
 * its score <= tau (Eq. 8).  d_accepted [B] receives the accepted length in
 * [0,k]; d_bif [B] the verifier's top-1 token on the row after the accepted
 * prefix (the replacement at the bifurcation, or the bonus token when a = k).
 * Does not commit.  beta >= 1, tau >= 0, 0 <= k <= k_max (k = 0: one row, the next greedy token). */
int specdec_verify(specdec_handle* h, const int32_t* d_draft, int k, int beta, float tau,
                   int32_t* d_accepted, int32_t* d_bif, void* stream);

/* Commit / rollback (Eq. 3): appends drafts[0..keep) and `next` to each
 * unfinished sequence, cuts after the first [EOS] and at the sequence's max
 * target length, marks finished sequences, and keeps only the KV-cache rows of
 * the kept prefix.  d_keep / d_next [B] may be NULL: the results of the last
 * specdec_verify are used.  Must follow a specdec_verify (it reuses its block). */
int specdec_commit(specdec_handle* h, const int32_t* d_keep, const int32_t* d_next, void* stream);

/* encode + (draft -> verify -> commit) until every sequence is finished.
 * d_out [B,out_stride] int32 receives the generated ids (without BOS),
 * d_out_len [B] their count.  h_stats may be NULL.  Synchronises `stream`.
 * k = 0 is plain greedy autoregressive decoding with the verifier alone (no drafter pass, one-row
 * verify blocks): the baseline SpecDec is compared with. */
int specdec_generate(specdec_handle* h, const int32_t* d_src, const int32_t* d_src_len,
                     const int32_t* d_max_tgt, int B, int S_max, int k, int beta, float tau,
                     int32_t* d_out, int out_stride, int32_t* d_out_len,
                     specdec_stats* h_stats, void* stream);

/* Same, with HOST buffers: the copies host->device (sources) and device->host
 * (ids, lengths) are part of the call.  Pinned host memory avoids a staging copy. */
int specdec_generate_host(specdec_handle* h, const int32_t* h_src, const int32_t* h_src_len,
                          const int32_t* h_max_tgt, int B, int S_max, int k, int beta, float tau,
                          int32_t* h_out, int out_stride, int32_t* h_out_len,
                          specdec_stats* h_stats, void* stream);

/* Current session state: committed ids [B,out_stride], lengths [B], finished flags [B]
 * (any pointer may be NULL). */
int specdec_get_output(specdec_handle* h, int32_t* d_out, int out_stride, int32_t* d_out_len,
                       int32_t* d_finished, void* stream);

/* The acceptance rule alone (Eq. 7-9) on caller-provided fp32 logits
 * d_logits [B,k+1,V]: same outputs as specdec_verify.  No handle, no workspace. */
int specdec_accept_scan(const float* d_logits, const int32_t* d_draft, int B, int k, int V,
                        int beta, float tau, int32_t* d_accepted, int32_t* d_bif, void* stream);

/* The same acceptance rule for callers that must not allocate device memory -- the paper has no
 * counterpart; this exists for embedding the rule in programs where the device allocator is off
 * limits: a serving process whose memory pool already owns all of HBM (so a later cudaMalloc
 * fails), or a latency-critical loop that cannot afford the device-wide synchronisation an
 * allocation or free implies.  Inputs and outputs are the caller's, exactly as for
 * specdec_accept_scan (d_logits [B,k+1,V] fp32, d_draft [B,k]; d_accepted, d_bif [B]).
 * Limits: B*(k+1) <= 4096, V <= 65536 and k+1 <= 2048; beyond them the call returns
 * SPECDEC_ERR_CAPACITY and launches nothing.  The call makes no cudaMalloc / cudaFree and uses
 * no allocating library routine; its intermediate statistics live in shared memory, so calls on
 * different streams or host threads do not disturb one another. */
int specdec_accept_scan_static(const float* d_logits, const int32_t* d_draft, int B, int k, int V,
                               int beta, float tau, int32_t* d_accepted, int32_t* d_bif, void* stream);

/* ---------------------------------------------------------------------------------------------------------------
 * Tree speculation on the caller's tensors.  A chain of drafts is verified by a handle, greedily, over the handle's
 * cache.  These operators serve a program that drafts several continuations of every sequence (a tree), samples
 * instead of taking the top token, and keeps the paged K/V cache in its own memory.  One decoding step is
 *     cache_reserve, (cache_append, tree_attention) in every layer, sample, tree_accept, cache_compact;
 * cache_fork and cache_release begin and end branches.  No handle; nothing is allocated; failures are reported as by
 * every other call (message: specdec_last_error(NULL)).  The device that holds a call's memory, and to which its stream
 * belongs, has to be the current one.  Operators on one cache are ordered by the caller (one stream, or events).
 *
 * A tree is its nodes' parents: node 0 is the root (the last committed token), node i > 0 hangs off parents[i] in
 * [0, i).  Any other value is no parent: the node begins a tree of its own, which a walk from node 0 never reaches.
 *
 * The cache: page p holds page_tokens token slots of every layer; a slot's row of n_heads x head_dim elements is found
 * by the strides (elements; head_dim is contiguous; stride_side leads from a layer's keys to its values), so pages of
 * [token, head] and of [head, token] order both do.  d_kv and all strides are multiples of 16 bytes (the stride of a
 * dimension of 1, here and of every other tensor, does not matter).  Slot t of
 * sequence s is slot t % page_tokens of page d_table[s * max_pages + t / page_tokens].  d_length[s] tokens are
 * committed, d_held[s] pages are in the sequence's table (entries behind them are -1), d_refs[p] sequences hold page p
 * (0: free).  Pages are given out lowest number first, so what a call does depends on its arguments alone.  A new cache has
 * d_table = -1 and everything else 0.  d_status[0] gathers SPECDEC_CACHE_* bits until the caller clears it; d_scratch holds
 * specdec_cache_scratch() int32 values, zero at first, and belongs to the calls in between.  Tokens are only ever
 * written to pages that one sequence holds: branches share full pages and copy the last, partly filled one. */
#define SPECDEC_CACHE_NO_PAGES    1   /* not enough free pages: the call changed nothing                              */
#define SPECDEC_CACHE_ROW_FULL    2   /* a sequence would hold more than max_pages: the call changed nothing           */
#define SPECDEC_CACHE_BAD_INDEX   4   /* a sequence number or a path out of range: that entry was skipped              */
#define SPECDEC_CACHE_UNRESERVED  8   /* a token's slot is in no page of the sequence's own: the token (compact: the
                                         sequence) was skipped                                                         */
#define SPECDEC_CACHE_TIMEOUT    16   /* tree_attention: a bounded wait inside a kernel gave up; its output is not valid */
typedef struct {
    void*     d_kv;
    int       dtype;                       /* SPECDEC_DTYPE_*                                                          */
    int       n_layers, n_heads, head_dim; /* K/V heads                                                                */
    int       n_pages, page_tokens;        /* page_tokens: a power of two                                              */
    int       n_seqs, max_pages;
    long long stride_layer, stride_side, stride_page, stride_token, stride_head;
    int32_t  *d_table, *d_length, *d_held, *d_refs, *d_status, *d_scratch;
} specdec_cache;

/* int32 values of d_scratch; negative on a bad argument. */
long long specdec_cache_scratch(int n_seqs, int max_pages, int n_pages);

/* The calls below take n sequence numbers d_seqs [n], all different.
 * reserve: pages for n_tokens slots behind the committed ones (those already held count).
 * append: writes rows t < (d_count ? d_count[i] : T) of d_k, d_v [n_layers, n, T, n_heads, head_dim] (head_dim contiguous, strides and
 *   addresses multiples of 16 bytes) of layers layer .. layer + n_layers - 1 into slots d_length + t.  Lengths stay.
 * compact: slots d_length + d_path[i, 0 .. d_n_path[i]) move to d_length, d_length + 1, ... in every layer; the length grows by d_n_path[i], and
 *   pages behind it are given back.  A path rises strictly (as the paths of specdec_tree_accept do); a sequence
 *   whose path does not is skipped (BAD_INDEX).
 * release: gives a sequence's pages back; its length is 0.
 * fork: sequence d_dst[i] becomes a copy of d_src[i] as that was before the call (so a permutation reorders beams), its old pages are
 *   given back.  Full pages are shared, the last, partly filled one is copied.  d_dst all different; a pair of equal numbers does nothing.
 * reorder: the n sequences are beams, in groups of `beams` that follow one another.  Sequence i of a group becomes what sequence d_parents[i] (0 .. beams - 1; -1: none, it
 *   is released) of the group was before the call.  Full pages are shared; the last, partly filled one goes on with one child (the parent itself if it is one, else the first) and is
 *   copied for the others, so that a permutation moves no data.  d_seqs all different, over all groups.  Pages that nobody holds any more are free, for the copies of this call too; they are given to the entries
 *   that copy in their order.  Pages behind the committed tokens are given back.  Any other parent, or one whose sequence number is out of range: the entry is its own (BAD_INDEX). */
int specdec_cache_reserve(const specdec_cache* c, const int32_t* d_seqs, int n, int n_tokens, void* stream);
int specdec_cache_append(const specdec_cache* c, const int32_t* d_seqs, int n, int layer, int n_layers, const void* d_k, const void* d_v, int T,
                         long long stride_layer, long long stride_seq, long long stride_token, long long stride_head,
                         const int32_t* d_count, void* stream);
int specdec_cache_compact(const specdec_cache* c, const int32_t* d_seqs, int n, const int32_t* d_path, int path_stride,
                          const int32_t* d_n_path, void* stream);
int specdec_cache_release(const specdec_cache* c, const int32_t* d_seqs, int n, void* stream);
int specdec_cache_fork(const specdec_cache* c, const int32_t* d_src, const int32_t* d_dst, int n, void* stream);
int specdec_cache_reorder(const specdec_cache* c, const int32_t* d_seqs, const int32_t* d_parents, int n, int beams, void* stream);

/* Trees of up to 1024 nodes.  d_n_nodes [B] (or NULL: T each) cuts a tree short.
 * ancestors: bit j of d_mask [B, T, ceil(T / 32)] row i is set iff node j is node i or one of its ancestors; d_depth [B, T] is the
 *   number of ancestors (-1 behind the last node, whose mask is 0).  Either output may be NULL.
 * accept: the walk from the root along the sampled tokens: from node i on to its first child whose token is d_sampled[i].  d_path [B, T]
 *   receives the nodes passed (the root first; -1 behind), d_n_path [B] their number, d_emitted [B, T] the sampled token of each (-1
 *   behind): the accepted drafts and, last, the token that no child had.  With tokens sampled from the verifier this emits what sampling
 *   token by token would.  A tree of no nodes has no path. */
int specdec_tree_ancestors(const int32_t* d_parents, const int32_t* d_n_nodes, int B, int T, uint32_t* d_mask, int32_t* d_depth, void* stream);
int specdec_tree_accept(const int32_t* d_parents, const int32_t* d_tokens, const int32_t* d_sampled, const int32_t* d_n_nodes, int B, int T,
                        int32_t* d_path, int32_t* d_n_path, int32_t* d_emitted, void* stream);

/* Attention of tree nodes over the cache: query t of batch row b sees the d_length committed tokens of sequence s = d_seqs[b] and the nodes
 * j < n_nodes (their keys and values are in slots d_length + j) whose bit is set in d_mask[b, t]:
 *     out[b, t, h] = sum_j p_j v_j,   p = softmax(scale q . k_j) over what it sees,   K/V head h / (n_q_heads / n_heads).
 * A query that sees nothing, and every query t >= n_nodes, gives zeros.  What is in slots that no query of the row may see (behind the
 * nodes, or masked for all) never matters.  T = 1 with a mask of 1 is the decoding of single tokens; nodes may attend to later ones. */
typedef struct {
    const void *d_q;                       /* [B, T, n_q_heads, head_dim] of the cache's type, head_dim contiguous       */
    void       *d_out;                     /* the same shape                                                             */
    long long   q_stride_b, q_stride_t, q_stride_h, out_stride_b, out_stride_t, out_stride_h;     /* elements            */
    int         B, T, n_q_heads, layer;
    const int32_t  *d_seqs;                /* [B]                                                                        */
    const uint32_t *d_mask; long long mask_stride_b;      /* [B, T, ceil(T / 32)]; stride 0: one tree for all            */
    const int32_t  *d_n_nodes;             /* [B] or NULL: T                                                             */
    int         max_length;                /* no d_length of the batch is larger (0: unknown, max_pages * page_tokens)  */
    float       scale;
    void       *d_workspace; long long workspace_bytes;   /* see below                                                   */
} specdec_tree_attention_args;
/* Bytes of workspace (0: none) that spread a call of these sizes over the GPU; 16-byte aligned, no state between calls.  max_length: what the call
 * takes it to be (its own, or max_pages * page_tokens if that is smaller or its own is 0), or 0 for as much as any length needs.  With less, a call
 * returns SPECDEC_ERR_CAPACITY.  head_dim: multiples of 8 up to 128. */
long long specdec_tree_attention_workspace(int B, int T, int n_q_heads, int n_kv_heads, int head_dim, int dtype, int page_tokens, int max_length);
int specdec_tree_attention(const specdec_cache* c, const specdec_tree_attention_args* a, void* stream);

/* A cache in 4 bits.  Sixteen channels of a token and head share a scale s, an 8-bit float (e4m3: 4 bits of exponent, 3 of fraction); a channel is a code of 0, 0.5, 1, 1.5, 2, 3, 4, 6 or
 * their negatives (e2m1; number 0 .. 7, + 8 for the sign), and stands for unit * s * code.  unit: d_unit [n_layers, 2, n_heads] fp32, positive and finite, or NULL: 1.  What is
 * written is, with x' = x / unit in fp32, s = the scale nearest to max |x'| / 6 (at most 448), code = the one nearest to x' / s, halfway the even number (beyond 6: 6; s = 0: 0).  A NaN makes its
 * block NaN.
 *   codes:    a specdec_cache of dtype SPECDEC_DTYPE_FP4 whose strides count bytes: channel 2 i of a token and head is in the low half of byte i of head_dim / 2; the tokens of a page
 *             and head follow one another (stride_token does not matter).  head_dim is 64 or 128, page_tokens a power of two from 16 on.
 *   d_scales: head_dim / 16 bytes a token and head, tokens of a page and head behind one another, with strides of their own (bytes).
 * Addresses and strides of both are multiples of 16 bytes.  Everything else, and the calls of the same names, are as above; they move codes and scales as they are.
 * append: the first d_some[i] (NULL: all T) tokens of sequence i, as above, of fp32, bf16 or fp16.  read: the values of tokens d_some[i] + t (NULL: d_length + t, the block behind the
 *   committed tokens), rounded to dtype once; zeros where the sequence has no page.  It takes sequences more than once. */
typedef struct {
    specdec_cache codes;
    void*         d_scales;
    long long     scale_stride_layer, scale_stride_side, scale_stride_page, scale_stride_head;
    const float*  d_unit;
} specdec_packed_cache;
int specdec_packed_cache_reserve(const specdec_packed_cache* c, const int32_t* d_seqs, int n, int n_tokens, void* stream);
typedef struct {                           /* tokens of n sequences, append's and read's                                 */
    const int32_t *d_seqs;                 /* [n]                                                                         */
    void          *d_k, *d_v;              /* [n_layers, n, T, n_heads, head_dim] of dtype; append only reads them        */
    const int32_t *d_some;                 /* [n] or NULL: append's counts (T), read's first tokens (d_length)            */
    long long      stride_layer, stride_seq, stride_token, stride_head;                           /* elements            */
    int            n, layer, n_layers, dtype, T;
} specdec_packed_tokens;
int specdec_packed_cache_append(const specdec_packed_cache* c, const specdec_packed_tokens* t, void* stream);
int specdec_packed_cache_read(const specdec_packed_cache* c, const specdec_packed_tokens* t, void* stream);
int specdec_packed_cache_compact(const specdec_packed_cache* c, const int32_t* d_seqs, int n, const int32_t* d_path, int path_stride, const int32_t* d_n_path, void* stream);
int specdec_packed_cache_release(const specdec_packed_cache* c, const int32_t* d_seqs, int n, void* stream);
int specdec_packed_cache_fork(const specdec_packed_cache* c, const int32_t* d_src, const int32_t* d_dst, int n, void* stream);
int specdec_packed_cache_reorder(const specdec_packed_cache* c, const int32_t* d_seqs, const int32_t* d_parents, int n, int beams, void* stream);
/* tree_attention over it: q and out are of `dtype` (fp32, bf16, fp16); the rest as there.  Products with the exact values, scores and sums in fp32; bf16 and fp32 queries are taken with a row's
 * largest number moved below 2^15 by a power of two, as fp16 (fp32: two of them, 22 bits), probabilities as fp16 (fp32: two).  With p the weights and S the largest sum of scale |q k| of the query's scores, an
 * output is off by at most (2^-10 + 1e-5) sum p |v| (fp32: 2^-21 in the place of 2^-10) + 2^-32 max |v| for each key, its own rounding, and what scores that are off by 2^-16 S make of it.  Scores may be of
 * any finite size. */
long long specdec_packed_attention_workspace(int B, int T, int n_q_heads, int n_kv_heads, int head_dim, int dtype, int page_tokens, int max_length);
int specdec_packed_attention(const specdec_packed_cache* c, const specdec_tree_attention_args* a, int dtype, void* stream);

/* One token per row of d_logits [rows, V] (row r at r * stride; V contiguous) from a given uniform random number in [0, 1).
 * With l = fp32 logits (NaN: never taken) and m their maximum, w_i = floor(2^40 exp((l_i - m) / T)) 2^-40: weights are whole numbers of
 * units, so that their sums are exact, and a token is the same however the work is split.
 *   top_k  > 0: the k largest (ties: lower index first) stay;
 *   top_p  < 1: of those, in that order, entry i stays if the weight ahead of it is below top_p times their total;
 *   min_p  > 0: entries with exp((l_i - m) / T) >= min_p stay;     the largest always stays (top_p, min_p NaN: off).
 *   token = the first index at which the running sum of the kept weights exceeds floor(uniform * total).
 * temperature <= 0 (or NaN) takes the largest entry (lowest index).  d_logprob (or NULL) = log of the token's share of the kept weights.  A row
 * of only -inf and NaN gives token -1, log probability -inf.
 * d_temperature, d_top_k, d_top_p, d_min_p (each or NULL: 1, 0, 1, 0) hold one entry for each rows_per_param rows. */
int specdec_sample(const void* d_logits, int dtype, long long stride, int rows, int V, const float* d_uniform,
                   const float* d_temperature, const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, int rows_per_param,
                   int32_t* d_token, float* d_logprob, void* stream);

/* Beam search: the n best continuations of each sentence's K beams.  Row (b, k) of d_logits [B, K, V] (row b * K + k at stride times that; V contiguous; fp32, bf16, fp16; NaN: never taken) belongs to a
 * beam of score d_scores [B, K] (-inf or NaN: none; its row is not read).  With l = a row's logits, log p_v = l_v - ln sum_w exp(l_w) (of infinite logits each has an equal share, the others
 * none).  Candidates are (k, v) with score s = d_scores[b, k] + log p_v and rank s * d_norm[b, k] (NULL: s), and for a beam with d_finished[b, k] != 0 only (k, end_token) with
 * s = d_scores[b, k].  The n of largest rank come out, best first: d_out_scores (s), d_out_parent (k), d_out_token (v) [B, n]; where there are fewer with a rank above
 * -inf, -inf, -1 and -1 follow.  Order: rank; of ranks alike the lower beam; of one beam the larger logit, then the lower token.  What is taken is what exact sums would give: sums are fp32
 * unless ranks of different beams lie within some 2^-19 of one another, then 64 bits.  d_norm is a length penalty's factor (positive, finite); scores and ranks are 64 bits inside.
 * K and n: at most 64, V 2^20, B * K 65535.  The workspace (8-byte aligned, no state between calls) has specdec_beam_select_workspace() bytes. */
long long specdec_beam_select_workspace(int B, int K, int V, int n, int dtype);
typedef struct {
    const void          *d_logits;         /* [B, K, V]; `stride` elements between rows                                  */
    const float         *d_scores;         /* [B, K]                                                                     */
    const unsigned char *d_finished;       /* [B, K] or NULL: none                                                       */
    const float         *d_norm;           /* [B, K] or NULL: 1                                                          */
    float               *d_out_scores;     /* [B, n]                                                                     */
    int32_t             *d_out_parent, *d_out_token;
    void                *d_workspace; long long workspace_bytes, stride;
    int                  dtype, B, K, V, n, end_token;
} specdec_beam_select_args;
int specdec_beam_select(const specdec_beam_select_args* a, void* stream);

/* Debug / parity helpers (not on the hot path).
 * specdec_debug_logits: re-runs the vocabulary projection of the last verify
 *   (which = 0, rows [B*(k+1)]) or draft (which = 1, rows [n_active*k]) pass
 *   unfused and stores fp32 logits [rows,V].
 * specdec_debug_row_stats: per verify row of the last specdec_verify, 6 floats:
 *   max logit, argmax id, log-sum-exp, count of entries above the draft's logit,
 *   the draft's logit (+inf on the bonus row), draft id (-1 on the bonus row). */
int specdec_debug_logits(specdec_handle* h, int which, float* d_logits, void* stream);
int specdec_debug_row_stats(specdec_handle* h, float* d_stats, void* stream);
/* With option "trace" != 0 the first CTA of some kernels records nanosecond time stamps of its phases into a
 * 256-entry device array; this copies the first n (<= 256) entries to the host.  Synchronises the device. */
int specdec_debug_trace(specdec_handle* h, long long* h_out, int n);

/* Integrity check (debugging aid; the paper has no counterpart).  The handle's device arena places a 256-byte red
 * zone with a fixed pattern behind every block it hands out (weights, activations, caches, row metadata, session
 * state), so a kernel that writes past the end of its buffer damages one.  This call checks every red zone and scans
 * the activation buffers, the encoder memories and the K/V caches for NaN / Inf, on `stream`, and synchronises it.
 * It returns SPECDEC_OK whenever the check itself ran; the findings are in *out (first_* are -1 when the count is 0;
 * buffers are numbered in the order: residual rows, mask rows, normalised rows, QKV rows, attention output, cross
 * query rows, feed-forward rows, encoder memory, the second encoder's six buffers, K caches, V caches, the drafter's
 * caches, cross K/V of the verifier and of the drafter).  With option "debug_checks" = 1 every encode / draft / verify /
 * commit / generate call runs it before returning and fails with SPECDEC_ERR_CORRUPT on a finding. */
typedef struct specdec_integrity {
    int32_t zones;                   /* red zones checked                                  */
    int32_t damaged_zones;
    int32_t first_damaged_zone;      /* index (allocation order) of the first damaged one  */
    int32_t first_nonfinite_buffer;
    int64_t nonfinite;               /* NaN / Inf values found                             */
} specdec_integrity;
int specdec_debug_integrity(specdec_handle* h, specdec_integrity* out, void* stream);

/* Diagnostics: the cost of one kernel boundary inside a step.  Replays (from a CUDA graph, on the handle's own stream)
 * a chain of n_links launches of `grid` CTAs, each of which waits for its predecessor (programmatic dependent
 * launch, as between the kernels of a step), reads the word it wrote and writes it back; returns the best of ten
 * replays divided by n_links, in microseconds.  Synchronises. */
int specdec_debug_link_cost(specdec_handle* h, int n_links, int grid, double* h_us_per_link);

/* Diagnostics: nanoseconds per exchange round between the CTAs of one thread-block cluster (8 or 16 CTAs of 256
 * threads) through distributed shared memory: every CTA stores bytes_per_peer (0 .. 8192, a multiple of 16) bytes into each
 * peer's shared memory, arrives on every peer's barrier and waits for all arrivals; `rounds` rounds back to back.
 * What a fused cluster kernel pays where separate kernels pay a kernel boundary.  Synchronises. */
int specdec_debug_cluster_round(specdec_handle* h, int cluster_size, int bytes_per_peer, int rounds, double* h_ns_per_round);

/* Diagnostics: clocks per tcgen05.mma (M = 128 x N = bn x K = 16, bf16) when the operands already sit in shared memory:
 * one CTA per SM issues n_mma of them back to back with no loads in the loop.  two_sm = 1: the cta_group::2 form
 * (M = 256 over two SMs).  *h_issue_clocks = clocks until the issuing thread is done, *h_done_clocks = until the last
 * MMA has completed, both per MMA.  Tells a main loop that waits for operands from one the tensor pipe limits.
 * bf16 handles only.  Synchronises. */
int specdec_debug_mma_rate(specdec_handle* h, int bn, int two_sm, int n_mma, double* h_issue_clocks, double* h_done_clocks);
/* The same with what a real main loop adds.  bg_stages (0..6): while the MMAs are issued, another thread of every CTA
 * keeps that many bulk copies of 16 KB in flight from global memory (the verifier's embedding table, at least 8 MB) into
 * a separate region of the CTA's shared memory, as a TMA producer would; *h_bg_bytes_per_clock = bytes it landed per SM
 * clock and CTA.  commit_every (0 = never, else): a tcgen05.commit after every k-block of four MMAs to a barrier nobody
 * waits on (the multicast form for two-SM tiles), as a main loop issues one.  Tells whether the producer's writes or
 * the commits slow the tensor pipe down.  Synchronises. */
int specdec_debug_mma_rate_bg(specdec_handle* h, int bn, int two_sm, int n_mma, int bg_stages, int commit_every,
                              double* h_issue_clocks, double* h_done_clocks, double* h_bg_bytes_per_clock);

/* Scripted drafts, a benchmark / test hook with no counterpart in the paper: random-init
 * models almost never agree, so a workload's acceptance pattern is imposed instead.  After the
 * drafter pass has run, draft i of a sequence with j committed tokens is replaced by
 * d_script[b*stride + j + i] wherever that entry is >= 0.  d_script = NULL turns it off. */
int specdec_set_draft_script(specdec_handle* h, const int32_t* d_script, int B, int stride, void* stream);

/* With option "profile" = 1, every vocabulary-projection launch of the verify step (B*(k+1) rows)
 * inside specdec_generate is bracketed by CUDA events; this returns their summed duration and
 * count since the option was set. */
int specdec_profile_read(specdec_handle* h, double* h_ms, long long* h_launches);

/* Options (experiments and on-device cross-checks; every combination computes the same result):
 * "drafter_prefix_causal" 0 (default) / 1: the second reading of the Spec-Drafter's decoder mask.  0: no self-attention
 *                mask at all (every row of [BOS, committed, MASK x k] sees every row: "mask-predict manner", Section 3.1);
 *                the whole input is recomputed every iteration.  1: the committed tokens attend causally among
 *                themselves and only the [MASK] rows see everything; the drafter's decoder then keeps a K/V cache of the
 *                committed positions and a draft pass computes only the newly committed tokens and the k [MASK] rows
 *                (Section 3.1.2: the decoder runs every iteration, so its cost should not grow with the prefix).  A
 *                different function of the same weights: drafts differ, the verified output under beta = 1, tau = 0
 *                does not.  Takes effect at the next specdec_encode.
 * "gemm"         0 SIMT reference GEMM / 1 tcgen05 tensor-core GEMM (bf16 handles; default 1)
 * "attn"         0 warp-per-row reference attention / 1 tile attention (bf16: 64-wide heads on tensor cores; fp32: head sizes 4 .. 128, powers
 *                of two; default 1)
 * "skinny"       0/1 weight-streaming GEMM for passes of few rows (at most 176, wider than 512 at most 96, of these up
 *                to 144 or 80 rows with the LayerNorm in front fused; reductions of 512 and, for output projections, 768 beyond that while their CTAs are
 *                resident: 512 wide QKV at most 224 rows, output projections 736, 768 wide 320; default 1); fp32 handles: the fp32 GEMM of passes of at most 768 rows, LayerNorm fused up to 512 wide
 * "sk_cluster"   0/1 (default 1): that GEMM splits reductions of 1024 and more across a cluster of 2 or 4 CTAs, and attention over few
 *                rows of 4 or 8 64-wide heads runs on to the output projection, a cluster per 16 rows
 * "pair"         0/1 two-SM tensor-core tiles (cta_group::2) for GEMMs with >= 1024 rows and columns (default 0)
 * "enc_skinny"   0 / 1 (default) / 2: the weight-streaming GEMM does not / does / does serve the encoders (up to 72 rows, wider
 *                than 512 up to 40; those reductions beyond that, output projections up to 320 rows, 768 wide 256)
 * "ln_fuse"      0/1 the LayerNorm that reads the residual stream next runs inside the residual GEMM (default 0)
 * "splitk"       0/1 residual GEMMs with K >= 768 over few row tiles split K across a cluster (default 1)
 * "attn_stream"  0 / 1 by rule (default) / 2 / 3 / 4: attention CTAs of 16 queries with the keys spread over their warps, or of
 *                64 (2) or 32 (3, 4: 32-key blocks) queries with 16 to a warp
 * "attn_warps"   0 by rule (default), 4 or 8: the former with that many warps.  ("attn_rs" and "attn_stream_keys" are accepted
 *                and do nothing: they chose between kernels that are one now)
 * "tc_bn"        0 choose (default), else the column width of the tensor-core tiles (64 / 128 / 256)
 * "pdl"          0/1 programmatic dependent launch between the kernels of a step (default 1)
 * "graphs"       0/1 replay steps from CUDA graphs (default 1)
 * "gate"         0 never (default) / 1 above batch 4 / 2 always: each iteration of specdec_generate is one graph
 *                behind a device-side IF node, so the host can queue iterations ahead of the counter it reads
 * "poll_flag"    0/1 specdec_generate learns of each commit from a word in pinned host memory (default 1)
 * "poll_lag"     n: specdec_generate reads the unfinished-sequences counter n iterations late (default 0; 2 behind a gate)
 * "stats_timing" 0/1 fill ms_draft / ms_verify / ms_commit of specdec_stats (default 0; turns the gate off)
 * "profile"      0/1 see specdec_profile_read
 * "row_lse"      0/1 also accumulate the log-sum-exp of every verifier row (reported by specdec_debug_row_stats)
 * "diag_repeat"  bit mask: launch every attention (1; with the projections that run inside it), LayerNorm (2), non-residual GEMM (4),
 *                vocabulary kernel (8) of the path twice in a row (same result), so the step time rises by that class's cost inside
 *                the pipeline and the launch count by its launches
 * "trace"        see specdec_debug_trace
 * "debug_checks" 0/1 see specdec_debug_integrity (default 0: the check synchronises)
 * "poke_zone" i / "heal_zones" / "poke_nan" 0|1: test hooks for that check -- damage red zone i from the host, restore
 *                every red zone, put a NaN (or a zero) into the last element of the attention-output buffer
 * "inject_error" code: test hook -- the next specdec_verify / specdec_generate finds this code in the device error
 *                word, as if a bounded device-side wait had given up (no kernel waits, nothing faults) */
int specdec_set_option(specdec_handle* h, const char* name, int value);

/* Number of kernels the library has launched on this handle since create. */
long long specdec_launch_count(const specdec_handle* h);

const char* specdec_last_error(const specdec_handle* h);

#ifdef __cplusplus
}
#endif
#endif /* SPECDEC_H */
