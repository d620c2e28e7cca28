/*
 * libfastar: the attention hot path of FAST-AR on one MI355X (gfx950), as a C ABI.
 *
 * Four operations, as the method section of the paper states them, plus the code they share:
 *   fastar_encode        shared low-dimensional 8-bit ANN code of queries / keys / prompt keys
 *   tempcache_compress   merge one frame of new K/V into the bounded per-head cache (TempCache)
 *   ann_select_self      key blocks each query block attends to (AnnSA)
 *   ann_select_cross     prompt tokens each query block attends to (AnnCA)
 *   ann_cross_attn_fwd   the same selection and the attention over it in one launch
 *   sparse_attn_fwd      softmax attention over the selected keys only, with the log-multiplicity bias
 *
 * and, for programs that serve several requests at a time, dense attention with grouped heads over packed sequences:
 *   prompt_attn_fwd      causal or full attention over whole prompts
 *   kv_pages_plan        block tables and slot maps of a paged cache from the requests' lengths
 *   kv_pages_write       new keys and values into its pages: E4M3 codes with a scale per page and head
 *   paged_attn_fwd       attention over those pages, for single tokens and chunks
 *   qk_norm_rope         queries and keys normed per head and rotated by their positions
 *   kv_pages_write_rope  the same, the keys and values going straight into pages
 *   kv_pages_fork        new requests that begin with another one's tokens and share its full pages
 *   kv_pages_free        requests that end or are cut back give up pages that nobody else holds
 *   kv_pages_compact     the tokens that a mask keeps move together, into fewer pages
 *
 * Conventions (all entry points):
 *   - Every pointer is a DEVICE pointer unless it points to one of the small structs below, which
 *     are read on the host at call time.  The caller owns every buffer; the library allocates
 *     nothing and never synchronises with the host.  It keeps no state that a result depends on: the
 *     only process-wide data are per-device marks that the one-time kernel set-up has been done
 *     (fastar_init, or lazily and thread-safely by the first call that needs it).
 *   - `stream` is a hipStream_t passed as void*.  Work is enqueued on it and the call returns.
 *   - Tensors are DENSE row-major: [H, N, d] means element (h, n, t) at (h*N + n)*d + t; there are no
 *     stride arguments (the calls that take fastar_rows have them).  The key/value tiles of the attention kernels are fetched straight into LDS
 *     from one base address per tile with fixed row pitch d * sizeof(element), and the cache arrays
 *     K, V, code, cnt, stamp are indexed by one slot number; a strided view would put an address
 *     computation per row back into those loops.  A caller that holds a strided view passes a
 *     contiguous copy.  The batch dimension is folded into H.  Rows of Q/K/V/O must be 16-byte aligned.
 *   - dtype: FASTAR_F32 (float) or FASTAR_BF16 (bfloat16).  Q, K, V, O of one call share it.
 *   - Return value: FASTAR_OK, or a negative code found on the host before anything is launched
 *     (INVALID_ARG: null / negative / inconsistent argument; UNSUPPORTED: a shape the kernels are
 *     not built for; WORKSPACE: workspace too small), or FASTAR_ERR_HIP when a launch failed.
 *     Conditions only the device can see (a full cache dropping tokens) are reported through the
 *     `stats` output, never through the return value.
 *   - Index outputs are deterministic: every decision is taken on exact integer scores with ties
 *     going to the lowest index, so repeated calls and other implementations of the same
 *     definition give identical bits.
 */
#ifndef FASTAR_H
#define FASTAR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FASTAR_OK 0
#define FASTAR_ERR_INVALID_ARG (-1)
#define FASTAR_ERR_UNSUPPORTED (-2)
#define FASTAR_ERR_WORKSPACE (-3)
#define FASTAR_ERR_HIP (-4)
#define FASTAR_ERR_STATIC_SCRATCH (-5) /* the problem needs more than FASTAR_STATIC_SCRATCH_BYTES */

/* size of the library's static device scratch (ann_select_self_static), held by every GPU the library runs on */
#define FASTAR_STATIC_SCRATCH_BYTES (32 * 1024 * 1024)

#define FASTAR_F32 0
#define FASTAR_BF16 1

#define FASTAR_OP_COMPRESS 1
#define FASTAR_OP_SELECT_SELF 2
#define FASTAR_OP_SELECT_CROSS 3
#define FASTAR_OP_SELECT_LSH 4
#define FASTAR_OP_SELECT_BUCKETS 5 /* pass the number of prompt tokens as r */
#define FASTAR_OP_ATTN 6           /* sparse_attn_fwd_ws, sparse_attn_fwd_fp8_ws: a fixed amount, whatever the shape */
#define FASTAR_OP_PAGED_ATTN 7     /* paged_attn_fwd: a fixed amount, whatever the shape */
#define FASTAR_OP_PAGES 8          /* kv_pages_free, kv_pages_compact: pass B as H, max_pages as n_q, n_pages as n_k, P as r */

/* representative key of a merged TempCache group (tempcache_compress, rep_mode) */
#define FASTAR_REP_LAST 0
#define FASTAR_REP_MEAN 1
#define FASTAR_REP_MEDOID 2

/*
 * Bounded per-head KV cache with multiplicities (Lemma 1 of the paper: a group of merged keys is
 * kept as one representative key, the mean of the group's values and the group size m, which
 * enters attention as a +log m logit shift).  Capacity C slots per head, len[h] <= C of them live.
 */
typedef struct {
    void *K;        /* [H,C,d] dtype   representative = most recent key of each group            */
    void *V;        /* [H,C,d] dtype   mean value of each group                                  */
    int8_t *code;   /* [H,C,r]         ANN code of K                                             */
    int32_t *cnt;   /* [H,C]           multiplicity m >= 1 of live slots                         */
    int32_t *stamp; /* [H,C]           frame id of the slot's last refresh                       */
    int32_t *len;   /* [H]             live slots                                                */
    int32_t H, C, d, r, dtype;
} fastar_cache;

/*
 * Definition of the ANN code (Sec. 5.1: shared low-dimensional random projection + low-bit
 * quantisation, 8 bit by default), in integer arithmetic so that every score is exact:
 *   xq[t] = clamp(rint(x[t] * qscale), -127, 127)           one float32 multiply, ties to even
 *   y[j]  = sum_t R[t][j] * xq[t]                           int32
 *   c[j]  = clamp(floor((y[j] + 2^(shift-1)) / 2^shift), -127, 127)
 */
typedef struct {
    const int8_t *R; /* [d,r] device, entries -1 / +1 */
    float qscale;
    int32_t shift;   /* >= 1 */
} fastar_codec;

/*
 * One-time set-up for the CURRENT device: lets the kernels that stage large tiles use more than 64 KB of LDS.
 * Optional: every entry point does the part it needs on its first call on a device (thread-safe).  Call it before
 * capturing entry points into a HIP graph, so that no attribute call falls inside the capture.  Launches nothing.
 */
int fastar_init(void);

/* Library version string (host pointer, static storage). */
const char *fastar_version(void);

/* Human-readable name of a return code (host pointer, static storage). */
const char *fastar_strerror(int code);

/*
 * Bytes of device workspace an operation needs (FASTAR_OP_*).  Arguments that an operation does
 * not use are ignored.  COMPRESS: H, C, n_new (as n_q), r.  SELECT_SELF: H, n_q, C (as n_k), BQ,
 * BK, n_rep, r.  SELECT_CROSS: H, n_q, n_p (as n_k), BQ.  SELECT_LSH: H, n_q, C (as n_k), n_bits (as r), BQ, BK,
 * n_rep.  Returns 0 for an unknown op.
 */
size_t fastar_workspace_bytes(int op, int H, int n_q, int n_k, int r, int BQ, int BK, int n_rep);

/*
 * ANN codes (Sec. 5.1) of n_vec vectors.
 *   x        [n_vec, d] dtype (device), d in {64, 128}
 *   codec    host struct; codec->R device [d, r], r in {32, 64}
 *   code_out [n_vec, r] int8 (device)
 */
int fastar_encode(const void *x, int dtype, int64_t n_vec, int d, const fastar_codec *codec, int r,
                  int8_t *code_out, void *stream);

/*
 * Prompt-induced buckets (Sec. 5.4, first paragraph: self-attention reuses the semantic buckets found by
 * cross-attention pruning; a query is assigned to one or more buckets and attends only to keys of the same
 * bucket(s)).  The prompt tokens are the buckets: a code belongs to the m prompt tokens with the largest code inner
 * product (the products ann_select_cross ranks prompt tokens by), ties to the smaller token id.
 *   code   [H,C,r] int8 (device), pcode [H,n_p,r] int8 (device), both 16-byte aligned
 *   idx    [H,n] int32 rows to assign (device; entries < 0 or >= C are skipped, repeats are harmless), or NULL for
 *          rows 0..n-1 (n <= C): a caller that keeps one bucket row per cache slot re-assigns only the slots
 *          tempcache_compress wrote (its merge_map)
 *   bucket [H,C,m] int32 out (device): token ids, best first; -1 where n_p < m; rows not named are left as they are
 * Supported: r in {32, 64}, n_p <= 2048, m <= 8.
 */
int ann_prompt_buckets(const int8_t *code, int C, const int32_t *idx, int n, const int8_t *pcode, int n_p, int H, int r,
                       int m, int32_t *bucket, void *stream);

/*
 * AnnSA on those buckets: a query block owns the buckets of its queries, a key block those of its live keys; a key
 * block is a candidate only if the two share a bucket; of the candidates the n_sel that share the most are kept
 * (ties: lowest index), written ascending to sel, -1 padded; nsel = their number (it can be 0).  The first n_sink and
 * the last n_local live key blocks are always kept and count against the budget (n_sink + n_local <= n_sel).
 *   qbucket [H,n_q,m], kbucket [H,C,m] int32 (entries outside [0, n_p) are ignored), len [H];
 *   sel [H,n_qb,n_sel], nsel [H,n_qb] out;  ws of fastar_workspace_bytes(FASTAR_OP_SELECT_BUCKETS, H, n_q, C, n_p, BQ, BK, 0).
 * Supported: n_p <= 2048; ceil(n_q/BQ) * ceil(n_p/32) * 4 bytes <= 48 KiB.
 */
int ann_select_buckets(const int32_t *qbucket, int n_q, const int32_t *kbucket, const int32_t *len, int H, int C, int m,
                       int n_p, int BQ, int BK, int n_sel, int n_sink, int n_local, int32_t *sel, int32_t *nsel, void *ws,
                       size_t ws_bytes, void *stream);

/*
 * Codes that are really `bits` wide (appendix, "Quantization precision for ANN matching": the bit width of the
 * retrieval codes is varied; narrower codes are cheaper to store and to stream).  As fastar_encode, but the last step
 * saturates to +-(2^(bits-1) - 1) and entry j of a vector occupies bits [bits*(j mod 8/bits), +bits) of byte
 * j / (8/bits): packed_out [n_vec, r*bits/8] uint8 (device, 4-byte aligned).  bits in {2, 4, 8}; 8 is fastar_encode.
 * Supported for bits < 8: r = 32.
 */
int fastar_encode_packed(const void *x, int dtype, int64_t n_vec, int d, const fastar_codec *codec, int r, int bits,
                         uint8_t *packed_out, void *stream);

/*
 * ann_select_self_forced on such packed codes: qcode [H,n_q,r*bits/8], kcode [H,C,r*bits/8]; the result is that of
 * ann_select_self_forced on the unpacked entries.  The key codes are streamed as they are stored (r*bits/8 bytes per
 * key) and widened in registers.  Same workspace as ann_select_self (the summaries are kept one byte per entry).
 * Supported for bits < 8: r = 32.
 */
int ann_select_self_packed(const int8_t *qcode, int n_q, const int8_t *kcode, const int32_t *len, int H, int C, int r,
                           int bits, int BQ, int n_rep, int BK, int n_sel, int n_sink, int n_local, int32_t *sel,
                           int32_t *nsel, void *ws, size_t ws_bytes, void *stream);

/*
 * Sign codes, the hash of the LSH paragraph of Sec. 5.1: one bit per random projection, the side of the
 * hyperplane the quantised vector lies on.  bit j = 1 iff sum_t R[t][j] * xq[t] >= 0, xq as in fastar_codec.
 *   x        [n_vec, d] dtype (device), d in {64, 128}
 *   R        [d, n_bits] int8 entries -1 / +1 (device), n_bits in {64, 128, 256}
 *   bits_out [n_vec, n_bits/32] uint32 (device); bit j of a vector sits in word j/32 at position j%32
 */
int fastar_encode_sign(const void *x, int dtype, int64_t n_vec, int d, const int8_t *R, float qscale, int n_bits,
                       uint32_t *bits_out, void *stream);

/*
 * Selection on sign codes (Sec. 5.3 / 5.4 with the LSH family of Sec. 5.1): candidates are ranked by the number of
 * hash bits they share with the query side.  Query block b (BQ queries) is summarised by n_rep majority codes, one
 * per run of BQ/n_rep queries (bit j = 1 iff at least half of the run's queries have it set); the score of key
 * block kb (BK keys) is the largest number of equal bits between a summary and a live key of the block; the
 * min(n_sel, ceil(len/BK)) best key blocks (ties: lowest index) are written ascending to sel, -1 padded.
 * n_rep = BQ, BK = 1 is the cross-attention form (a prompt token is scored by its best-matching query).
 *   qbits [H,n_q,W], kbits [H,C,W] uint32 (W = n_bits/32), len [H];  sel [H,n_qb,n_sel], nsel [H,n_qb] out.
 * Supported: n_bits in {64,128,256}; BK a power of two <= 64 or a multiple of 64; BQ a multiple of n_rep.
 */
int ann_select_lsh(const uint32_t *qbits, int n_q, const uint32_t *kbits, const int32_t *len, int H, int C,
                   int n_bits, int BQ, int n_rep, int BK, int n_sel, int32_t *sel, int32_t *nsel, void *ws,
                   size_t ws_bytes, void *stream);

/*
 * Hash-table form of ann_select_lsh (Sec. 5.1, LSH paragraph: a query only compares against keys that land in the same
 * bucket(s); Sec. 2: multi-table bucket probing).  The hash bits are cut into n_bits / band_bits bands, one table each;
 * a vector's bucket in a table is its band.  A summary and a key collide in a table when their buckets differ in at
 * most `radius` bits (0: the same bucket; more: the neighbouring buckets are probed as well).  A pair scores its
 * colliding tables, a key block its best (summary, live key) pair; key blocks without a collision are no candidates;
 * of the candidates the n_sel best are kept (ties: lowest index), -1 padded; nsel = their number (it can be 0).  The
 * first n_sink / last n_local live key blocks are always kept (n_sink + n_local <= n_sel).
 * Same arrays and workspace as ann_select_lsh.  Supported: band_bits in {4, 8, 16, 32}.
 */
int ann_select_lsh_buckets(const uint32_t *qbits, int n_q, const uint32_t *kbits, const int32_t *len, int H, int C,
                           int n_bits, int band_bits, int radius, int BQ, int n_rep, int BK, int n_sel, int n_sink,
                           int n_local, int32_t *sel, int32_t *nsel, void *ws, size_t ws_bytes, void *stream);

/*
 * TempCache (Sec. 5.2 and Lemma 1): merge one frame of n_new tokens per head into the cache.  Every
 * decision is taken against the cache as it is at entry; a chunk of several frames is several calls.
 *   1. probe code cp_i = code(P_new[i]) (P_new NULL => K_new), key code ck_i = code(K_new[i]).
 *   2. top-1 match among the candidate slots (cand [H,n_cand] names a SET of slot ids: its order and
 *      repeated ids mean nothing, ids outside [0,len) are skipped; cand NULL => every live slot):
 *      j*(i) = argmax_j S(i,j), ties to the smallest slot,
 *      S = 2 cp_i.code_j - |code_j|^2 (metric 0, nearest in code space) or cp_i.code_j (metric 1).
 *   3. similarity threshold on the 8-bit quantised full-width keys a = xq(K_new[i]), b = xq(K[j*]):
 *      merged_i <=> a.b > 0 and (a.b)^2 * 65536 >= tau2_q16 * |a|^2 |b|^2, with
 *      tau2_q16 = rint(tau^2 * 65536) in [0, 131072].
 *   4. every slot keeps, of the tokens merged into it, the one closest in code space (metric 0:
 *      S - |cp_i|^2, metric 1: S; ties to the smallest token) as its new representative key; its
 *      value becomes the mean over the enlarged group and its multiplicity grows by the joiners.
 *      rep_mode FASTAR_REP_MEAN (appendix ablation "Representative selection in KV merging") stores the
 *      multiplicity-weighted mean key instead: float32, multiplicity * old key, then the joiners' keys in
 *      ascending token order, one division, one rounding to dtype; the slot's code is the code of the
 *      stored key (one more launch).  FASTAR_REP_MEDOID stores the medoid key: of the slot's stored key (standing for
 *      the multiplicity tokens merged so far) and this call's joiners (weight 1 each) the one with the smallest weighted
 *      total squared distance to the others in code space (exact integers; ties to the stored key, then the smaller
 *      token); the stored key winning leaves key and code as they are.  FASTAR_REP_LAST is the method's own choice and
 *      the fast path.
 *   5. unmerged tokens are appended in token order.  If the cache would exceed C, the live slots
 *      that received no token in this call are evicted, smallest (stamp, slot) first, and refilled
 *      in ascending slot order; if there are too few of those, the last unmerged tokens are dropped.
 *   K_new, V_new, P_new [H,n_new,d] dtype;  frame_id is stored as the stamp of every written slot.
 * Outputs:
 *   merge_map [H,n_new] int32  destination slot of each token, -1 if dropped
 *   merged    [H,n_new] uint8  1 if the token joined an existing slot
 *   stats     [H,8]     int32  {len after, n_merged, n_appended, n_evicted, n_dropped, 0, 0, status}
 *                              status 0; 1 if a bounded wait inside the eviction plan ran out (its workgroups, which
 *                              meet through global memory, were not all running at once): nothing of this call is
 *                              applied to the head then, its K, V, code, cnt, stamp and len stay as they were, every
 *                              token of the head is reported dropped (merge_map -1, merged 0, n_dropped = n_new), and a
 *                              persistent workspace has to be zero-filled again before its next use; 2 if the stamps
 *                              of the evictable slots span 2^20 frames or more: the choice of victims is then not
 *                              guaranteed to be the oldest-first one.  With ws_persistent, C <= 65536 and n_new <= 2048
 *                              neither occurs: nothing waits there, and the choice is exact for any stamps (frames of
 *                              up to 8192 tokens too while the heads are few);
 *                              3 if ws_persistent was set for a workspace that is neither zero-filled nor left by
 *                              a finished call: nothing is applied either (as for status 1)
 *   ws / ws_bytes              workspace of fastar_workspace_bytes(FASTAR_OP_COMPRESS, ...), 256-byte aligned
 *   ws_persistent              0: the workspace may hold anything (the call clears what it needs: one launch more).
 *                              1: the caller zero-filled the workspace once and since then only calls of this
 *                              function on this cache have written to it (frames may differ in length: the workspace
 *                              is then sized for the longest); every call leaves it as clean as a
 *                              zero-filled one, so the match can go straight on to the threshold test (candidate
 *                              lists that fit LDS, P_new NULL) and short caches are settled in one launch.  A
 *                              workspace whose per-head marks say otherwise is reported (status 3) by every such
 *                              call; of the rest of its contents, calls without a list, with one that does not fit
 *                              LDS or with P_new clear what they need.  The library still keeps no state of its own:
 *                              the state is the caller's buffer.
 * The cache struct and the codec struct are host structs; cache->len is updated on the device.
 * Supported: d in {64,128}, r in {32,64}; C up to about 393 000 * min(16, 1024 / H) slots per head (the eviction
 *            plan runs on that many workgroups per head and each keeps a bitmap of its share of the slots in LDS):
 *            6 million for up to 64 heads; FASTAR_ERR_UNSUPPORTED otherwise.
 */
int tempcache_compress(const fastar_cache *cache, const fastar_codec *codec, const void *K_new,
                       const void *V_new, const void *P_new, int n_new, const int32_t *cand, int n_cand,
                       int metric, int32_t tau2_q16, int32_t frame_id, int rep_mode, int32_t *merge_map,
                       uint8_t *merged, int32_t *stats, void *ws, size_t ws_bytes, int ws_persistent, void *stream);

/*
 * AnnSA (Sec. 5.4 with the ANN goal of Sec. 5.1): for every head and every block of BQ queries,
 * the n_out = min(n_sel, ceil(len/BK)) key blocks of BK keys with the largest code score.
 *   Query block b is summarised by n_rep mean codes, one per run of g = BQ/n_rep queries:
 *   rep = floor((sum of the run's codes + floor(g/2)) / g); runs without a query are skipped.
 *   Score of key block kb = max over summaries and over the block's live keys k < len of rep.code_k.
 *   Ties go to the smaller block index; the result is written in ascending block order.
 *   qcode [H,n_q,r], kcode [H,C,r], len [H]
 *   sel   [H,n_qb,n_sel] int32 out, padded with -1;  nsel [H,n_qb] int32 out;  n_qb = ceil(n_q/BQ)
 * Supported: r in {32,64}; BQ a multiple of n_rep; n_rep in {1,2,4,8,16,32}; BK a multiple of 32;
 *            at most 1024 query blocks per head.
 */
int ann_select_self(const int8_t *qcode, int n_q, const int8_t *kcode, const int32_t *len, int H, int C, int r,
                    int BQ, int n_rep, int BK, int n_sel, int32_t *sel, int32_t *nsel, void *ws,
                    size_t ws_bytes, void *stream);

/*
 * AnnSA with forced key blocks (Sec. 2: rolling-window generators keep their first frames as an attention sink; a
 * local window is the usual companion): as ann_select_self, but the first n_sink key blocks and the last n_local live
 * key blocks of every head are always among the selected ones.  They count against the budget
 * (n_sink + n_local <= n_sel, FASTAR_ERR_INVALID_ARG otherwise); the rest of it goes to the best-scoring other blocks.
 * n_sink = n_local = 0 is ann_select_self.  Same workspace.
 */
int ann_select_self_forced(const int8_t *qcode, int n_q, const int8_t *kcode, const int32_t *len, int H, int C, int r,
                           int BQ, int n_rep, int BK, int n_sel, int n_sink, int n_local, int32_t *sel, int32_t *nsel,
                           void *ws, size_t ws_bytes, void *stream);

/*
 * ann_select_self for callers that cannot allocate or bring a workspace: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and bit-identical outputs as ann_select_self,
 * but the summaries and the score rows live in a static device array of FASTAR_STATIC_SCRATCH_BYTES inside the library
 * (each GPU holds its own copy until the process ends; its address is looked up once per device, by fastar_init or by
 * the first call).  The call allocates nothing: no hipMalloc / hipFree, no workspace argument.
 *   - Problems that need more scratch than that (fastar_workspace_bytes(FASTAR_OP_SELECT_SELF, ...) is the amount;
 *     the world-model layer with 40 heads x 29 query blocks x 3600 key blocks needs 16.8 MB) return
 *     FASTAR_ERR_STATIC_SCRATCH and launch nothing.
 *   - All calls on one GPU share the one array: calls that may overlap on a GPU (different streams, different host
 *     threads) race on it.  Calls on one stream are ordered and safe.  Nothing in the array has to start from zero
 *     and nothing of a previous call is read.
 */
int ann_select_self_static(const int8_t *qcode, int n_q, const int8_t *kcode, const int32_t *len, int H, int C, int r,
                           int BQ, int n_rep, int BK, int n_sel, int32_t *sel, int32_t *nsel, void *stream);

/*
 * AnnCA (Sec. 5.3): for every head and every block of BQ queries, the min(n_sel, n_p) prompt tokens
 * with the largest max over the block's queries of c_q.c_p (a token is kept when at least one query
 * of the block is its neighbour).  Ties to the smaller token index, ascending output, -1 padding.
 *   qcode [H,n_q,r], pcode [H,n_p,r];  sel [H,n_qb,n_sel], nsel [H,n_qb] out.
 * BQ is free (it need not be sparse_attn_fwd's block size): BQ = tokens per frame gives the per-frame selection
 * of Sec. 5.3, whose list the caller then shares among the query blocks of that frame's attention call.
 * Supported: r in {32,64}; n_p <= 12288 (the scores of one query block over the prompt live in LDS).
 */
int ann_select_cross(const int8_t *qcode, int n_q, const int8_t *pcode, int n_p, int H, int r, int BQ,
                     int n_sel, int32_t *sel, int32_t *nsel, void *ws, size_t ws_bytes, void *stream);

/*
 * AnnCA in one launch (Sec. 5.3): the selection of ann_select_cross followed by the attention of sparse_attn_fwd
 * over it (BK = 1, no multiplicities, every prompt token live), for callers that need both and no lse:
 *   sel, nsel  exactly what ann_select_cross(qcode, pcode, BQ, n_sel) writes;
 *   O          exactly what sparse_attn_fwd(Q, Kp, Vp, NULL, len = n_p, sel, nsel, BQ, 1, n_sel, scale) computes
 *              (same arithmetic: bf16 products, fp32 softmax over the selected tokens in one piece).
 *   Q [H,n_q,d], Kp, Vp [H,n_p,d] bf16;  qcode [H,n_q,r], pcode [H,n_p,r];  O [H,n_q,d] bf16 out.
 * Supported: bf16, d = 128, BQ = 128, n_sel <= 64, r in {32,64}, n_p <= 12288; anything else is
 * FASTAR_ERR_UNSUPPORTED and the two separate calls do the same work.  No workspace.
 */
int ann_cross_attn_fwd(const void *Q, const int8_t *qcode, int n_q, const void *Kp, const void *Vp,
                       const int8_t *pcode, int n_p, int H, int d, int dtype, int r, int BQ, int n_sel, float scale,
                       int32_t *sel, int32_t *nsel, void *O, void *stream);

/*
 * Block-sparse attention (Eq. 1 restricted to the candidate set of Sec. 5.1, logits shifted by
 * +ln(cnt) as in Lemma 1).  For query i of query block b, over the live keys J of the key blocks
 * sel[h][b][0 .. nsel[h][b]):  l_j = scale * q_i.k_j + ln(cnt_j);  o_i = sum_j softmax(l)_j v_j;
 * lse_i = ln sum_j exp(l_j).  J empty => o_i = 0, lse_i = -inf.
 *   Q [H,n_q,d], K,V [H,C,d] dtype;  cnt [H,C] or NULL (no bias);  len [H];
 *   sel [H,n_qb,n_sel] (entries < 0 are padding), nsel [H,n_qb];
 *   O [H,n_q,d] dtype out;  lse [H,n_q] float out or NULL.
 * Supported: bf16 with d in {64,128}, BQ in {64,128}, BK a power of two <= 64 (MFMA path, fp32
 * softmax and accumulation); fp32 with d in {64,128}, BQ <= 128, BK <= 64 (plain fp32 arithmetic).
 * scale must be positive and finite (FASTAR_ERR_INVALID_ARG otherwise).  bf16: tile rows are addressed by 32-bit
 * byte offsets inside a head, so C * d * 2 must stay below 2^32 (FASTAR_ERR_UNSUPPORTED otherwise).
 */
int sparse_attn_fwd(const void *Q, int n_q, const void *K, const void *V, const int32_t *cnt,
                    const int32_t *len, int H, int C, int d, int dtype, const int32_t *sel, const int32_t *nsel,
                    int BQ, int BK, int n_sel, float scale, void *O, float *lse, void *stream);

/*
 * sparse_attn_fwd with a workspace: same arguments, same result (to the tolerance of the attention itself: a block
 * that several workgroups share is put together from their partial sums).  Two kinds of bf16, d = 128, BQ = 128 launches
 * leave such partial sums (fragments) in `ws`, and a second small launch combines them:
 *   - more (head, query block) pairs than the chip holds at once, in a number that would leave a short last round of
 *     workgroups: whole rounds of query blocks are taken by one workgroup each, and the blocks left over are cut into
 *     equal shares of their tiles for all resident workgroups;
 *   - at most 128 pairs with more than 8 tiles of 64 listed keys each (n_sel * BK > 512): a block's tiles are cut into
 *     runs, a workgroup each, where that is expected to be faster than keeping a block in one launch.
 * Which launches these are follows from H, n_q, n_sel and BK alone (attn_split_full_per and attn_parts in common.hpp,
 * waves_per_group in attention.hip).
 * Every other call runs exactly as sparse_attn_fwd and leaves `ws` untouched.  Calls that may be in flight at the same
 * time (two streams, two threads) need a workspace each; one is enough for calls that follow one another on a stream.
 *   ws / ws_bytes  fastar_workspace_bytes(FASTAR_OP_ATTN, ...) bytes, 256-byte aligned; contents need not be kept
 */
int sparse_attn_fwd_ws(const void *Q, int n_q, const void *K, const void *V, const int32_t *cnt, const int32_t *len,
                       int H, int C, int d, int dtype, const int32_t *sel, const int32_t *nsel, int BQ, int BK, int n_sel,
                       float scale, void *O, float *lse, void *ws, size_t ws_bytes, void *stream);

/*
 * 8-bit floating-point K/V for the attention itself (Sec. 5.1, quantised-search paragraph; appendix ablation
 * "Quantization precision for ANN matching" carried over from the retrieval codes to the attended keys and values).
 * Format: E4M3 (OCP 8-bit floating point, "FN": bias 7, subnormals, no infinities, largest finite value 448); values
 * beyond +-448 saturate; conversion rounds to nearest, ties to even.
 *
 * fastar_kv_to_fp8 keeps an 8-bit copy of a bf16 / fp32 cache (d = 128) up to date:
 *   K8   [H, Cp, 128] uint8      codes of the keys, rows as in cache->K; Cp = C rounded up to a multiple of 64
 *   V8T  [H, Cp/64, 128, 64]     codes of the values, every block of 64 slots transposed:
 *                                element (h, blk, t, j) = code of V[h][64 blk + j][t]
 * Every block of 64 slots that holds a live slot with stamp >= stamp_lo is rewritten whole (live slots with the codes
 * of the stored rows, dead slots with zero); other blocks are not touched.  After tempcache_compress(frame_id = f),
 * stamp_lo = f brings the copy up to date; stamp_lo = INT32_MIN rebuilds it.  The caller zero-fills K8 and V8T once:
 * the attention reads whole blocks and a dead slot must hold a finite code.
 */
int fastar_kv_to_fp8(const fastar_cache *cache, int32_t stamp_lo, uint8_t *K8, uint8_t *V8T, void *stream);

/*
 * sparse_attn_fwd over that copy: the same definition (Eq. 1 restricted to the selected key blocks, +ln(cnt) bias of
 * Lemma 1) on the exact values of the E4M3 codes of K and V and of Q rounded to E4M3.  Both products run on the 8-bit
 * floating-point matrix instructions (fp32 accumulation); the softmax weights are rounded to E4M3 before the second
 * product and the row sums are taken over the rounded weights, so every output is a convex combination of the stored
 * values.  Q, O [H,n_q,128] bf16; cnt [H,C] or NULL; len [H]; sel / nsel as for sparse_attn_fwd; lse [H,n_q] or NULL.
 * Supported: d = 128, BQ = 128, BK = 64 (one selection entry = one block of the copy); FASTAR_ERR_UNSUPPORTED otherwise.
 */
int sparse_attn_fwd_fp8(const void *Q, int n_q, const uint8_t *K8, const uint8_t *V8T, const int32_t *cnt,
                        const int32_t *len, int H, int C, int d, const int32_t *sel, const int32_t *nsel, int BQ, int BK,
                        int n_sel, float scale, void *O, float *lse, void *stream);

/*
 * sparse_attn_fwd_fp8 with a workspace, as sparse_attn_fwd_ws is to sparse_attn_fwd: same arguments, same result (to the
 * tolerance of the attention itself).  The same two kinds of launches leave fragments in `ws` for a second small launch to
 * combine: those that would end in a short last round of workgroups, and those of at most 256 (head, query block) pairs
 * whose lists are long enough for several workgroups each.  Every other call runs exactly as sparse_attn_fwd_fp8 and
 * leaves `ws` untouched.  Calls that may be in flight at the same time need a workspace each.
 *   ws / ws_bytes  fastar_workspace_bytes(FASTAR_OP_ATTN, ...) bytes, 256-byte aligned; contents need not be kept
 */
int sparse_attn_fwd_fp8_ws(const void *Q, int n_q, const uint8_t *K8, const uint8_t *V8T, const int32_t *cnt,
                           const int32_t *len, int H, int C, int d, const int32_t *sel, const int32_t *nsel, int BQ,
                           int BK, int n_sel, float scale, void *O, float *lse, void *ws, size_t ws_bytes, void *stream);

/* ================================================================================================================
 * Several requests at a time.  The tokens of B sequences lie one sequence after the other in arrays of n_tok rows
 * (packed): sequence b owns rows cu[b] .. cu[b+1]-1, cu [B+1] int32 on the device, not falling.  Offsets are cut to
 * [0, n_tok]; rows outside of every sequence are neither read nor written.  A sequence may have no rows.
 *
 * Grouped heads: Hq query heads share Hkv key heads, Hq a multiple of Hkv; query head h reads key head h / (Hq / Hkv).
 *
 * Causal: the last query of a sequence is its last key.  With a queries and n keys, query i sees keys j <= n - a + i; for
 * a > n the first a - n queries see nothing.  A query without a key: o = 0, lse = -inf.
 * ================================================================================================================ */

/*
 * A strided view [H, n, d]: element (h, i, t) at p + h*head + i*row + t, strides in elements, >= 0, every row 16-byte
 * aligned; the stride of a dimension of one may be anything.  [H, n, d] and [n, H, d] arrays and the parts of a fused projection's output are such views.  Rows of an
 * output must not overlap: one of the strides is at least d, the other at least the first one's extent.  An output shares no
 * memory with an input.
 */
typedef struct {
    void *p;
    int64_t head, row;
} fastar_rows;

/*
 * Attention over whole prompts: l_j = scale * q_i.k_j over the keys j that query i sees, o_i = sum_j softmax(l)_j v_j,
 * lse_i = ln sum_j exp(l_j).
 *   Q [Hq,n_tok_q,d], K, V [Hkv,n_tok_k,d], O [Hq,n_tok_q,d] views of dtype;  lse [Hq,n_tok_q] float (dense) or NULL
 *   cu_q [B+1] rows of Q and O;  cu_k [B+1] rows of K and V, or NULL: cu_q
 *   causal  0: every query sees all keys of its sequence;  1: as above
 * bf16: bf16 products (the weights are rounded to bf16; those below 2^-126 of a row's largest are zero), fp32 softmax and
 * sums; fp32: plain fp32 arithmetic.
 * Supported: d in {64, 128}; scale positive, scale * log2(e) finite; rows of K and V at most 2^24 bytes apart;
 * n_tok_q * Hq < 2^30, n_tok_k <= 2^30; n_tok_q * Hq / 256 + (B + 1) * Hkv < 2^23 (fp32: n_tok_q * Hq / 64 ... < 2^24).  No workspace.  n_tok_q = 0 or B = 0 launches nothing.
 * Where a causal call meets infinities or NaN among the values, or any call values near the end of the range, the queries of the tiles
 * concerned are done again one by one, so that none sees what is masked for it and no mean is lost: right, and many times slower.
 */
int prompt_attn_fwd(const fastar_rows *Q, const fastar_rows *K, const fastar_rows *V, const int32_t *cu_q,
                    const int32_t *cu_k, int B, int n_tok_q, int n_tok_k, int Hq, int Hkv, int d, int dtype, int causal,
                    float scale, const fastar_rows *O, float *lse, void *stream);

/*
 * A cache in pages of P tokens.  Keys and values are E4M3 codes (the format of fastar_kv_to_fp8) in cells of 16 tokens x
 * 16 coordinates, 256 bytes: a cell of K8 holds a token's 16 coordinates together, one of V8 a coordinate's 16 tokens, so
 * that 16 consecutive bytes are an operand of the matrix instructions for either product.
 *   K8 [n_pages, Hkv, P/16, d/16, 16 tokens, 16 coordinates], V8 [n_pages, Hkv, P/16, d/16, 16 coordinates, 16 tokens]
 *   kscale, vscale [n_pages, Hkv] float, powers of two: a code stands for its E4M3 value times the scale of its page and
 *   head.  E4M3 has an exponent of its own, so that a finer scale would not make codes more precise; a power of two lets
 *   the codes of a page be carried to a larger scale without a second rounding (but for those that become subnormal).
 * P in {16, 32, 64}, n_pages * P < 2^31, Hkv * P * d < 2^31.  Token i of a sequence lies in page table[b][i / P] of its block table, at i % P.
 */
typedef struct {
    uint8_t *K8, *V8;
    float *kscale, *vscale;
    int32_t n_pages, Hkv, P, d;
} fastar_pages;

/*
 * Block tables and slot maps for the next step of B requests.
 *   n_new [B]             tokens that request b appends; 0: none; negative: the request has ended
 *   len [B]               tokens that it holds
 *   table [B, max_pages]  block tables, updated;  the first ceil(len/P) entries of a row count, others mean nothing
 *   pool [n_pages]        free pages, a stack whose first pool_n[0] entries count, updated
 * 1. The pages of ended requests go on top of the stack, in the order of the requests and of their tables.
 * 2. Request b needs ceil((len+n_new)/P) - ceil(len/P) pages.  They are taken from the top, in the order of the requests.
 *    A request is refused, and keeps what it has, if its table is too short (status 2), if its rows go beyond n_tok
 *    (status 3), or if it needs pages and those needed up to and including it are more than there are (status 1; requests
 *    refused for status 2 or 3 need none).
 * Outputs:
 *   len_out [B]       tokens after the step (0 for ended requests); may be len itself
 *   pool_n_out [1]    free pages after the step; may be pool_n itself
 *   cu [B+1]          rows of the requests' new tokens: the prefix sums of max(n_new, 0), cut to n_tok
 *   slot [n_tok]      page * P + offset of each new token; -1 where the request is refused.  Rows from cu[B] on stay as they
 *                     are: an array that is used again, in a replayed graph say, is set to -1 before, or kv_pages_write finds
 *                     the slots of an earlier step there
 *   status [B]        0 (also for ended requests), 1, 2 or 3
 * Lengths and counts are cut to what the arrays hold; a table entry outside of [0, n_pages) gives slot -1.
 * Supported: P in {16, 32, 64}; max_pages * P and n_pages * P < 2^31.  One launch for few tokens, two for many; no workspace.
 */
int kv_pages_plan(const int32_t *n_new, const int32_t *len, int32_t *table, int B, int max_pages, int32_t *pool,
                  const int32_t *pool_n, int n_pages, int P, int n_tok, int32_t *len_out, int32_t *pool_n_out, int32_t *cu,
                  int32_t *slot, int32_t *status, void *stream);

/*
 * New keys and values into their pages.  K_new, V_new [Hkv,n_tok,d] views of dtype; slot [n_tok] int32 as kv_pages_plan
 * writes it: rows of one page follow one another, in the order of their slots, and a page has one such run of rows in a
 * call; negative slots and those >= n_pages * P are passed over.
 * Of a run the largest finite |x| per head asks for the scale s = 2^max(-100, ceil(log2(|x| / 448))).  A run that begins at
 * offset 0 begins the page anew: the page takes s, and codes behind the run stay as they are (they mean nothing).  Any other
 * run raises the page's scale to s if that is larger; all other codes of the page and head are then carried over to it (value
 * of the code times the old scale over the new one, rounded to nearest, ties to even).  New codes: x / scale rounded to
 * nearest, ties to even; infinities become the largest code of their sign, NaN stays NaN.
 * Supported: rows of K_new and V_new at most 2^24 bytes apart, (n_tok + P) * Hkv <= 2^29 - 1.
 */
int kv_pages_write(const fastar_pages *pages, const fastar_rows *K_new, const fastar_rows *V_new, int dtype,
                   const int32_t *slot, int n_tok, void *stream);

/*
 * Attention over such a cache: prompt_attn_fwd's definition with the keys and values that the codes stand for.
 *   Q, O [Hq,n_tok,d] bf16 views;  cu_q [B+1];  len [B] keys of every sequence (those of the queries among them, written
 *   before);  table [B, max_pages];  lse [Hq,n_tok] float or NULL;  causal as for prompt_attn_fwd
 * Keys on pages outside of [0, n_pages) are left out, like masked ones; len is cut to [0, max_pages * P].
 * Products in bf16 (codes are widened exactly; where a sequence has at most eight query rows on a key head and sequences have
 * at most 16 on average, weights have 16 bits), fp32 softmax and sums.  Sequences share the chip by their lengths, which the
 * device reads: long ones are cut into pieces whose fragments lie in ws, and a second launch puts them together.
 *   ws / ws_bytes  fastar_workspace_bytes(FASTAR_OP_PAGED_ATTN, ...) bytes, 256-byte aligned; contents need not be kept.
 *                  Calls that may be in flight at the same time need a workspace each.
 * Supported: bf16, d in {64, 128}, scales of the pages 2^-100 .. 2^120, max_pages * P <= 2^30; scale, n_tok * Hq and values that
 * are no numbers as for prompt_attn_fwd.
 */
int paged_attn_fwd(const fastar_rows *Q, const int32_t *cu_q, const int32_t *len, const int32_t *table, int B, int max_pages,
                   int n_tok, int Hq, const fastar_pages *pages, int dtype, int causal, float scale, const fastar_rows *O,
                   float *lse, void *ws, size_t ws_bytes, void *stream);

/* ---- norm and rotation ---- */

/*
 * What is done to every row x [d] of queries and keys.
 *   Norm:      y_c = x_c w_c / sqrt(mean(x^2) + eps)
 *   Rotation:  of the first rot coordinates, in pairs (a, b) -> (a cos t - b sin t, a sin t + b cos t), t = position * freq[pair];
 *              the others stay as they are
 * All in 32 bits, angles in 64 before they are reduced to a turn, rounded once to the type of the output.
 */
typedef struct {
    const float *qw, *kw;   /* [d] weights of queries and of keys, or NULL: ones (device)                      */
    const double *freq;     /* [rot/2] radians per position (device)                                           */
    const int32_t *axis;    /* [rot/2] which row of `pos` a pair goes by (device), or NULL: row 0               */
    float eps;              /* >= 0                                                                            */
    int32_t norm;           /* 0: no norm (qw, kw and eps mean nothing);  1: as above                           */
    int32_t rot;            /* 0 .. d, a multiple of 16;  0: no rotation (freq and axis mean nothing)           */
    int32_t interleaved;    /* pair i is (i, i + rot/2);  1: (2i, 2i + 1)                                      */
    int32_t n_axes;         /* rows of `pos`, 1 .. 4                                                           */
} fastar_rope;

/*
 * Norm and rotation of packed queries and keys.
 *   Q, Qo [Hq,n_tok,d], K, Ko [Hkv,n_tok,d] views of dtype; either pair may be missing (Hq = 0 or Hkv = 0, pointers NULL).
 *   pos [n_axes, n_tok] int32 positions, negative ones too; an axis that is none goes as the nearest.  NULL: row i of the a rows
 *       of sequence b is at position len[b] - a + i on every axis (the last row is the sequence's last token).
 *   cu [B+1], len [B]: the sequences, where pos is NULL.  With pos: cu NULL (and B = 0): all rows;  otherwise rows outside of every
 *       sequence are not written, whatever they hold, and len may be NULL.
 * An output may be its input (the same address and strides); otherwise they share no memory.
 * Rows that hold infinities or NaN give what the formula gives, in that row alone; a row of zeros with eps = 0 is NaN.  Weights that are infinite or
 * NaN reach the coordinates that the formula brings them to, and no others.
 * Supported: d in {64, 128}; n_tok <= 2^30; n_tok times 1 .. (Hq + Hkv) * d / 512 wavefronts in 2^32 threads.  No workspace.
 */
int qk_norm_rope(const fastar_rows *Q, const fastar_rows *K, const int32_t *pos, const int32_t *cu, const int32_t *len, int B,
                 int n_tok, int Hq, int Hkv, int d, int dtype, const fastar_rope *rope, const fastar_rows *Qo, const fastar_rows *Ko,
                 void *stream);

/*
 * qk_norm_rope of Q into Qo and of the keys, and kv_pages_write of those keys and of V_new, without the keys between the two: they are
 * rounded once, from 32 bits to their codes (the two calls round them to dtype first).  Q and Qo may be missing (Hq = 0).
 * Arguments as for the two; slots of rows outside of every sequence (cu) are passed over whatever they say.  Supported as both.
 */
int kv_pages_write_rope(const fastar_pages *pages, const fastar_rows *Q, const fastar_rows *K_new, const fastar_rows *V_new, int dtype,
                        const int32_t *slot, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok, int Hq,
                        const fastar_rope *rope, const fastar_rows *Qo, void *stream);

/* ---- requests that share pages ---- */
/*
 * A page may be in several block tables: it is held as often as tables name it (their first ceil(len/P) entries; entries outside of
 * [0, n_pages) name nothing).  Only full pages come to be shared, and kv_pages_write writes behind a request's last token, so that
 * nobody writes to a page that others hold.  kv_pages_plan gives the pages of an ended request back whoever else holds them:
 * where requests share, they end by kv_pages_free.
 */

/*
 * Requests that begin with the tokens of another one.  Fork i: request child[i], which holds nothing, gets the first
 * m = min(keep[i], len[parent[i]]) tokens of request parent[i] (keep NULL: all; negative: none): its full pages by their numbers,
 * and, if m is no multiple of P, a page of its own from the pool, into which the page with the last of them is copied (all its codes
 * and scales).  An entry of the parent's table that names no page is taken over as it is.  The parents are those before the call.
 *   parent, child, keep [n];  len [B];  table [B, max_pages]: the children's rows are written up to ceil(m/P) entries
 *   pool [n_pages], pool_n [1]: as for kv_pages_plan; pages are taken from the top, in the order of the forks
 *   len_out [B]       tokens after the call; may be len itself
 *   pool_n_out [1]    free pages after it; may be pool_n itself
 *   status [n]        0;  1: it needs a page, and those needed up to and including it are more than there are;  2: parent or child is no
 *                     request, the child holds tokens, or an earlier fork of the call names the same child.  Refused forks change nothing.
 * Lengths and counts are cut to what the arrays hold.
 * Supported: n <= 1024; B * max_pages < 2^31; P and n_pages as for kv_pages_plan.  No workspace.
 */
int kv_pages_fork(const fastar_pages *pages, const int32_t *parent, const int32_t *child, const int32_t *keep, int n, const int32_t *len,
                  int32_t *table, int B, int max_pages, const int32_t *pool, const int32_t *pool_n, int32_t *len_out, int32_t *pool_n_out,
                  int32_t *status, void *stream);

/*
 * Requests that end or are cut back: request b keeps its first keep[b] tokens (none if negative, all if there are no more).  It gives up
 * the pages behind them; those that nobody holds any more go on top of the pool, in the order of the requests and of their
 * tables, each at the place of its last holder.  Cutting into a page that others hold is refused, as the next token would be written
 * to it (kv_pages_fork makes a request that may): by the tables before the call, whoever else gives the page up.
 *   keep, len [B];  table [B, max_pages] (not changed);  pool [n_pages], pool_n [1]: as for kv_pages_plan
 *   len_out [B]       tokens after the call; may be len itself
 *   pool_n_out [1]    free pages after it; may be pool_n itself
 *   status [B]        0, or 1: refused, the request keeps what it has
 *   ws / ws_bytes     fastar_workspace_bytes(FASTAR_OP_PAGES, B, max_pages, n_pages, P, ...) bytes, 256-byte aligned; contents need not be
 *                     kept.  Calls that may be in flight at the same time need a workspace each.
 * Lengths and counts are cut to what the arrays hold; pages beyond what the pool can hold are lost.
 * Supported: B * max_pages < 2^31; B * ceil(max_pages / 256) < 2^22; P and n_pages as for kv_pages_plan.
 */
int kv_pages_free(const int32_t *keep, const int32_t *len, const int32_t *table, int B, int max_pages, int32_t *pool, const int32_t *pool_n,
                  int n_pages, int P, int32_t *len_out, int32_t *pool_n_out, int32_t *status, void *ws, size_t ws_bytes, void *stream);

/*
 * Requests that thin out their caches: the tokens i < len[b] of request b with keep[b][i] != 0 that lie on pages become its tokens
 * 0, 1, .. in their order.  A new page whose tokens are all those that the request holds in one old page, at the same places, is that
 * page.  Any other is a fresh one from the pool, its scale per head the largest of its tokens' old ones, codes carried over to it (value of
 * the code times the old scale over the new one, rounded to nearest, ties to even), codes behind the last token zero.  Old
 * scales that are NaN (of pages that nothing was written to) are passed over as zeros; their tokens' codes become NaN.
 * Request b needs as many pages as it has fresh ones; they are taken from the top of the pool, in the order of the requests and of their
 * tables.  A request is refused, and keeps what it has (status 1), if it needs pages and those needed up to and including it are more than
 * there are.  Then the old pages that are not kept are given up as in kv_pages_free, on top of what is left.
 * A mask that keeps or drops whole pages (the last one as far as its tokens go) needs none: with an empty pool, cut at multiples of P.
 *   keep [B, max_pages * P] uint8, 16-byte aligned;  len [B];  table [B, max_pages];  pool [n_pages], pool_n [1]
 *   len_out [B]               tokens after the call;  may be len itself
 *   table_out [B, max_pages]  block tables after it, -1 behind a request's last page (rows of refused requests as they were);  may be table itself
 *   pool_out [n_pages]        the pool after it; entries that nothing was put into as they were;  may be pool itself
 *   pool_n_out [1]            free pages after it; may be pool_n itself
 *   status [B]                0 or 1
 *   ws / ws_bytes             as for kv_pages_free
 * Keys keep the positions that they were rotated by.  Lengths and counts are cut to what the arrays hold.
 * Supported: as for kv_pages_free, max_pages * P <= 2^30.
 */
int kv_pages_compact(const fastar_pages *pages, const uint8_t *keep, const int32_t *len, const int32_t *table, int B, int max_pages,
                     const int32_t *pool, const int32_t *pool_n, int32_t *len_out, int32_t *table_out, int32_t *pool_out, int32_t *pool_n_out,
                     int32_t *status, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FASTAR_H */
