/*
 * graphkv.h -- C ABI of the MI355X (gfx950) GraphKV eviction library.
 *
 * One call handles one transformer layer: the paper states the problem per
 * layer, with key/value matrices K^l, V^l of n x d and a layer budget k_l
 * (Methodology, "Problem Formulation").  The KV heads of the layer are
 * independent instances of that problem and are processed together.
 *
 * Conventions for every entry point
 *   - All tensor pointers are DEVICE pointers, contiguous, row-major with the
 *     head dimension innermost, 16-byte aligned.  The params struct and the
 *     returned strings live on the HOST.
 *   - The caller owns every buffer.  The library allocates nothing, never
 *     synchronises and never copies to the host.  It keeps no state between calls
 *     except which kernels have had their one-time opt-in to large shared memory
 *     (process-wide, guarded by a mutex: first calls may come from several host
 *     threads) and the measurement aid at the end of this header.
 *     All work is enqueued on `stream` (a hipStream_t passed as void*; NULL is
 *     the default stream).  Inputs are read-only unless stated otherwise.
 *   - `ws` is scratch memory of at least graphkv_workspace_bytes(params) bytes,
 *     256-byte aligned; its contents are undefined before and after a call.
 *     Two calls that overlap in time need two workspaces.  (graphkv_select does
 *     without, see there; graphkv_score_knorm uses none.)
 *   - Return value: GRAPHKV_OK (0) or a negative code.  Arguments are checked
 *     on the host before anything is enqueued: on GRAPHKV_EINVAL or
 *     GRAPHKV_EWORKSPACE nothing has run.  GRAPHKV_EHIP reports a failed
 *     launch (earlier launches of the same call may already be queued).
 *   - Results are deterministic: the same inputs give byte-identical outputs.
 *   - NaN inputs are not supported: selection order is then unspecified (every
 *     index written is still that of a token of the row).
 *
 * Symbols: N tokens in the layer's cache, of which the last w are the
 * observation window; P = N - w prefix tokens are the graph nodes; H_kv / H_q
 * key-value / query heads, G = H_q / H_kv; d head dimension; B retained tokens
 * per head (window included); S source nodes (k in Eq. 2); m neighbours per
 * source (Eq. 3); T propagation rounds (Eq. 5); alpha decay strength.
 */
#ifndef GRAPHKV_H
#define GRAPHKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    GRAPHKV_OK = 0,
    GRAPHKV_EINVAL = -1,      /* a constraint listed below is violated, or a required pointer is NULL/misaligned */
    GRAPHKV_EWORKSPACE = -2,  /* ws is NULL, misaligned or smaller than graphkv_workspace_bytes() */
    GRAPHKV_EHIP = -3,        /* a kernel launch failed */
    GRAPHKV_ESCRATCH = -4     /* graphkv_compress_static: the params need more scratch than its built-in buffer holds */
};

enum { GRAPHKV_FP32 = 0, GRAPHKV_BF16 = 1 };
enum { GRAPHKV_POOL_AVG = 0, GRAPHKV_POOL_MAX = 1 };
/* Signal sent to the neighbours of a source (Discussion, "Diversity of Graph
 * Signal"): decay multiplies by (1 - alpha e), enhanced by (1 + alpha e),
 * evicted sets the score to -infinity. */
enum { GRAPHKV_SIGNAL_DECAY = 0, GRAPHKV_SIGNAL_ENHANCED = 1, GRAPHKV_SIGNAL_EVICTED = 2 };
/* Kernel family: AUTO picks the bf16 MFMA kernels when the shape allows them
 * (bf16 and d = 128; for scoring also G*w at most 256, and w a multiple of 32 with
 * max pooling) and matrix-core kernels for any type and head dimension otherwise;
 * GENERIC forces the scalar kernels (same results up to fp32 rounding order). */
enum { GRAPHKV_IMPL_AUTO = 0, GRAPHKV_IMPL_GENERIC = 1 };
/* Which tensors the edges of the whole-pass calls are cosines of (Discussion,
 * "Exploration of similarity for Graph Edge"): e_ij = cos(x_i, y_j) with x the
 * source's row and y the other node's row.  KK is Eq. 1 (keys, keys); KV takes the
 * source's key and the other node's value; VV values on both sides.  Pairings
 * with queries need the prefix tokens' queries, which these calls do not
 * receive: graphkv_propagate_edges takes any two tensors. */
enum { GRAPHKV_EDGES_KK = 0, GRAPHKV_EDGES_KV = 1, GRAPHKV_EDGES_VV = 2 };
/* Indicator that initialises the node scores in the whole-pass calls ("Sparse Graph
 * Building", first paragraph: attention-based scores or KNorm): ATTENTION is
 * graphkv_score, KNORM is graphkv_score_knorm (the queries are not read). */
enum { GRAPHKV_SCORER_ATTENTION = 0, GRAPHKV_SCORER_KNORM = 1 };

typedef struct graphkv_params {
    int32_t n_kv_heads;    /* H_kv >= 1                                              */
    int32_t n_q_heads;     /* H_q, a multiple of H_kv (ignored by propagate/select)  */
    int32_t head_dim;      /* d, a multiple of 8, <= 512                             */
    int32_t n_tokens;      /* N, rows of Kc/Vc per head, window included             */
    int32_t window;        /* w >= 1, P = N - w >= 1                                 */
    int32_t pool_kernel;   /* odd, >= 1 (1 = no pooling)                             */
    int32_t pool_mode;     /* GRAPHKV_POOL_*                                         */
    int32_t budget;        /* B, w < B <= N (select/compress only)                   */
    int32_t n_sources;     /* S, 1 <= S <= min(P, 65535) when rounds > 0             */
    int32_t n_neighbors;   /* m, 1 <= m <= P - 1 when rounds > 0                     */
    int32_t rounds;        /* T >= 0                                                 */
    float   decay;         /* alpha in [0, 1]                                        */
    int32_t reselect;      /* 0: sources and neighbourhoods fixed from round 1
                              (Eq. 2 / Eq. 5 as printed); 1: re-picked from the
                              refined scores every round (Fig. 1's caption lets the
                              pick-and-propagate step run more than once)            */
    int32_t dtype;         /* GRAPHKV_FP32 / GRAPHKV_BF16: type of Kc, Vc, Qw        */
    float   softmax_scale; /* 0 selects 1/sqrt(d)                                    */
    int32_t signal;        /* GRAPHKV_SIGNAL_*                                       */
    int32_t impl;          /* GRAPHKV_IMPL_*                                         */
    int32_t edges;         /* GRAPHKV_EDGES_* (compress calls only)                  */
    int32_t scorer;        /* GRAPHKV_SCORER_* (compress calls only)                 */
} graphkv_params;

/* Bytes of scratch any of the calls below needs for these params (0 if the
 * params are invalid). */
size_t graphkv_workspace_bytes(const graphkv_params *p);

/*
 * Stage I, the initial importance score s^(0) of every prefix token.  The
 * paper leaves the indicator to a host method ("Sparse Graph Building", first
 * paragraph); this is the observation-window attention score of SnapKV:
 * logits <q_r, k_j> * scale for the w window queries of each query head, row r
 * (token P + r) seeing columns 0..P+r, softmax over the visible columns, summed
 * over the window rows for j < P, 1-D pooled per query head (stride 1,
 * length-preserving; average pads with zeros and divides by pool_kernel), then
 * averaged over the G query heads of each KV head.
 *   Kc     [H_kv, N, d]  in   keys
 *   Qw     [H_q, w, d]   in   window queries
 *   scores [H_kv, P]     out  fp32
 * The `scorer` field is ignored here (this call is the attention scorer); the
 * workspace must have the size graphkv_workspace_bytes() returns for the params
 * with scorer = GRAPHKV_SCORER_ATTENTION, else GRAPHKV_EWORKSPACE.
 */
int32_t graphkv_score(const graphkv_params *p, const void *Kc, const void *Qw,
                      float *scores, void *ws, size_t ws_bytes, void *stream);

/*
 * KNorm-style initial score, another indicator the paper plugs GraphKV into
 * (Baseline Methods, the key-norm method): scores[h, j] = -||k_j||, so that the
 * low-norm keys that method keeps rank highest.  The scores are negative: see
 * graphkv_propagate for what the signal does to them.
 */
int32_t graphkv_score_knorm(const graphkv_params *p, const void *Kc, float *scores,
                            void *ws, size_t ws_bytes, void *stream);

/*
 * Stages II and III, T rounds on any score array (plug-and-play: Introduction,
 * last paragraph before the contributions).  Per round and head: source nodes =
 * the S largest scores (Eq. 2, Alg. 1); edges e_ij = cosine of keys i and j
 * for every source i and prefix node j != i (Eq. 1); neighbourhood of i = its
 * m largest edges (Eq. 3); every score s_j is multiplied by the product of
 * (1 - alpha e_ij) over the sources whose neighbourhood holds j, factors taken
 * in ascending source index (Eq. 4, Eq. 5, Alg. 2).  Ties in either top-k go
 * to the lowest index; a zero-norm key has e = 0.  rounds = 0, or decay = 0
 * with a multiplicative signal, leaves scores untouched.
 * Scores of either sign: Eq. 4 / Eq. 5 are written for a non-negative indicator.
 * The signal acts on the magnitude of the score a round starts with, s_j' = s_j -
 * alpha e_ij |s_j| (Eq. 4), so that the decay lowers a negative score too, as
 * "Decay Signal Propagation" says it should (it reduces the scores of redundant
 * tokens); the factor of Eq. 5 is then (1 + alpha e_ij) for s_j < 0.  The enhanced
 * signal mirrors this.
 *   Kc      [H_kv, N, d]       in
 *   scores  [H_kv, P]          in/out  fp32
 *   dbg_src [T, H_kv, S]       out, optional (NULL): sources, ascending
 *   dbg_nbr [T, H_kv, S, m]    out, optional: neighbours of each source, ascending
 *   dbg_e   [T, H_kv, S, m]    out, optional: their edge weights, fp32
 * With reselect = 0 the rows of rounds 2..T repeat round 1.
 */
int32_t graphkv_propagate(const graphkv_params *p, const void *Kc, float *scores,
                          int32_t *dbg_src, int32_t *dbg_nbr, float *dbg_e,
                          void *ws, size_t ws_bytes, void *stream);

/*
 * The same rounds with edges e_ij = cosine of row i of Ac and row j of Bc: the
 * source's feature comes from the first tensor, the other node's from the second
 * (Discussion, "Exploration of similarity for Graph Edge": query-to-key,
 * query-to-query, key-to-value, value-to-value similarities as decay signals; the
 * paper gives no formula, this is the reading taken).  Ac = Bc = keys is
 * graphkv_propagate.
 *   Ac, Bc  [H_kv, N, d]  in  of type p->dtype; everything else as above
 */
int32_t graphkv_propagate_edges(const graphkv_params *p, const void *Ac, const void *Bc,
                                float *scores, int32_t *dbg_src, int32_t *dbg_nbr, float *dbg_e,
                                void *ws, size_t ws_bytes, void *stream);

/*
 * Stage IV, selection ("Decay Signal Propagation", closing paragraph: the k_l
 * tokens with the highest refined score are kept).  idx[h, 0..B-w) = the B - w
 * best prefix tokens in ascending order (ties to the lowest index), followed by
 * the window tokens P..N-1.
 *   scores [H_kv, P]  in   fp32
 *   idx    [H_kv, B]  out  int32
 * `ws` is optional and changes nothing but the time.  Few rows of more than 32768
 * entries are shared out to many workgroups where it is there, 256-byte aligned and
 * of at least graphkv_select_workspace_bytes() bytes (0: none is used; never more
 * than graphkv_workspace_bytes()); NULL, or a smaller or misaligned one, is no error:
 * a workgroup takes each row.  Used or not, calls that overlap in time must not share
 * one.
 */
size_t graphkv_select_workspace_bytes(const graphkv_params *p);
int32_t graphkv_select(const graphkv_params *p, const float *scores, int32_t *idx,
                       void *ws, size_t ws_bytes, void *stream);

/*
 * The whole pass for one layer: score -> propagate -> select -> gather of the
 * compressed sub-matrices K_s, V_s of k_l x d ("Problem Formulation").
 *   Kc, Vc     [H_kv, N, d]  in
 *   Qw         [H_q, w, d]   in
 *   Kout, Vout [H_kv, B, d]  out  rows idx[h, t] of Kc / Vc, byte copies
 *   idx        [H_kv, B]     out  int32
 *   scores_out [H_kv, P]     out, optional (NULL): refined scores s^(T), fp32
 * B = N gives the identity copy.  p->edges picks the tensors behind the edges,
 * p->scorer the indicator of stage I (with GRAPHKV_SCORER_KNORM Qw is not read and
 * may be NULL, and n_q_heads, pool_* and softmax_scale are ignored).
 */
int32_t graphkv_compress(const graphkv_params *p, const void *Kc, const void *Vc,
                         const void *Qw, void *Kout, void *Vout, int32_t *idx,
                         float *scores_out, void *ws, size_t ws_bytes, void *stream);

/*
 * The same pass for n_layers layers in one go.  The per-layer call keeps only H_kv
 * workgroups busy in its selection and update kernels and pays every launch per
 * layer; since all (layer, head) pairs are independent instances of the paper's
 * per-layer problem, a whole model can be pushed through each kernel at once
 * when its cache is one slab.
 *   Kc, Vc     [n_layers, H_kv, N, d]   in   contiguous
 *   Qw         [n_layers, H_q, w, d]    in
 *   budgets    HOST array [n_layers] of per-layer budgets B_l (w < B_l <= N), or
 *              NULL for p->budget everywhere (p->budget is ignored otherwise)
 *   Kout, Vout packed: layer l occupies rows [H_kv * sum_{l'<l} B_l', +H_kv * B_l),
 *              each layer laid out [H_kv, B_l, d]
 *   idx        packed the same way, [H_kv, B_l] per layer
 *   scores_out [n_layers, H_kv, P] or NULL
 *   ws         graphkv_workspace_bytes_batched(p, n_layers) bytes
 * Layers are processed in groups: at most 64 layers, fewer while the scratch
 * memory of a group would exceed 2000 MiB (long prompts).  Results are identical
 * to n_layers per-layer calls, byte for byte, with one exception: where
 * graphkv_uses_mfma() and G*w is a multiple of 32, a group of more than 2^19 keys
 * (layers * H_kv * N) sums its softmax rows in longer runs.  Its scores then agree
 * to the rounding of a 32-bit sum, and what is selected agrees unless two
 * candidates lie within that of each other.
 */
size_t graphkv_workspace_bytes_batched(const graphkv_params *p, int32_t n_layers);
int32_t graphkv_compress_batched(const graphkv_params *p, int32_t n_layers, const int32_t *budgets,
                                 const void *Kc, const void *Vc, const void *Qw, void *Kout,
                                 void *Vout, int32_t *idx, float *scores_out, void *ws,
                                 size_t ws_bytes, void *stream);

/*
 * graphkv_compress for callers that cannot allocate device memory or size a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that
 * forbid allocation.  Same arguments and results as graphkv_compress, without
 * `ws`: the scratch memory is a buffer of GRAPHKV_STATIC_SCRATCH_BYTES that
 * belongs to the library's code object (every GPU the library runs on holds its
 * own copy until the process ends).  The call allocates and frees nothing.
 *   - params that need more scratch than GRAPHKV_STATIC_SCRATCH_BYTES are rejected
 *     with GRAPHKV_ESCRATCH before anything is enqueued.  Whatever
 *     graphkv_workspace_bytes() puts within it is taken, and what it puts slightly
 *     above may be, by a slower way with less scratch and the same results;
 *   - every call on a GPU uses that GPU's one buffer: calls that overlap in time on
 *     one GPU (two streams, two host threads) race -- serialise them, or use
 *     graphkv_compress with a workspace each;
 *   - the first call on a device resolves the buffer's address and opts kernels in
 *     to large shared memory: make it outside a graph capture.
 */
#define GRAPHKV_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
int32_t graphkv_compress_static(const graphkv_params *p, const void *Kc, const void *Vc,
                                const void *Qw, void *Kout, void *Vout, int32_t *idx,
                                float *scores_out, void *stream);

/*
 * A paged cache, and attention over it.
 *
 * Where the calls above take a prompt's cache as one matrix a head, these keep the
 * rows of many sequences, evicted or whole, in the pages of a pool: what
 * graphkv_compress leaves is written to pages (graphkv_cache_write), the tokens that
 * are generated behind it are appended the same way, graphkv_attend computes the
 * attention of new tokens over what a sequence holds, and graphkv_cache_read lays
 * rows of a sequence out again, as graphkv_compress takes them.  One call handles one
 * layer.
 *
 *   pools     [n_pages, H_kv, page_tokens, d], one for keys and one for values: rows
 *             of p->dtype (GRAPHKV_PAGES_PLAIN) or 8-bit codes (see below)
 *   scales    [n_pages, H_kv, page_tokens] fp32, of the codes: a row's values are its
 *             codes times its scale (NULL with GRAPHKV_PAGES_PLAIN); with
 *             GRAPHKV_PAGES_*_BLOCKS [n_pages, H_kv, page_tokens / scale_tokens]
 *   table     [n_seqs, table_pages] int32: entry i of sequence s is the page that holds
 *             its positions i * page_tokens and on
 *   seq_len   [n_seqs] int32: tokens of a sequence, new ones included
 *   row_start [n_seqs + 1] int32, ascending: rows row_start[s] .. row_start[s+1]-1 of
 *             the row tensors (K, V, Q, out, lse) belong to sequence s and are its LAST
 *             tokens.  With n of them, row row_start[s] + i has position
 *             seq_len[s] - n + i.
 * table, seq_len and row_start are DEVICE arrays, read when the kernels run: a captured
 * graph serves batches whose lengths change from replay to replay (make the first call
 * with a set of params outside a capture: it opts kernels in to large shared memory).  Rows before
 * row_start[0] and from row_start[n_seqs] on belong to no sequence: none of their
 * outputs is written (a batch padded to a fixed number of rows).
 *
 * No content of these arrays makes a call touch memory outside the tensors.  Lengths
 * are cut to 0 .. table_pages * page_tokens, row numbers to 0 .. n_rows and to
 * max_rows a sequence.  A position whose page number is not one of 0 .. n_pages-1, and
 * a row whose position is negative (more rows than tokens), has no place: it is not
 * written, it reads as zeros, nothing sees it.  (Where row numbers do not ascend, a row that
 * several sequences would take gets what any of them gives it, or parts of each.)
 *
 * 8-bit forms keep a row of a head with one scale: the least power of two 2^k with
 * max|x| <= 448 * 2^k and codes in e4m3 (OCP, no infinities), or max|x| / 127 rounded
 * to 32 bits and integer codes; codes are the values nearest to x / scale, ties to the even
 * one.  Rows with max|x| < 2^-100 have scale and codes 0.  Infinities and NaN in rows
 * to be written are not supported with them; magnitudes beyond 1.9 * 2^127 may come back as
 * infinities, since the nearest code may stand for 2^128.
 *
 * GRAPHKV_PAGES_FP8_BLOCKS and GRAPHKV_PAGES_INT8_BLOCKS keep a scale for each block of
 * scale_tokens tokens of a head (positions that are next to one another, beginning at a multiple
 * of scale_tokens): the same scale and codes, with max|x| over all rows of a block.  A block
 * whose first token a call writes takes its scale from the rows of that call.  Rows that a call
 * adds behind tokens which a block holds already keep the block's scale if it is as large as theirs would be;
 * otherwise it becomes theirs, and the codes of the tokens before them become those nearest to code * old scale /
 * new scale (for e4m3 the least bits of small values go, for integers each such step adds at most half of one of the new scale).
 * A scale does not shrink while its block grows, not even where tokens that had asked for it were taken back.  (Pools filled by
 * other means: attention takes scales that are 0 or above, and codes that are 0 where the scale is.)
 */
enum { GRAPHKV_PAGES_PLAIN = 0, GRAPHKV_PAGES_FP8 = 1, GRAPHKV_PAGES_INT8 = 2,
       GRAPHKV_PAGES_FP8_BLOCKS = 5, GRAPHKV_PAGES_INT8_BLOCKS = 6 };

typedef struct graphkv_paged_params {
    int32_t n_kv_heads;    /* H_kv, 1 .. 65535                                           */
    int32_t n_q_heads;     /* H_q, a multiple of H_kv, <= 65535 (attend only)            */
    int32_t head_dim;      /* d, a multiple of 8 (16 with 8-bit pages), <= 512           */
    int32_t dtype;         /* GRAPHKV_FP32 / GRAPHKV_BF16: type of the rows K, V, Q, out */
    int32_t page_format;   /* GRAPHKV_PAGES_*                                            */
    int32_t page_tokens;   /* tokens a page holds, a power of two, <= 65536              */
    int32_t n_pages;       /* n_pages * H_kv * page_tokens < 2^31                        */
    int32_t n_seqs;        /* 0 .. 2^20                                                  */
    int32_t table_pages;   /* >= 1, table_pages * page_tokens <= 2^30                    */
    int32_t n_rows;        /* rows of the row tensors, 0 .. 2^24 - 1                     */
    int32_t max_rows;      /* no sequence has more rows than this; 0: n_rows.  Tell it:  */
                           /*   attend chooses its kernels by it (see there)             */
    float   softmax_scale; /* attend: 0 selects 1/sqrt(d), else in (0, 2^127]            */
    int32_t impl;          /* GRAPHKV_IMPL_*: GENERIC forces the scalar kernel (attend)  */
    int64_t row_stride;    /* elements between rows and between heads of K and V (write, */
    int64_t head_stride;   /*   read) or Q (attend); both 0: packed [n_rows, heads, d].  */
    int64_t out_row_stride;   /* the same for the output of attend.  Strides are         */
    int64_t out_head_stride;  /*   multiples of 16 bytes, <= 2^38; output rows must not overlap */
    int32_t scale_tokens;  /* with GRAPHKV_PAGES_*_BLOCKS: tokens that a scale belongs to, a */
                           /*   power of two, 16 .. page_tokens (not read with other formats) */
} graphkv_paged_params;

/*
 * Writes rows to the places of their tokens, encoded where the pages hold codes.
 *   K, V            [n_rows, H_kv, d] with the params' strides, in
 *   Kpages, Vpages  in/out: places of other tokens keep what they hold
 *   Kscale, Vscale  in/out, with 8-bit pages
 * No two rows of a call may have the same place (sequences that share pages must not
 * write to them): such a place would hold a mixture of their rows.
 */
int32_t graphkv_cache_write(const graphkv_paged_params *p, const void *K, const void *V, void *Kpages,
                            void *Vpages, float *Kscale, float *Vscale, const int32_t *table,
                            const int32_t *seq_len, const int32_t *row_start, void *stream);

/*
 * The reverse: K, V [n_rows, H_kv, d] (out, with the params' strides) get the rows' values,
 * rounded once to p->dtype.  Strides of n_rows * d between heads and d between rows
 * give the [H_kv, n_rows, d] of the calls above.
 */
int32_t graphkv_cache_read(const graphkv_paged_params *p, const void *Kpages, const void *Vpages,
                           const float *Kscale, const float *Vscale, const int32_t *table,
                           const int32_t *seq_len, const int32_t *row_start, void *K, void *V, void *stream);

/*
 * Causal attention of new tokens over the cache, which already holds their own rows:
 * a row at position t sees the positions 0 .. t of its sequence,
 *   out = sum_j softmax_j(<q, k_j> * scale) v_j,   lse = log sum_j exp(<q, k_j> * scale),
 * with query head i on key-value head i / (H_q / H_kv).  One token a sequence, a few
 * drafted ones, a chunk of a prompt, or a mixture of these in one call.
 *   Q    [n_rows, H_q, d] in, out [n_rows, H_q, d] out, with their strides; they must not
 *        overlap
 *   lse  [n_rows, H_q]    out, optional (NULL), fp32
 *   ws   graphkv_attend_workspace_bytes(p) bytes, 256-byte aligned
 * Sequences of few rows and of many have kernels of their own, and the host, which does not
 * know the lengths, goes by max_rows: a step of single tokens that leaves it 0 is planned as
 * one that may hold a chunk of n_rows, in blocks for many rows or with a launch that finds nothing.
 * Work is counted in 32 bits: where the matrix-core kernels run (AUTO, d up to 256 for bf16
 * and 128 for fp32), params are refused with n_rows * H_q / H_kv > 2^30, with n_rows * H_q + 192 *
 * n_seqs * H_kv >= 2^35, or, if some sequences may go to the kernel for few rows (max_rows * H_q / H_kv
 * <= 32, or 8 sequences and more), with n_seqs * H_kv * ceil(table_pages * page_tokens / 128) >= 2^31.
 * graphkv_attend_workspace_bytes() is 0 for params that are refused, and where no scratch
 * memory is needed: by the scalar kernel, and without rows or sequences.
 * Softmax statistics and sums are held in 32 bits.  With bf16 rows the weights (times the
 * values' scales, of 8-bit pages) are rounded to bf16 for the product with the values, where what is below 2^-126 may be
 * lost; where the kernel for few rows reads plain pages, to two bf16 numbers each, which keep 15 bits.  The sums of the softmax
 * are of the weights as they were before.  With fp32 rows none is rounded to fewer than 24 bits; over pages in blocks,
 * of queries, and of weights times scales, what is below 2^-126 may be lost (queries or values of less than 2^-70 have fewer than 24 bits then).  (Sums of values
 * beyond 2^100 may leave the range of 32 bits.)  A row that sees nothing, or
 * nothing but logits of -infinity, has out = 0 and lse = -infinity.  What lies in places that a row does not see (later
 * positions, the rest of a page) has no influence on it, whatever its bits.
 * Results are deterministic; a sequence's may differ in their last bits with the
 * sequences beside it, which change where its sums are cut.
 */
size_t graphkv_attend_workspace_bytes(const graphkv_paged_params *p);
int32_t graphkv_attend(const graphkv_paged_params *p, const void *Q, const void *Kpages, const void *Vpages,
                       const float *Kscale, const float *Vscale, const int32_t *table,
                       const int32_t *seq_len, const int32_t *row_start, void *out, float *lse, void *ws,
                       size_t ws_bytes, void *stream);

/*
 * Attention of rows over all that another sequence holds (a decoder's rows over an encoder's states, or over anything
 * that is no part of their own sequence): as graphkv_attend, but the rows of sequence s are no tokens of it, and each of
 * them sees all positions 0 .. seq_len[s] - 1.  A sequence may have more rows than tokens; where seq_len[s] is 0, or
 * none of its positions has a place, out = 0 and lse = -infinity.  The states are written once by graphkv_cache_write, in any page format.
 *   ws   graphkv_attend_workspace_bytes(p) bytes, 256-byte aligned
 */
int32_t graphkv_cross_attend(const graphkv_paged_params *p, const void *Q, const void *Kpages, const void *Vpages,
                             const float *Kscale, const float *Vscale, const int32_t *table, const int32_t *seq_len,
                             const int32_t *row_start, void *out, float *lse, void *ws, size_t ws_bytes, void *stream);

/*
 * What the calls above go by, made on the device: pages dealt to the sequences of a batch, their lengths and row
 * numbers, and the place of each row.  One call serves all layers of a model, whose pools share a table.
 *
 * Sequence s, with len_before[s] tokens (cut to 0 .. table_pages * page_tokens), keeps the first keep[s] of them (cut to
 * 0 .. that; keep = NULL: all) and gets new_rows[s] more (below 0: none).  It then needs more pages than it had, or fewer, and
 * the rest go back.  Free pages are a stack: free_pages[0 .. n - 1] are free, n = free_before[0] (cut to 0 .. n_pages).
 *   1. Refused are sequences with new_rows[s] > max_rows (n_rows if that is 0) or more tokens in the end than a table
 *      holds, and then, in ascending order, those whose new rows, with the new rows of all sequences before them that are not
 *      refused for these reasons, would be more than n_rows.
 *   2. The pages that other sequences have too many go on the stack, those of the last sequence first, of each the last page first.
 *   3. Sequences that need more pages take them from its top, in ascending order, for ascending entries of their table.  One that needs
 *      more than are left is refused, and so is every later one that needs any.
 * A refused sequence keeps its tokens and pages as they are and has no rows: seq_len[s] = len_before[s].  Others have
 * seq_len[s] = kept + new.  new_rows[s] > 0 with row_start[s + 1] = row_start[s] tells a refusal.
 *   seq_len     [n_seqs]              out, may be len_before
 *   table       [n_seqs, table_pages] in/out: entries of pages that a sequence gets are written, no others
 *   free_pages  [n_pages]             in/out
 *   free_after  [1]                   out: how many are free then; may be free_before
 *   row_start   [n_seqs + 1]          out: row_start[0] = 0, rows of refused sequences left out
 *   positions   [n_rows]              out, optional (NULL): position of each row in its sequence, -1 from row_start[n_seqs] on
 *   slots       [n_rows]              out, optional: page * page_tokens + place within it of each row, -1 likewise and
 *                                     where a table names no page
 *   ws          graphkv_assign_workspace_bytes(p) bytes, 256-byte aligned (0 up to 1024 sequences: it may be NULL)
 * No other arrays may overlap.  Of the params, page_tokens, n_pages, n_seqs, table_pages, n_rows and max_rows are used, and all are
 * checked.  A page belongs to one sequence or to the stack; where that is not so, pages may be lost or have two
 * owners, but nothing outside the arrays is touched.
 */
size_t graphkv_assign_workspace_bytes(const graphkv_paged_params *p);
int32_t graphkv_cache_assign(const graphkv_paged_params *p, const int32_t *keep, const int32_t *new_rows, const int32_t *len_before,
                             int32_t *seq_len, int32_t *table, int32_t *free_pages, const int32_t *free_before, int32_t *free_after,
                             int32_t *row_start, int32_t *positions, int32_t *slots, void *ws, size_t ws_bytes, void *stream);

/* Host string for a return code (static storage). */
const char *graphkv_strerror(int32_t code);

/*
 * Measurement aid (not part of the method): per-kernel timing with HIP events.
 * Between graphkv_profile_begin() and graphkv_profile_end() every kernel the
 * library launches is bracketed by two events on the caller's stream (the event
 * pool is created on first use and kept; process-wide: one recording at a time,
 * begin and end from one host thread).  graphkv_profile_end() waits for the
 * recorded events and adds up, per kernel id, the elapsed milliseconds into
 * ms[GRAPHKV_N_KERNELS] and the number of launches into launches[...] (HOST
 * arrays, either may be NULL).  The GENERIC ids count the scalar kernels and, with
 * GRAPHKV_IMPL_AUTO, the matrix-core kernels that take their place; an update of the
 * scores that the next selection does first is counted with that selection, and so is
 * the gather of few rows behind it; a later round's bound and filter in one launch count
 * as cosine_bound_new.  attend_many counts both kernels for many rows, that for blocks of
 * 256 and that for smaller ones.  graphkv_cross_attend is counted with graphkv_attend, graphkv_cache_assign with
 * cache_write.
 */
enum {
    GRAPHKV_K_SCORE_STATS = 0, GRAPHKV_K_SCORE_VOTES, GRAPHKV_K_POOL, GRAPHKV_K_TOPK_SOURCES,
    GRAPHKV_K_COSINE, GRAPHKV_K_TOPK_NEIGHBORS, GRAPHKV_K_DECAY, GRAPHKV_K_TOPK_FINAL,
    GRAPHKV_K_GATHER, GRAPHKV_K_GENERIC_LOGITS, GRAPHKV_K_GENERIC_VOTES, GRAPHKV_K_GENERIC_COSINE,
    GRAPHKV_K_KNORM, GRAPHKV_K_COPY, GRAPHKV_K_COSINE_BOUND,
    GRAPHKV_K_COSINE_FILTER, GRAPHKV_K_NBR_SELECT, GRAPHKV_K_REDO_ROWS,
    GRAPHKV_K_MATCH_SOURCES,
    /* later rounds when neighbour lists are kept: source selection, and the bound, filter and
     * select passes over the few sources that have no list yet */
    GRAPHKV_K_TOPK_SOURCES_LATER, GRAPHKV_K_COSINE_BOUND_NEW, GRAPHKV_K_COSINE_FILTER_NEW,
    GRAPHKV_K_NBR_SELECT_LATER,
    /* paged cache */
    GRAPHKV_K_CACHE_WRITE, GRAPHKV_K_CACHE_READ, GRAPHKV_K_ATTEND_GENERIC, GRAPHKV_K_ATTEND_FEW,
    GRAPHKV_K_ATTEND_MANY, GRAPHKV_K_ATTEND_JOIN, GRAPHKV_N_KERNELS
};
int32_t graphkv_profile_begin(void);
int32_t graphkv_profile_end(double *ms, int64_t *launches);
const char *graphkv_kernel_name(int32_t id);

/* 1 if AUTO would run the streaming bf16 kernels (d = 128) for scoring with these params, 0 otherwise. */
int32_t graphkv_uses_mfma(const graphkv_params *p);

#ifdef __cplusplus
}
#endif
#endif /* GRAPHKV_H */
