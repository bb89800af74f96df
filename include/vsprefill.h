/*
 * vsprefill.h - C ABI of the MI355X (gfx950) vertical-slash sparse-prefill library.
 *
 * The library implements the inference hot path of VSPrefill: VSIndexer scoring, the
 * cumulative-threshold budget with TopK, and causal vertical-slash sparse attention with the
 * per-query-tile index merge done inside the attention kernel, plus a dense causal attention
 * kernel on the same layout and the vertical-slash aggregation of the dense attention map (the
 * indexer's distillation target and the Attention Recall metric).  "Around the prefill" has what a serving
 * program needs beside it: norm and rotation of a projection's rows, a paged 4-bit cache of keys and values,
 * and the attention of single tokens and short chunks over that cache.
 *
 * Conventions shared by every call
 *   - Every tensor pointer is a DEVICE pointer owned by the caller, contiguous, 16-byte
 *     aligned.  The library never allocates or frees device memory: scratch space is a caller
 *     workspace whose size comes from the matching *_workspace() query (0 bytes is possible;
 *     then ws may be NULL).  Structs (vs_indexer_t, vs_budget_t) live in HOST memory and are
 *     read during the call; the float arrays a vs_indexer_t points to are device memory.
 *   - bf16 tensors are [heads, n, 128] row-major (head_dim is fixed at 128).
 *   - GQA: query head h reads KV head h / (q_heads / kv_heads).
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls enqueue
 *     work and return without synchronising; outputs are valid once the stream has run.
 *   - Return value: VS_OK (0) or a negative vs_status.  Argument checks happen on the host
 *     before anything is launched.  Data-dependent conditions (selection larger than the
 *     capacity, NaN scores) never abort: they are flagged in a device status word.
 *   - Calls on the same workspace must not overlap in time.
 */
#ifndef VSPREFILL_H
#define VSPREFILL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    VS_OK = 0,
    VS_ERR_INVALID_ARG = -1, /* null / misaligned pointer, non-positive size, tau outside [0,1] ... */
    VS_ERR_UNSUPPORTED = -2, /* q_heads % kv_heads != 0, d_h not a multiple of 64 or > 1024, n > 2^20 ... */
    VS_ERR_WORKSPACE = -3,   /* ws_bytes smaller than the *_workspace() answer, or ws NULL when bytes are needed */
    VS_ERR_CAPACITY = -4,    /* forced entries alone exceed cap_v / cap_s, or caps <= 0 */
    VS_ERR_HIP = -5,         /* a HIP call failed; vs_last_hip_error() has the hipError_t */
    VS_ERR_STATIC_LIMIT = -6 /* vs_sparse_prefill_static: the call needs more scratch than the library's fixed array holds */
} vs_status;

#define VS_HEAD_DIM 128
#define VS_MAX_SEQ (1 << 20)

/* bits of the per-head device status word written by vs_select_budget */
#define VS_STATUS_OVERFLOW 1  /* selection exceeded the capacity and was truncated by rank */
#define VS_STATUS_BAD_SCORE 2 /* a NaN or negative score was treated as 0 */
#define VS_STATUS_SATURATED 4 /* a score above 1 was given the mass of 1 */

/*
 * Rotary embedding, in place (Appendix, "RoPE Matrix Representation": block-diagonal 2x2
 * rotations, plane p turns by position * theta_base^(-2p/128)).  Input preparation for Q and K.
 *   x        [heads, n, 128] bf16, rotated in place; row r is position pos0 + r
 *   pairing  0: plane p couples elements (2p, 2p+1) (the appendix matrix); 1: (p, p+64)
 * Angles and the rotation are evaluated in fp64 and rounded once to bf16 (nearest even).
 */
int vs_rope_apply(void* x_bf16, int heads, int64_t n, int64_t pos0, double theta_base, int pairing,
                  void* stream);

/*
 * VSIndexer weights (Sec. "VSIndexer Design": Z = act(concat(K, V) W_U + b_U), one logit per
 * direction from W_V / W_S).  One set per layer, shared by all KV heads.  The struct is host
 * memory; the arrays are fp32 device memory.
 */
typedef struct {
    const float* W_U; /* [256, d_h] row-major: rows 0..127 multiply K, rows 128..255 multiply V */
    const float* b_U; /* [d_h] */
    const float* W_V; /* [d_h] vertical down-projection */
    const float* W_S; /* [d_h] slash down-projection */
    float b_V, b_S;   /* scalar output biases (they cancel in the softmax over positions) */
    int d_h;          /* hidden width: multiple of 64, 64..1024 */
    int act;          /* 0 = SiLU, 1 = GELU (erf form) */
} vs_indexer_t;

size_t vs_index_score_workspace(int kv_heads, int64_t n, int d_h);

/*
 * VSIndexer forward (Sec. "VSIndexer Design", Eqs. X, Z, A_v, A_s).
 *   k, v      [kv_heads, n, 128] bf16; k already carries RoPE
 *   a_v, a_s  [kv_heads, n] fp32 out: softmax over the n positions of each head.  a_v[g, j] is
 *             the score of key column j; a_s[g, t] is the score of slash offset o = t.
 * Arithmetic: bf16 inputs times W_U split into two bf16 terms on the matrix cores, fp32
 * accumulation, fp32 activation / down-projection / softmax.
 */
int vs_index_score(const void* k_bf16, const void* v_bf16, int kv_heads, int64_t n, const vs_indexer_t* w,
                   float* a_v, float* a_s, void* ws, size_t ws_bytes, void* stream);

/*
 * Budget rule (Sec. "Adaptive Sparse Index Selection", Eqs. k_d and I_d), host struct.
 *   mode 0  cumulative threshold: per head and direction, the fewest top-ranked scores whose
 *           mass reaches tau_d of the total mass.  Masses are integers, floor(score * 2^40), so
 *           the result does not depend on summation order; rank is (score descending, index
 *           ascending).  The threshold is ceil(tau * total) evaluated in fp64.
 *   mode 1  fixed k_v / k_s with the same ranking.
 * After the rule, columns 0..n_sink-1 and offsets 0..max(n_local,1)-1 are added (offset 0, the
 * diagonal, is always present) and each list is emitted in ascending order.  If a list would
 * exceed its capacity the forced entries stay, the best-ranked others fill the rest and
 * VS_STATUS_OVERFLOW is set for that head.
 */
typedef struct {
    int mode;
    double tau_v, tau_s;
    int k_v, k_s;
    int n_sink;
    int n_local;
    int cap_v, cap_s;
} vs_budget_t;

/* Bytes of device workspace with which vs_select_budget spreads every (head, direction) problem over many
 * workgroups; 0 for lengths short enough for one workgroup per problem (n < 32768).  Contents need no initialisation. */
size_t vs_select_budget_workspace(int heads, int64_t n);

/*
 *   a_v, a_s      [heads, n] fp32 scores (finite, in [0,1] expected; see status bits)
 *   idx_v, idx_s  [heads, cap_v] / [heads, cap_s] int32 out, ascending, first cnt entries valid
 *   cnt_v, cnt_s  [heads] int32 out
 *   status        [heads] int32 out (bit-or of VS_STATUS_* over both directions) or NULL
 *   ws, ws_bytes  device workspace of at least vs_select_budget_workspace() bytes (16-byte aligned), or NULL / 0: the
 *                 call then uses one workgroup per problem (same results; about three times slower at 128k).  A
 *                 non-NULL workspace that is too small is VS_ERR_WORKSPACE.
 */
int vs_select_budget(const float* a_v, const float* a_s, int heads, int64_t n, const vs_budget_t* b,
                     int32_t* idx_v, int32_t* cnt_v, int32_t* idx_s, int32_t* cnt_s, int32_t* status,
                     void* ws, size_t ws_bytes, void* stream);

size_t vs_sparse_prefill_workspace(int q_heads, int kv_heads, int index_heads, int64_t n);

/*
 * Causal vertical-slash sparse attention (Sec. "Sparse Attention Formulation", Eqs. M_S and
 * A-hat, with the mask of Sec. "Linear-Complexity Mask Construction"; kernel behaviour of Sec.
 * "Fused attention kernel implementation": indices are read per query tile, merged on the fly,
 * keys fetched on demand).  Row i of query head h attends to
 *     { j : 0 <= j <= i  and  ( j in I_v  or  i - j in I_s ) },   each key once,
 * with softmax(scale * q.k) renormalised over that set.  A row with no key gives zeros and
 * lse = -inf.
 *   q            [q_heads, n, 128] bf16;  k, v  [kv_heads, n, 128] bf16
 *   idx_v/cnt_v  [index_heads, cap_v] / [index_heads] selected key columns
 *   idx_s/cnt_s  [index_heads, cap_s] / [index_heads] selected diagonal offsets (0 = diagonal)
 *                Lists must be strictly ascending with entries in [0, n); out-of-range entries
 *                are ignored, other violations are undefined.
 *   index_heads  kv_heads (one mask per KV group, the paper's setting) or q_heads
 *   o            [q_heads, n, 128] bf16 out;  lse [q_heads, n] fp32 out or NULL
 * Arithmetic: bf16 MFMA for QK^T and PV, fp32 accumulation and softmax, P rounded to bf16.
 */
int vs_sparse_prefill(const void* q, const void* k, const void* v, int q_heads, int kv_heads, int64_t n,
                      float scale, const int32_t* idx_v, const int32_t* cnt_v, int cap_v,
                      const int32_t* idx_s, const int32_t* cnt_s, int cap_s, int index_heads,
                      void* o_bf16, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Tile-granular slash variant of vs_sparse_prefill (Sec. "Fused attention kernel implementation": the merged index
 * set is built per query block).  slash_granularity g groups the query rows in aligned blocks of g rows; row i keeps
 *     { j : 0 <= j <= i  and  ( j in I_v  or  i' - j in I_s for SOME row i' of the block of i ) },
 * a superset of the element-exact mask (g = 1, identical to vs_sparse_prefill).  Supported: g = 1 and g = 32.
 * All other arguments, the workspace and the error behaviour are those of vs_sparse_prefill; an unsupported g
 * returns VS_ERR_UNSUPPORTED.
 */
int vs_sparse_prefill_tiled(const void* q, const void* k, const void* v, int q_heads, int kv_heads, int64_t n,
                            float scale, const int32_t* idx_v, const int32_t* cnt_v, int cap_v,
                            const int32_t* idx_s, const int32_t* cnt_s, int cap_s, int index_heads,
                            int slash_granularity, void* o_bf16, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Chunked prefill (Sec. "Efficient VS Sparse Attention Inference": the same per-layer pipeline, applied to a block of
 * new query positions against all keys so far).  vs_sparse_prefill_tiled for n_q query rows that are the positions
 * pos0 .. pos0 + n_q - 1 of a sequence whose keys 0 .. n_kv - 1 are present:
 *   q, o   [q_heads, n_q, 128];  k, v  [kv_heads, n_kv, 128];  lse [q_heads, n_q];  pos0 + n_q <= n_kv
 *   (the keys behind the chunk, pos0 + n_q .. n_kv - 1, are not read: the unfilled end of a cache may hold anything)
 * The mask speaks of absolute positions: the query at position i keeps key j iff j <= i and (j in I_v or i - j in I_s);
 * lists hold columns and offsets in [0, n_kv).  Running the chunks of a sequence one after the other gives, row for
 * row, the results of one call on the whole sequence (up to the order of summation).  pos0 may be any position for
 * slash_granularity 1; granularity 32 groups positions in aligned blocks of 32 and needs pos0 % 32 == 0
 * (VS_ERR_UNSUPPORTED otherwise).  Workspace: vs_sparse_prefill_workspace(q_heads, kv_heads, index_heads, n_kv).
 *
 * Batches: a batch of B sequences of equal length is B * q_heads query heads and B * kv_heads KV heads in the same
 * layout ([B, heads, n, 128] contiguous), with one index list per (sequence, index head); every call of this library
 * accepts that directly because head h always reads KV head h / (q_heads / kv_heads).  Which kernel runs a call follows from
 * its sizes (heads, rows, keys, list capacities), so the last bits of a head's result may differ between a call on one
 * sequence and the same heads inside a batch; the same attention call always gives the same bits.
 */
int vs_sparse_prefill_chunk(const void* q, const void* k, const void* v, int q_heads, int kv_heads, int64_t n_q,
                            int64_t n_kv, int64_t pos0, float scale, const int32_t* idx_v, const int32_t* cnt_v,
                            int cap_v, const int32_t* idx_s, const int32_t* cnt_s, int cap_s, int index_heads,
                            int slash_granularity, void* o_bf16, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Debug check of index lists before they are given to vs_sparse_prefill / vs_aggregate (whose behaviour is undefined for
 * lists that are not strictly ascending).  One report word per head, written on the device:
 * 0 = usable, else a bit-or of the VS_LIST_* flags.  Out-of-range entries alone are legal input (they are ignored).
 *   idx [heads, cap] int32, cnt [heads] int32, report [heads] int32 out (all device memory)
 */
#define VS_LIST_BAD_COUNT 1     /* cnt < 0 or cnt > cap */
#define VS_LIST_OUT_OF_RANGE 2  /* an entry < 0 or >= n */
#define VS_LIST_NOT_ASCENDING 4 /* an entry not larger than its predecessor (unsorted or duplicate) */
int vs_validate_lists(const int32_t* idx, const int32_t* cnt, int cap, int heads, int64_t n, int32_t* report, void* stream);

/*
 * vs_sparse_prefill for callers that cannot allocate or pass a workspace: code under HIP graph capture, tight serving
 * loops, harnesses that forbid allocation.  Same arguments, results and error behaviour as vs_sparse_prefill, but the
 * scratch (bitmaps, diagonal lists, counters) lives in an array of VS_STATIC_SCRATCH_BYTES that the library holds on
 * every GPU it runs on until the process ends; the call allocates nothing and frees nothing.
 *   - A call whose vs_sparse_prefill_workspace() exceeds VS_STATIC_SCRATCH_BYTES returns VS_ERR_STATIC_LIMIT before
 *     anything is launched (32 / 8 heads with one mask per KV head fit up to n = 262144; n = 2^20 fits with one or two
 *     index heads).
 *   - All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two streams, two threads)
 *     race.  Calls that follow each other on one stream are safe; every call rewrites what it reads.
 */
#define VS_STATIC_SCRATCH_BYTES (4u << 20)
int vs_sparse_prefill_static(const void* q, const void* k, const void* v, int q_heads, int kv_heads, int64_t n,
                             float scale, const int32_t* idx_v, const int32_t* cnt_v, int cap_v,
                             const int32_t* idx_s, const int32_t* cnt_s, int cap_s, int index_heads,
                             void* o_bf16, float* lse, void* stream);

/*
 * Dense causal attention on the same layout (Sec. "Attention Computation", Eqs. P, A, O, with
 * j <= i): the in-library full-attention baseline.  Same kernel pipeline as the sparse call.
 */
int vs_dense_prefill(const void* q, const void* k, const void* v, int q_heads, int kv_heads, int64_t n,
                     float scale, void* o_bf16, float* lse, void* stream);

/* The same for a chunk of n_q query rows at positions pos0 .. pos0 + n_q - 1 against n_kv keys (layouts as for
 * vs_sparse_prefill_chunk). */
int vs_dense_prefill_chunk(const void* q, const void* k, const void* v, int q_heads, int kv_heads, int64_t n_q,
                           int64_t n_kv, int64_t pos0, float scale, void* o_bf16, float* lse, void* stream);

size_t vs_aggregate_workspace(int q_heads, int kv_heads, int index_heads, int64_t n);

/*
 * Vertical-slash aggregation of the dense causal attention map (Sec. "Vertical-Slash Aggregation for Distillation
 * Training", paragraph "Obtaining Ground Truth": A = softmax(Q K^T / sqrt(d)) summed along columns and along diagonals,
 * both divided by n) and, optionally, the Attention Recall of a vertical-slash mask (Sec. "Sparse Attention
 * Formulation", Eq. R(S)).  A is never stored: it is recomputed tile by tile from Q, K and the row normalisers.
 *   q           [q_heads, n, 128] bf16;  k  [kv_heads, n, 128] bf16 (both already carry RoPE)
 *   lse         [q_heads, n] fp32 natural-log row normalisers as written by vs_dense_prefill for the same q, k and
 *               scale, or NULL: then a first sweep over the scores computes them into the workspace
 *   out_heads   q_heads: one pair of vectors per query head;  kv_heads: the mean over the query heads of each KV group
 *   a_v, a_s    [out_heads, n] fp32 out.  a_v[., j] = (1/n) sum_i A[i, j];  a_s[., o] = (1/n) sum_i A[i, i - o].
 *               Each row sums to 1.  Accumulated with atomics: the last bits depend on the order of execution.
 *   recall      [out_heads] fp32 out or NULL.  When given, idx_v / cnt_v / cap_v / idx_s / cnt_s / cap_s / index_heads
 *               describe the mask as for vs_sparse_prefill (element-exact rule) and
 *               recall[.] = (1/n) sum over kept (i, j), j <= i, of A[i, j].  When NULL the list arguments are ignored.
 * Arithmetic: bf16 MFMA for Q K^T with fp32 accumulation, fp32 exponentials and sums.
 * Workspace from vs_aggregate_workspace (index_heads = 0 when no recall is wanted); errors as for the other calls.  Per query head
 * and position a call needs 4 bytes, and up to 1024 groups of 256 positions (q_heads x ceil(n / 256), n > 256) 20 and 8 for each of
 * the workgroups that then share a group's work, 10 MB at most; the answer for n is enough for shorter sequences of the same heads, too.
 */
int vs_aggregate(const void* q, const void* k, int q_heads, int kv_heads, int64_t n, float scale, const float* lse,
                 int out_heads, float* a_v, float* a_s, const int32_t* idx_v, const int32_t* cnt_v, int cap_v,
                 const int32_t* idx_s, const int32_t* cnt_s, int cap_s, int index_heads, float* recall, void* ws,
                 size_t ws_bytes, void* stream);

size_t vs_index_train_workspace(int kv_heads, int64_t n, int d_h);

/*
 * One distillation step of the VSIndexer without the optimizer (Sec. "Vertical-Slash Aggregation for Distillation
 * Training", paragraph "Loss function design"): forward as vs_index_score, then
 *     L = (1 / kv_heads) * sum over heads of [ KL(A^_v || A_v) + KL(A^_s || A_s) ],
 *     KL(P || Q) = sum_t P_t (ln P_t - ln max(Q_t, eps))            (prediction first, as the paper prints it)
 * and the gradient of L with respect to W_U, b_U, W_V, W_S (the scalar output biases cancel in the softmax: their
 * gradient is zero).  Only the indexer is differentiated; K, V and the targets are constants (frozen backbone).
 *   k, v        [kv_heads, n, 128] bf16 as for vs_index_score
 *   t_v, t_s    [kv_heads, n] fp32 target distributions, e.g. vs_aggregate's a_v / a_s with out_heads = kv_heads
 *   eps         floor of the targets inside the logarithm (> 0)
 *   loss        [1] fp32 out (device);  dW_U [256, d_h], db_U, dW_V, dW_S [d_h] fp32 out (device, overwritten)
 * Arithmetic: the inference kernels for the forward; fp64 sums for the loss; the hidden activations are recomputed on
 * the matrix cores (W_U as two bf16 terms), pre-activation gradients enter the second contraction as two bf16 terms,
 * fp32 partial sums over at most 1/256 of the tokens (or 256 tokens) that are added in fp64 in a fixed order: the step is
 * deterministic.
 */
int vs_index_train_step(const void* k_bf16, const void* v_bf16, int kv_heads, int64_t n, const vs_indexer_t* w,
                        const float* t_v, const float* t_s, float eps, float* loss, float* dW_U, float* db_U,
                        float* dW_V, float* dW_S, void* ws, size_t ws_bytes, void* stream);

/*
 * Number of MFMA tiles the last vs_sparse_prefill that used this workspace executed.  One tile is
 * (32 query rows of one head) x (32 keys): 1024 score elements, 4 * 128 * 1024 flop.  The kernel
 * counts them itself (tiles it skipped as fully masked are not counted).  Synchronises `stream`,
 * then copies the counter to the HOST integer `executed_tiles_host`.
 */
int vs_sparse_prefill_tiles(const void* ws, size_t ws_bytes, void* stream, int64_t* executed_tiles_host);

/*
 * The three counters of the last vs_sparse_prefill that used this workspace, copied to the HOST array counters_host[3]
 * after synchronising `stream`: [0] executed MFMA tiles (as vs_sparse_prefill_tiles), [1] 32-key tiles staged in LDS by
 * row gathers of selected columns (each is 32 rows of K and of V, 256 bytes per row: 16 KiB), [2] 32-key tiles staged
 * as contiguous key blocks of the slash part.
 * ws, ws_bytes: that workspace (at least 256 bytes).  VS_ERR_INVALID_ARG where it is plain that no sparse call has written it,
 * VS_ERR_WORKSPACE for the copy of a workspace that ends before its counters.
 */
int vs_sparse_prefill_counters(const void* ws, size_t ws_bytes, void* stream, int64_t* counters_host);

/*
 * ---- Around the prefill: from a layer's projection to the calls above, and single tokens after the prompt ----
 *
 * One convention holds for the calls below: `lens` [batch] int32 (device) is the number of tokens that each sequence
 * holds, the new ones among them, and a call's `rows` (or n_q) rows of a sequence are its LAST tokens: row r is position
 * lens[b] - rows + r.  One array serves a whole decoding step; a slot with lens 0 is idle; a batch of prompts of different
 * lengths is padded in front (rows of negative position have no token).  So only a sequence that holds no more than `rows` tokens can have fewer new ones than the
 * others: in one that holds more, all rows are tokens, and vs_cache_write writes them all, vs_cache_weigh adds the queries of them all.  Sequences that go on by
 * different numbers of tokens take a call for each number.  `lens` and page tables may begin at any element of an array (4-byte alignment).
 */

/* Rows of 128 bf16 elements: head h of token t at data + t * token_stride + h * head_stride (strides in elements, multiples of 8,
 * at least 128; data 16-byte aligned).  A part of a packed projection [tokens, heads, 128] as well as [heads, tokens, 128]. */
typedef struct {
    const void* data;
    int64_t token_stride, head_stride;
} vs_rows_t;

/* Rotation of the first rot_dim elements of a head (a multiple of 8, 8..128); the others keep their values.  Host struct. */
typedef struct {
    const double* freq; /* [rot_dim / 2] device: angle in radians per position of every plane (vs_rope_frequencies or any other) */
    int rot_dim;
    int pairing;        /* 0: plane p couples elements (2p, 2p+1);  1: (p, p + rot_dim / 2) */
    float magnitude;    /* factor of the rotated elements, 1 for a pure rotation */
} vs_rotation_t;

/*
 * The frequencies theta_base^(-2p / rot_dim), p < rot_dim / 2, scaled for contexts longer than the model was trained on, into HOST
 * memory (the caller copies them to the device once).
 *   scaling  0: as they are (the other arguments are ignored)
 *            1: divided by factor (positions shrunk)
 *            2: by wavelength.  A plane turns `original` * f / (2 pi) times over the original context: with `low` turns or fewer it
 *               is divided by factor, with `high` or more it is kept, in between the two are mixed linearly in the turns.
 */
int vs_rope_frequencies(double theta_base, int rot_dim, int scaling, double factor, double low, double high, double original,
                        double* freq_host);

/*
 * Norm of queries and keys per head and rotary embedding in one pass, with the change of layout from a projection's output:
 *     y = x * w / sqrt(mean(x^2) + eps)  over the 128 elements of a head (w_q / w_k [128] fp32, or NULL: y = x),
 *     planes (a, b) of y -> magnitude * (a cos t - b sin t, a sin t + b cos t),  t = position * freq[plane].
 *   q, k, v     batch * rows tokens (sequence after sequence) of q_heads / kv_heads heads; v may be NULL (then v_out, too); v is copied
 *   lens, pos0  row r of sequence b is position lens[b] - rows + r, or pos0 + r where lens is NULL (rows of negative position are
 *               computed like the others)
 *   q_out [batch, q_heads, rows, 128], k_out, v_out [batch, kv_heads, rows, 128] bf16.  An output may be its own input where both
 *               have the same layout; otherwise they must not overlap.
 *   eps         FLT_MIN .. 1 (ignored without w_q and w_k);  pos0 + rows at most 2^31
 *   rows        at most 2^20, batch at most 65535, batch * rows at most 2^26, heads at most 4096 (VS_ERR_UNSUPPORTED beyond)
 * Arithmetic: angles reduced in fp64, sine, cosine, norm and rotation in fp32, one rounding to bf16: before it within 2^-19 of magnitude
 * (|a| + |b|) where |position * freq| < 2^31 (freq <= 1 at every position; larger angles lose 3 * 2^-53 of themselves more).
 */
int vs_qk_norm_rope(const vs_rows_t* q, const vs_rows_t* k, const vs_rows_t* v, int batch, int64_t rows, int q_heads, int kv_heads,
                    const float* w_q, const float* w_k, float eps, const vs_rotation_t* rotation, const int32_t* lens, int64_t pos0,
                    void* q_out, void* k_out, void* v_out, void* stream);

/*
 * Paged cache of keys and values in 4 bits.  An element is held as an E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), 32 channels of
 * a token share a scale 2^(E - 127), E one byte: 136 bytes per token and head for K and V together, against 512 in bf16.  The
 * scale is the smallest power of two s with max |x| <= 7 s (2 <= E <= 252; a group of zeros has E = 0), the code the number nearest to
 * x / s, ties to the even one, 6 beyond 6.  A group with a NaN or an infinity in it is held as NaN (E = 255).
 * Memory is divided in pages of page_size tokens (a multiple of 64), each [kv_heads, page_size / 64] blocks of VS_CACHE_BLOCK_BYTES.
 * A page that is taken into use need not be cleared.  Host struct.
 */
#define VS_CACHE_BLOCK 64
#define VS_CACHE_BLOCK_BYTES 8704
typedef struct {
    void* data;           /* [pages, kv_heads, page_size / 64, VS_CACHE_BLOCK_BYTES] device */
    int64_t pages;
    int kv_heads;
    int page_size;
    const int32_t* table; /* [batch, max_pages] device: page number of tokens i * page_size .. of sequence b; NULL: b * max_pages + i */
    int max_pages;
} vs_cache_t;

/* Bytes of `data`; 0 for sizes that name no cache, 2^64 less a page (more than any memory) where the product passes 64 bits.  The calls
 * take pages < 2^31, kv_heads <= 4096, page_size <= VS_MAX_SEQ, batch * kv_heads <= 65535 and caches of less than 2^63 bytes; others are
 * VS_ERR_UNSUPPORTED. */
size_t vs_cache_bytes(int64_t pages, int kv_heads, int page_size);

/*
 * Shared by the calls on a cache:
 *   lens   [batch] int32 (device), values outside [0, max_n] count as the nearer end; NULL: every sequence holds max_n tokens
 *   max_n  bound of lens that the host knows, at most max_pages * page_size
 * Entries of the table that name no page (outside [0, pages)) are legal: their tokens are not written, not read and not attended to.
 * Sequences may share pages that are only read; no page may be written for two sequences in one call, nor for two parts of one.
 *
 * Writes the last `rows` tokens of each sequence; rows of negative position are skipped and all other tokens keep what they hold.
 *   k, v  [batch, kv_heads, rows, 128] bf16 (k carries RoPE)
 */
int vs_cache_write(const vs_cache_t* cache, const void* k, const void* v, int batch, int64_t rows, const int32_t* lens, int64_t max_n,
                   void* stream);

/*
 * Reads the last `rows` tokens of each sequence back (exactly what the cache holds); rows of negative position and of missing pages are left
 * as they were.  With lens = NULL, max_n = the end and rows = its distance from the beginning it reads any range, for instance all keys
 * in front of a chunk for vs_sparse_prefill_chunk.
 *   k, v  [batch, kv_heads, rows, 128] bf16 out; one of the two may be NULL
 */
int vs_cache_read(const vs_cache_t* cache, int batch, int64_t rows, const int32_t* lens, int64_t max_n, void* k, void* v, void* stream);

/*
 * Attention of the last n_q tokens (1 .. VS_CACHE_MAX_NEW) of each sequence over the cache, which already holds them:
 *     o[b, h, r] = sum_j softmax_j(scale * q[b, h, r] . K_j) V_j  over  j <= lens[b] - n_q + r.
 *   q, o  [batch, q_heads, n_q, 128] bf16 (not overlapping);  lse [batch, q_heads, n_q] fp32 out or NULL
 * A row without a key (negative position, idle slot, missing pages only) gives zeros and lse = -inf.  Longer chunks: vs_cache_prefill, or vs_cache_read and then
 * vs_sparse_prefill_chunk.
 * Arithmetic: K and V are exact in bf16; bf16 MFMA, fp32 accumulation and softmax, P as two bf16 terms (2^-15 of a weight; the output's own
 * rounding is 2^-8).  The same call always gives the same bits.  A key whose weight is below 2^-126 of the row's largest counts as zero, and one whose weight
 * times V is far below the others' may lose up to 2^-107 (in the units of V).
 * A score has to lie within fp32's range, and so do sums of V times weights of up to 2^8 (they do for |V| < 2^96).
 * At most 4096 query heads and 2^24 - 1 rows in a call (batch * q_heads * n_q).  Workspace: vs_cache_attend_workspace; the answer for max_n is enough for every smaller max_n of the same call.
 */
#define VS_CACHE_MAX_NEW 128
size_t vs_cache_attend_workspace(int batch, int q_heads, int kv_heads, int n_q, int64_t max_n);

int vs_cache_attend(const void* q, const vs_cache_t* cache, int batch, int q_heads, int n_q, const int32_t* lens, int64_t max_n,
                    float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * The same attention for any number of new tokens (1 .. VS_MAX_SEQ), a chunk of a prompt for instance; sequences of a batch may differ in length, prompts
 * shorter than n_q are padded in front.  Layouts, masks, rows without a key (zeros, lse = -inf) and missing pages as for vs_cache_attend, whose kernels take
 * up to VS_CACHE_MAX_NEW rows, within its limits, where there is little work (by batch, q_heads, n_q and max_n, not by lens).
 * Arithmetic otherwise: K is exact in bf16; V in fp16 in units of the largest scale so far of its 32 channels, and 64 tokens with one below 2^-27 of that or not finite
 * among them in bf16, exact too; P in fp16, 11 significant bits down to 2^-21 of the row's largest weight and steps of 2^-31 of it below, where vs_cache_attend's kernels have 15
 * bits of every weight (the output's own rounding is 2^-8; which of the two a call of up to VS_CACHE_MAX_NEW rows has goes by its sizes, as above); fp32 accumulation and
 * softmax.  The same call always gives the same bits.
 * So a key whose weight is below 2^-32 of the row's largest counts as zero in the output; V below 2^-126 of the largest of its 32 channels, too.  Scores have to lie
 * within fp32's range, and V within 2^96.  At most 4096 query heads.  Workspace: vs_cache_prefill_workspace; the answer for max_n is enough for every smaller
 * max_n of the same call.
 */
size_t vs_cache_prefill_workspace(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n);

int vs_cache_prefill(const void* q, const vs_cache_t* cache, int batch, int q_heads, int64_t n_q, const int32_t* lens, int64_t max_n,
                     float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * The weight that each held token gets from the last n_q tokens' queries (1 .. VS_MAX_SEQ), added to what it had:
 *     weights[b, g, j] = decay * old[b, g, j] + sum over the query heads h of KV head g and the rows r that see j, j <= lens[b] - n_q + r, of
 *                        exp(scale * q[b, h, r] . K_j - lse[b, h, r])
 * for j < lens[b]; entries behind stay as they are.  The last `fresh` tokens have no weight yet: what `old` holds for them is not read
 * (fresh = n_q in a decoding step or a chunk, whose own tokens are the new ones; max_n or old = NULL to begin anew).
 *   q       [batch, q_heads, n_q, 128] bf16;  lse [batch, q_heads, n_q] fp32, as vs_cache_attend or vs_cache_prefill left it for the same rows
 *   old     [batch, kv_heads, stride] fp32 or NULL (zeros); may be `weights`, must not overlap it otherwise
 *   decay   0 .. 1; with 0 `old` is not read
 *   weights [batch, kv_heads, stride] fp32 out, stride >= max_n
 * A row without a key (lse = -inf; padding in front of a prompt, too) adds nothing.  A token of a missing page gets nothing and keeps decay * old.  scale * log2(e) has to be a normal fp32 number.
 * Arithmetic: K is exact in bf16; bf16 MFMA, fp32 exponentials and sums in a fixed order: the same call always gives the same bits.  lse may be of any size; it is
 * taken as it is, and what its own rounding to fp32 left out (128 and more from 2^31 on) is missing in the exponents.
 * At most 4096 query heads and 2^30 - 1 rows of a KV head (q_heads / kv_heads * n_q).  Workspace: vs_cache_weigh_workspace; the answer for max_n is enough for every smaller max_n of the same call.
 */
size_t vs_cache_weigh_workspace(int batch, int q_heads, int kv_heads, int64_t n_q, int64_t max_n);

int vs_cache_weigh(const void* q, const float* lse, const vs_cache_t* cache, int batch, int q_heads, int64_t n_q, const int32_t* lens,
                   int64_t max_n, float scale, const float* old, float decay, int64_t fresh, float* weights, int64_t stride, void* ws,
                   size_t ws_bytes, void* stream);

/*
 * Eviction: of each sequence and KV head `keep` tokens stay, in their order, as the tokens 0 .. of the same cache or of another one.  The first n_sink
 * and the last n_recent stay in any case, then those with the largest weights, of equal ones the first (NaN is below every number, the two zeros are
 * equal).  Tokens of missing pages do not stay: min(keep, tokens that are there) tokens of every head remain, all of them where that is no more than keep.
 * Codes and scales are moved as they are.  Positions are baked into K: tokens that come later are rotated by their own position (lens of
 * vs_qk_norm_rope: tokens seen), not by their place in the cache (lens of the calls on the cache: tokens held).
 *   weights      [batch, kv_heads, stride] fp32, stride >= max_n, e.g. vs_cache_weigh's
 *   keep         1 .. VS_MAX_SEQ, at most to->max_pages * page_size;  n_sink + n_recent <= keep
 *   to           where the tokens go (kv_heads as in `cache`, any page size); NULL: the same cache.  Its pages that take tokens must belong to one sequence only,
 *                and where `to` is another cache in the same memory not to `cache`'s sequences.  Tokens whose page is missing in `to` are lost; what
 *                `to` holds behind the last token stays.
 *   weights_out  [batch, kv_heads, stride_out] fp32 out: weights of the tokens that stay, stride_out >= keep; NULL, or `weights` with the same stride
 *   kept         [batch, kv_heads, keep] int32 out or NULL: their numbers, ascending, -1 behind them
 *   lens_out     [batch] int32 out: tokens that each sequence then holds; may be `lens`
 * Workspace: vs_cache_evict_workspace.
 */
size_t vs_cache_evict_workspace(int batch, int kv_heads, int64_t max_n, int64_t keep);

int vs_cache_evict(const vs_cache_t* cache, const float* weights, int64_t stride, int batch, const int32_t* lens, int64_t max_n, int64_t keep,
                   int64_t n_sink, int64_t n_recent, const vs_cache_t* to, float* weights_out, int64_t stride_out, int32_t* kept,
                   int32_t* lens_out, void* ws, size_t ws_bytes, void* stream);

const char* vs_strerror(int status);
int vs_last_hip_error(void);
const char* vs_version(void);

#ifdef __cplusplus
}
#endif
#endif /* VSPREFILL_H */
