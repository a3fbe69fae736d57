/*
 * libosdn -- OSDN hot path on one AMD MI355X (gfx950): the chunkwise-parallel gated
 * delta-rule recurrence whose write-side key is rescaled per feature by an online
 * diagonal preconditioner, forward and backward.
 *
 * What is computed (paper: "OSDN: Improving Delta Rule with Provable Online
 * Preconditioning in Linear Attention"), per batch b and head h independently, for
 * t = 1..T, with S in R^{V x K}, d in R^K:
 *
 *   phase 1 (Algorithm 1; Eq. (dt_update), with retention Eq. (dt_update_apf)):
 *       k~_t = d_t (.) k_t
 *       s = k_t (.) k_t,  n = max(sum s, eps),  p = <d_t, s>,  b' = beta_t (or 1 if !beta_aware)
 *       d_{t+1} = clip( r_t d_t + eta b' (1 - b' p)/n * s , d_min, d_max )
 *   phase 2 (Eq. (equiv_update)/(recurrent_form), gated as in Appendix B.1):
 *       S_t = alpha_t S_{t-1} + beta_t (v_t - alpha_t S_{t-1} k_t) k~_t^T ,  alpha_t = exp(log_alpha_t)
 *       o_t = scale * S_t q_t
 *
 * The library evaluates phase 2 in the chunkwise WY/UT form (Appendix A.2, B.1) with
 * chunk length 64; results equal the recurrence up to floating-point reassociation.
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers owned by the caller; tensors are contiguous,
 *     row-major, in the stated layout.  Inputs are never written; outputs must not alias
 *     inputs or each other.  Optional pointers may be NULL where stated.
 *   - q, k, v, o, dO, dq, dk, dv, k_tilde have element type params->io_dtype (fp32 or
 *     bf16).  beta, log_alpha, retention, every d and every S (and their gradients) are
 *     always fp32: the recurrent state and the preconditioner are kept in fp32.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls only
 *     enqueue work and return without synchronising.
 *   - Return value: OSDN_OK (0) or a negative osdn_status.  On an argument error nothing
 *     is launched.  osdn_strerror() gives a static description.
 *   - The library allocates no device memory: scratch comes from the caller's `workspace`
 *     (256-byte aligned, at least osdn_workspace_bytes()).  It reads no environment variables.
 *     Process-wide state: the optional profiling switch at the end of this file and, created on
 *     first use and kept until the process ends, one side stream with a few events per
 *     (device, caller stream): osdn_fwd / osdn_bwd run the preconditioner phase on it, forked
 *     from and joined back into `stream` with events, so that to the caller all work still is
 *     ordered as if enqueued on `stream` (also under stream capture: the side stream joins the
 *     capture and leaves it inside the call).  Calls on different streams share nothing; calls
 *     that share one stream must be issued one after the other, as any work on one stream.
 *     params->segments = 1 keeps everything on `stream`.
 *     With at most 32 (batch, head) chains of at least 24 chunks (64, if eta > 5e-5 K) osdn_fwd computes the
 *     preconditioner as a few sweeps over pieces of the sequence that run side by side, all on `stream`;
 *     osdn_bwd does so with a retention gate and eta <= 2.5e-4 K, beyond 16 chains up to 64 chunks, with fp32
 *     I/O and K = 128 beyond 8 chains up to 96.  params->p1_pieces = -1 keeps the one sequential sweep per
 *     chain.  d, k~ and the adjoint of d then agree with the sequential sweep's to the tolerance of the sweeps,
 *     1e-6 relative, and not bit for bit, and a call cut in two with (S, d) carried over agrees with the
 *     whole one no closer than that (below those lengths bit for bit).  What is made of d can differ by more: the
 *     projection decides for every coordinate whether it met the box, and where d comes within that tolerance of a
 *     face the decision, and with it the gradients that pass through it, may fall the other way; without a
 *     state gate and with bf16 I/O, S keeps every rounding of k~ that falls the other way (o and the gradients
 *     2e-3 in norm over 3000 tokens, as far from the exact values as the sequential sweep's).
 *   - retention values are assumed >= 0 (they are sigmoid gates in the paper).  Wherever a
 *     signature says retention / dretention [B,T,H], params->retention_per_channel = 1 makes
 *     it [B,T,H,K]: one value per coordinate.  Likewise params->gate_per_channel = 1 makes
 *     log_alpha / dlog_alpha [B,T,H,K]: one state gate per key channel, S <- S Diag(alpha_t)
 *     (online-scaled KDA, appendix section on Kimi Delta Attention with online scaling).
 *   - Supported shapes: chunk == 64; any T >= 1 (in a ragged last chunk, osdn_fwd/osdn_bwd
 *     treat the tokens that do not exist as ones that change nothing; osdn_precond_update needs
 *     T % 64 == 0 only when d_ckpt is asked for; 1 <= T <= 64 for osdn_step); K in {64, 128}
 *     (K = 256 is not built: the [64 x K] operand tiles of the chain and backward kernels would
 *     no longer fit the 160 KB of LDS next to each other); V a multiple of 64 up to 512; B, H >= 1 with H * max(K, V) < 2^24 (the 64 token rows of
 *     a chunk are addressed with 32-bit byte offsets).  Anything else returns OSDN_ERR_SHAPE.
 */
#ifndef OSDN_H
#define OSDN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { OSDN_F32 = 0, OSDN_BF16 = 1 } osdn_dtype;

typedef enum {
    OSDN_OK = 0,
    OSDN_ERR_NULL = -1,       /* a required pointer is NULL */
    OSDN_ERR_SHAPE = -2,      /* unsupported B/T/H/K/V/chunk */
    OSDN_ERR_DTYPE = -3,      /* io_dtype is neither OSDN_F32 nor OSDN_BF16 */
    OSDN_ERR_WORKSPACE = -4,  /* workspace too small or not 256-byte aligned */
    OSDN_ERR_PARAM = -5,      /* eta < 0, eps <= 0, or a non-finite scalar */
    OSDN_ERR_LAUNCH = -6      /* the HIP runtime reported a launch error */
} osdn_status;

typedef struct {
    int32_t B, T, H, K, V, chunk;   /* chunk must be 64 */
    int32_t io_dtype;               /* osdn_dtype */
    float scale;                    /* multiplies q in the read-out (Listing 1: K^-0.5) */
    float eta;                      /* online step size of the d update (paper: 0.003) */
    float d_min, d_max;             /* box of the projection (paper: 0.5, 2.0); d_min > d_max => none */
    float eps;                      /* floor of the squared key norm (Listing 1: 1e-6) */
    int32_t beta_aware;             /* 1: beta enters the d update (default); 0: replaced by 1 there */
    int32_t retention_per_channel;  /* 0: retention is one gate per (token, head), [B,T,H] (Section 4.4);
                                       1: one per coordinate, [B,T,H,K], diag(r_t) in place of r_t I (the
                                       vector-retention extension stated with the proposition that APF is a
                                       piecewise-affine recurrence); dretention then has that shape too */
    int32_t gate_per_channel;       /* 0: log_alpha is one state gate per (token, head), [B,T,H];
                                       1: one per key channel, [B,T,H,K]: S <- S Diag(alpha_t), the
                                       online-scaled KDA recurrence (appendix section on Kimi Delta
                                       Attention with online scaling; its K x V state is the transpose
                                       of the [V,K] state kept here); dlog_alpha then has that shape
                                       too and log_alpha must not be NULL.  In the chunkwise entry
                                       points the cumulative log-decay of a channel inside a chunk
                                       of 64 tokens has to stay above about -80 */
    /* Scheduling knobs; 0 everywhere = the library decides (what the benchmarks use).  They change
       how the work is cut, not what is computed (p1_pieces: to the sweeps' tolerance, see above). */
    int32_t segments;               /* > 0: cut the sequence into this many segments of chunks for the
                                       two-stream pipeline of osdn_fwd / osdn_bwd (1: one stream) */
    int32_t p1_pieces;              /* > 0: the preconditioner runs as sweeps over this many pieces per
                                       chain (osdn_bwd: with a retention gate, unless segments > 1 or it takes
                                       the solved form); -1: never (always the sequential sweep) */
    int32_t p1_piece_sweeps;        /* > 0: at most this many such sweeps (up to 13) before the sequential
                                       sweep finishes the chains that have not settled */
    int32_t p1_solved;              /* osdn_bwd: 1: the reverse sweep takes chunks in solved form (a 64 x 64
                                       triangular system per chunk, inverted for all chunks side by side):
                                       without retention the chunks in which no coordinate met the box, with
                                       one retention value per (token, head) every chunk; -1: never; 0: the
                                       library decides (only ever without retention) */
} osdn_params;

/* Bytes of scratch osdn_fwd needs (for_backward == 0) or osdn_fwd followed by osdn_bwd
 * needs (for_backward != 0).  Returns 0 if the parameters are invalid. */
size_t osdn_workspace_bytes(const osdn_params *p, int for_backward);

const char *osdn_strerror(int status);

/*
 * Phase 1 alone (Algorithm 1 / Eq. (dt_update_apf)); also the preconditioner half of a
 * streaming decode step (T may be 1).
 *   k         [B,T,H,K] io_dtype   keys (read side)
 *   beta      [B,T,H]   fp32
 *   retention [B,T,H]   fp32 or NULL (=> r = 1)
 *   d_in      [B,H,K]   fp32 or NULL (=> ones); not projected on entry
 *   k_tilde   [B,T,H,K] io_dtype   out: d_t (.) k_t, rounded once from fp32
 *   d_out     [B,H,K]   fp32       out: d after the last token
 *   d_ckpt    [B,H,T/64,K] fp32 or NULL   out: d at the start of every chunk (needs T % 64 == 0)
 */
int osdn_precond_update(const osdn_params *p, const void *k, const float *beta,
                        const float *retention, const float *d_in, void *k_tilde, float *d_out,
                        float *d_ckpt, void *stream);

/*
 * The same map as osdn_fwd in its recurrent form, for short inputs: the decode step of
 * Appendix K (state gate, rank-one write with the scaled key, read, then the preconditioner
 * update with its projection), token by token for 1 <= T <= 64 tokens in one launch, the state
 * in registers and fp32 throughout (k~ is not rounded to io_dtype here).  No workspace.
 *   q, k      [B,T,H,K] io_dtype ;  v [B,T,H,V] io_dtype
 *   beta      [B,T,H] fp32 ;  log_alpha, retention [B,T,H] fp32 or NULL
 *   d_in      [B,H,K] fp32 or NULL (=> ones) ;  S_in [B,H,V,K] fp32 or NULL (=> zeros)
 *   o         [B,T,H,V] io_dtype  out
 *   S_out     [B,H,V,K] fp32      out; MAY be the same buffer as S_in (updated in place)
 *   d_out     [B,H,K]   fp32      out; must NOT be d_in (OSDN_ERR_NULL if it is)
 * T > 64 returns OSDN_ERR_SHAPE (use osdn_fwd); params->chunk is still required to be 64.
 */
int osdn_step(const osdn_params *p, const void *q, const void *k, const void *v, const float *beta,
              const float *log_alpha, const float *retention, const float *d_in, const float *S_in,
              void *o, float *S_out, float *d_out, void *stream);

/*
 * Forward (both phases).
 *   q, k      [B,T,H,K] io_dtype ;  v [B,T,H,V] io_dtype
 *   beta      [B,T,H] fp32 ; log_alpha [B,T,H] fp32 (<= 0) or NULL (=> ungated, alpha = 1)
 *   retention, d_in as above ;  S_in [B,H,V,K] fp32 or NULL (=> zeros)
 *   o         [B,T,H,V] io_dtype  out
 *   S_out     [B,H,V,K] fp32      out: state after the last token
 *   d_out     [B,H,K]   fp32      out
 *   workspace: scratch; when osdn_bwd follows, pass the same buffer, untouched, to it.
 *     What only a backward pass reads (the chunks' (I + A)^-1 and intra-chunk scores) is written
 *     iff workspace_bytes >= osdn_workspace_bytes(p, 1); osdn_bwd rejects a smaller workspace, so a
 *     forward call that is to be followed by osdn_bwd must already be given the larger size.
 */
int osdn_fwd(const osdn_params *p, const void *q, const void *k, const void *v, const float *beta,
             const float *log_alpha, const float *retention, const float *d_in, const float *S_in,
             void *o, float *S_out, float *d_out, void *workspace, size_t workspace_bytes,
             void *stream);

/*
 * osdn_fwd for callers that cannot allocate device memory and have no workspace to hand in
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the
 * same computation with the scratch taken from a fixed device array that is part of the
 * library, OSDN_NOALLOC_MAX_WORKSPACE bytes, which every GPU the library is used on holds from
 * the moment the library is loaded until the process ends.  The call allocates nothing, creates
 * no stream or event, and runs entirely on `stream`; all other arguments are those of osdn_fwd.
 *   - Problems whose osdn_workspace_bytes(p, 0) exceeds OSDN_NOALLOC_MAX_WORKSPACE return
 *     OSDN_ERR_WORKSPACE and launch nothing; if the array's address cannot be obtained,
 *     OSDN_ERR_LAUNCH.
 *   - All calls on one GPU share that GPU's array: calls that may overlap in time (different
 *     streams, different threads) race on it and must be ordered by the caller.  Nothing in it
 *     has to start at zero (every buffer is written before it is read), so what the previous
 *     call left behind is harmless.
 *   - The scratch is not a workspace for osdn_bwd: use osdn_fwd with a caller workspace when a
 *     backward pass follows.
 */
#define OSDN_NOALLOC_MAX_WORKSPACE ((size_t)64 << 20)
int osdn_fwd_noalloc(const osdn_params *p, const void *q, const void *k, const void *v, const float *beta,
                     const float *log_alpha, const float *retention, const float *d_in, const float *S_in,
                     void *o, float *S_out, float *d_out, void *stream);

/*
 * Backward of osdn_fwd (Section 4.5: phase 2 yields dL/dk~; dL/dd_t = k_t (.) dL/dk~_t,
 * dL/dk_t += d_t (.) dL/dk~_t; reverse sweep through the projected affine d recurrence,
 * whose projection passes gradient where d_min <= unprojected value <= d_max).
 *   forward inputs exactly as given to osdn_fwd, and the workspace it filled
 *   dO        [B,T,H,V] io_dtype   gradient of o
 *   dS_out    [B,H,V,K] fp32 or NULL (=> 0)   gradient of S_out
 *   dd_out    [B,H,K]   fp32 or NULL (=> 0)   gradient of d_out
 *   dq, dk    [B,T,H,K] io_dtype out ; dv [B,T,H,V] io_dtype out
 *   dbeta     [B,T,H] fp32 out ; dlog_alpha [B,T,H] fp32 out (may be NULL iff log_alpha is)
 *   dretention [B,T,H] fp32 out (may be NULL iff retention is)
 *   dd_in     [B,H,K] fp32 out ; dS_in [B,H,V,K] fp32 out
 */
int osdn_bwd(const osdn_params *p, const void *q, const void *k, const void *v, const float *beta,
             const float *log_alpha, const float *retention, const float *d_in, const float *S_in,
             const void *dO, const float *dS_out, const float *dd_out, void *dq, void *dk, void *dv,
             float *dbeta, float *dlog_alpha, float *dretention, float *dd_in, float *dS_in,
             void *workspace, size_t workspace_bytes, void *stream);

/*
 * Packed sequences (the training set-up in the appendix on training and evaluation details,
 * paragraph on optimizer, batch and precision: one long token axis per device that holds
 * variable-length segments back to back, their boundaries in cu_seqlens, the recurrent state
 * reset at every boundary).  The _packed entry points are osdn_fwd / osdn_bwd for that input:
 *   params->B must be 1 and params->T the total number of tokens;
 *   cu_seqlens  HOST pointer to n_seqs + 1 ascending int32 token offsets, cu_seqlens[0] = 0,
 *               cu_seqlens[n_seqs] = T; sequence s is the tokens [cu_seqlens[s], cu_seqlens[s+1]);
 *               read before the call returns (it need not outlive the call); every sequence
 *               has at least one token, else OSDN_ERR_SHAPE;
 *   token tensors (q, k, v, beta, log_alpha, retention, o, dO and the token gradients) are
 *               [1,T,H,*] as before;
 *   carried tensors have one entry per sequence: d_in, d_out, dd_out, dd_in are [n_seqs,H,K];
 *               S_in, S_out, dS_out, dS_in are [n_seqs,H,V,K].  Every sequence starts from its own
 *               d_in / S_in entry (NULL => ones / zeros: the reset) and leaves its own final
 *               d and S; no state crosses a boundary.
 * Sequences need not be whole chunks: the token tensors are read and written where they are, and
 * inside the workspace each sequence starts on a chunk boundary.  The sequential kernels run one
 * chain per (sequence, head).
 * osdn_workspace_bytes_packed sizes the workspace for exactly this cu_seqlens (0 on invalid
 * arguments); osdn_bwd_packed takes the same cu_seqlens and the workspace osdn_fwd_packed filled.
 */
size_t osdn_workspace_bytes_packed(const osdn_params *p, const int32_t *cu_seqlens, int32_t n_seqs,
                                   int for_backward);

int osdn_fwd_packed(const osdn_params *p, const void *q, const void *k, const void *v, const float *beta,
                    const float *log_alpha, const float *retention, const float *d_in, const float *S_in,
                    void *o, float *S_out, float *d_out, const int32_t *cu_seqlens, int32_t n_seqs,
                    void *workspace, size_t workspace_bytes, void *stream);

int osdn_bwd_packed(const osdn_params *p, const void *q, const void *k, const void *v, const float *beta,
                    const float *log_alpha, const float *retention, const float *d_in, const float *S_in,
                    const void *dO, const float *dS_out, const float *dd_out, void *dq, void *dk, void *dv,
                    float *dbeta, float *dlog_alpha, float *dretention, float *dd_in, float *dS_in,
                    const int32_t *cu_seqlens, int32_t n_seqs, void *workspace, size_t workspace_bytes,
                    void *stream);

/*
 * Around the recurrence: the rows of queries, keys and values of a layer, each K adjacent elements of io_dtype (K in {64, 128, 256}),
 * wherever the caller has them (slices of one projection's output, views): element (b, t, h, i) stands
 * batch b + token t + head h + i elements behind data.  Rows need no more alignment than their elements; rows that start on 16
 * bytes are read and written in one piece.  No two rows that a call writes may overlap.  Within one output, or a cache that is appended
 * to, that is looked at, and the call refused unless the axes of more than one entry nest: taken from the smallest step on,
 * each step is at least the extent of those before it (so in every slice or reordering of an array).
 */
typedef struct { void *data; int64_t batch, token, head; } osdn_rows;

typedef enum { OSDN_NORM_NONE = 0, OSDN_NORM_RMS = 1, OSDN_NORM_L2 = 2 } osdn_norm;

typedef struct {
    int32_t B, T, Hq, Hk, K;        /* batch entries, tokens, heads of the queries and of the keys (and values), width */
    int32_t io_dtype;               /* osdn_dtype of the rows (and of a cache) */
    int32_t norm;                   /* osdn_norm: r = (sum x^2 / K + eps)^-1/2, (sum x^2 + eps)^-1/2, or 1 */
    int32_t rotary_dim;             /* elements that turn, from the front of a row: 0, or a multiple of 16 up to K */
    int32_t rotary_rows;            /* positions that the table has */
    int32_t interleaved;            /* pairs that turn: 0: (i, i + rotary_dim / 2); 1: (2i, 2i + 1) */
    float eps;                      /* > 0, finite (norm = NONE: not looked at) */
} osdn_norm_params;

/*
 * Norm of queries and keys for each head, with the position rotation in the same pass.  A row x becomes
 *     z = R(p) (w . x r),
 * R(p): pair i of the first rotary_dim elements turned by the angle whose cosine and sine are rotary[p][i] and
 * rotary[p][rotary_dim / 2 + i].  Computed in fp32, rounded once; a row of finite elements whose sum of squares passes what
 * fp32 holds becomes zeros, and so does its gradient.  (norm = L2 without weights or rotation is what osdn_fwd expects of its
 * caller's queries and keys.)
 *   q, k              [B,T,Hq,K], [B,T,Hk,K]; Hq or Hk may be 0, then its arguments are not looked at
 *   weight_q, weight_k [K] fp32 or NULL (=> ones)
 *   rotary            [rotary_rows, rotary_dim] fp32, NULL iff rotary_dim == 0
 *   positions         [B,T] int32 or NULL (=> t).  A negative position is a token that does not exist: its
 *                     outputs (and gradients) are zero.  A position that the table does not have makes them NaN.
 *   q_out, k_out      out; may be the input rows themselves (same pointer and strides)
 * At most 2^31 - 1 rows.
 */
int osdn_qk_norm_fwd(const osdn_norm_params *p, const osdn_rows *q, const osdn_rows *k, const float *weight_q,
                     const float *weight_k, const float *rotary, const int32_t *positions, const osdn_rows *q_out,
                     const osdn_rows *k_out, void *stream);

/*
 * Backward of osdn_qk_norm_fwd from its inputs (nothing is kept by the forward pass):
 *   dq_out, dk_out    gradients of q_out and k_out
 *   dq, dk            out; may be the rows of dq_out and dk_out, or of q and k, themselves
 *   dweight_q, dweight_k [K] fp32 out, summed over all tokens and heads in a fixed order; NULL where it is not wanted
 *   workspace         osdn_qk_norm_bwd_workspace_bytes(p) bytes, 256-byte aligned; may be NULL where neither dweight is wanted
 */
size_t osdn_qk_norm_bwd_workspace_bytes(const osdn_norm_params *p);
int osdn_qk_norm_bwd(const osdn_norm_params *p, const osdn_rows *q, const osdn_rows *k, const float *weight_q,
                     const float *weight_k, const float *rotary, const int32_t *positions, const osdn_rows *dq_out,
                     const osdn_rows *dk_out, const osdn_rows *dq, const osdn_rows *dk, float *dweight_q, float *dweight_k,
                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * A paged cache of keys and values: n_pages pages of page_size tokens (a power of two).  The row of page g, slot s, head h of the
 * keys starts k_page g + k_token s + k_head h elements behind k (likewise the values); rows start on 16 bytes.
 * Token i of sequence n stands in page table[n][i / page_size], slot i % page_size; table entries
 * outside [0, n_pages) are pages that are not there.
 */
typedef struct {
    void *k, *v;                                    /* io_dtype */
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
    const int32_t *table;                           /* [n_seqs, max_pages], rows table_stride entries apart */
    int64_t table_stride;
    int32_t n_pages, page_size, n_seqs, max_pages;
} osdn_cache;

/*
 * Append keys and values to a paged cache, and make the queries of the same tokens ready, in one pass: the row of a key is
 * treated as by osdn_qk_norm_fwd and written to its place in the cache, the row of a value is copied to its own, the
 * row of a query is treated as by osdn_qk_norm_fwd.
 *   q, q_out          [B,T,Hq,K]; both NULL iff Hq == 0; q_out may be q
 *   k, v              [B,T,Hk,K], Hk >= 1
 *   positions         [B,T] int32: place of the token in its sequence, also what it is rotated by.  Negative: no token,
 *                     nothing is appended and its query is zero
 *   seq               [B,T] int32 or NULL (=> the batch entry): the sequence (row of the table) that the token belongs to
 * A token whose sequence or page is not there is not appended.  Two tokens of one call must not have the same place (what it
 * then holds is undefined).  Nothing else in the cache is touched.
 */
int osdn_paged_append(const osdn_norm_params *p, const osdn_cache *cache, const osdn_rows *q, const osdn_rows *k, const osdn_rows *v,
                      const float *weight_q, const float *weight_k, const float *rotary, const int32_t *positions,
                      const int32_t *seq, const osdn_rows *q_out, void *stream);

typedef struct {
    int32_t B, Hq, Hk, K;           /* queries (one token each), their heads, heads of the cache (Hq a multiple of it), width */
    int32_t io_dtype;               /* osdn_dtype of q, o and the cache */
    int32_t window;                 /* > 0: only the last so many tokens are seen; 0: all */
    int32_t max_length;             /* no length is above it (the launch is sized by it) */
    int32_t shares;                 /* scheduling: > 0 (up to 65535): cut the tokens among so many workgroups; -1: no row is cut (a row: a
                                       sequence, a key head and up to 16 of its query heads), a workgroup takes one, two or
                                       four adjacent ones, as the library decides; 0: the library decides all of it */
    float scale;                    /* multiplies the scores (usually K^-1/2) */
} osdn_decode_params;

/*
 * Attention of one new token per sequence over a paged cache that holds it already.  Query head h reads head h Hk / Hq of the cache:
 *     s_j = scale <q, k_j> for max(0, length - window) <= j < length,  m = max_j s_j,
 *     lse = m + log sum_j e^(s_j - m),  o = sum_j e^(s_j - lse) v_j
 * in fp32; with bf16 I/O the weights e^(s_j - m) go into the product with the values as the sum of two bf16 numbers (2^-16 off at most).
 *   q, o              [B,Hq,K] (rows; token is not used); o may be q
 *   lengths           [B] int32, tokens of the sequence in the cache; 0 (or less): none, o is zero and lse minus infinity, whatever
 *                     stands for the sequence (a slot that nobody uses)
 *   seq               [B] int32 or NULL (=> b): row of the table.  Several queries may read one sequence, each
 *                     with its own length: drafted tokens, or a prompt token by token
 *   lse               [B,Hq] fp32 or NULL
 *   workspace         osdn_paged_decode_workspace_bytes(p) bytes (0 also for invalid parameters), 256-byte aligned; may be NULL if that is 0
 * B is at most 65535, B Hq below 2^21, and B Hk max_length / 64 (with more than 16 query heads a key head as many times that) below
 * 2^31.
 * What a length hides is not looked at, whatever the cache holds there.  A length above max_length or above what a row of the
 * table holds, a sequence or a page that is not there: o and lse are NaN, and nothing outside the cache is read.
 */
size_t osdn_paged_decode_workspace_bytes(const osdn_decode_params *p);
int osdn_paged_decode(const osdn_decode_params *p, const osdn_cache *cache, const osdn_rows *q, const int32_t *lengths,
                      const int32_t *seq, const osdn_rows *o, float *lse, void *workspace, size_t workspace_bytes,
                      void *stream);

/*
 * The pages of a cache from the lengths of requests, on the device: nothing of it has to be known to the host, and it may be
 * captured into a graph.  A list holds the pages that are not in use: entries [0, n_free) of free_list, taken from its end.
 */
typedef struct {
    int32_t *table;                 /* [n_seqs, max_pages], rows table_stride entries apart */
    int64_t table_stride;
    int32_t *free_list;             /* [free_capacity] page numbers */
    int32_t free_capacity;
    int32_t n_pages, page_size, n_seqs, max_pages;          /* as those of osdn_cache */
} osdn_pages;

/*
 * Places for the new tokens of B requests.  Request b brings fresh[b] tokens to sequence seq[b], which has cached[b]: it needs
 * ceil((cached + fresh) / page_size) - ceil(cached / page_size) more pages.  Requests are looked at in their order: one is served if it
 * needs no page or the needs up to it (served or not) are no more than the list holds, and if it brings no token or those up to it
 * are no more than `tokens`.  The i-th page that is granted is the i-th from the end of the list.
 *   cached, fresh     [B] int32
 *   seq               [B] int32 or NULL (=> b)
 *   n_free            [1] int32: how many pages the list holds;  n_free_out [1] int32 out: and how many it holds then (may be n_free)
 *   lengths           [B] int32 out: cached + fresh, or cached of a request that is not served (may be cached)
 *   starts            [B + 1] int32 out: where the request's tokens begin on the token axis, and their number last
 *   positions, rows   [tokens] int32 out: position and sequence of every token (-1 and -1 behind the last), as osdn_paged_append takes them
 *   slots             [tokens] int64 out or NULL: page * page_size + place in the page; -1 behind the last, and where the page is not there
 * Not served either, and without a part in the sums: a request whose sequence is not in the table, whose cached or fresh is negative or whose
 * tokens its row of the table or 31 bits do not hold; and those that bring tokens to a sequence that another one brings some too.
 * (lengths: 0 where the sequence is not in the table or cached is negative.)  B is at most 65535, tokens from 1 to 2^30;
 * with seq, n_seqs is at most 131072.
 */
int osdn_paged_plan(const osdn_pages *pages, int32_t B, int32_t tokens, const int32_t *cached, const int32_t *fresh, const int32_t *seq,
                    const int32_t *n_free, int32_t *n_free_out, int32_t *lengths, int32_t *starts, int32_t *positions, int32_t *rows,
                    int64_t *slots, void *stream);

/*
 * The pages of B sequences that end go back onto the list, and their entries of the table become -1: the first
 * ceil(lengths[b] / page_size) of row seq[b], those that are there.  They lie so that the next requests take them in the order that they
 * had.  A sequence that is named twice keeps its pages; a page that stands in two rows goes back with each of them (pages that sequences
 * share are the caller's to keep track of).  What the list has no room for is dropped.  Limits as for osdn_paged_plan, and
 * up to 1024 B as many times max_pages entries of the table at most 2^30.
 */
int osdn_paged_release(const osdn_pages *pages, int32_t B, const int32_t *lengths, const int32_t *seq, const int32_t *n_free,
                       int32_t *n_free_out, void *stream);

/*
 * A paged cache in 4 bits (the microscaling format with 4-bit floats): blocks of 32 adjacent elements of a row share a scale 2^e, kept
 * as the byte e + 127, and every element is a code of four bits: a sign (8) and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6.  The byte 255 makes all of a
 * block NaN; what fp32 does not hold is infinite (4 * 2^126 and more, which no append leaves).  A row is K / 2 bytes of codes, two to a
 * byte (the first in the lower bits), and K / 32 bytes of scales, which stand apart.  Steps are in bytes; rows of codes start on 16 bytes,
 * rows of scales, for K = 256, on 2.  The page table is as in osdn_cache.
 */
typedef struct {
    void *k, *v;                                    /* codes */
    uint8_t *k_scale, *v_scale;
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
    int64_t k_scale_page, k_scale_token, k_scale_head, v_scale_page, v_scale_token, v_scale_head;
    const int32_t *table;
    int64_t table_stride;
    int32_t n_pages, page_size, n_seqs, max_pages;
} osdn_cache_mx;

/*
 * osdn_paged_append for a cache in 4 bits.  e is the least, from -120 to 125, with the largest element of the block no more than 7 * 2^e
 * (a block without an element that is not zero: -120), the codes are the nearest values, ties to the even code; a block with an
 * infinity or a NaN is kept as NaN.  Keys are normed and rotated in 64 bits and not rounded before, so that a code does not hang on the order of a sum.
 * Queries are those of osdn_paged_append.
 */
int osdn_paged_append_mx(const osdn_norm_params *p, const osdn_cache_mx *cache, const osdn_rows *q, const osdn_rows *k, const osdn_rows *v,
                         const float *weight_q, const float *weight_k, const float *rotary, const int32_t *positions,
                         const int32_t *seq, const osdn_rows *q_out, void *stream);

/*
 * The rows that tokens have in a cache in 4 bits, as the values that they stand for (exact in both types of rows).
 *   p                 B, T, Hk, K and io_dtype are looked at
 *   positions, seq    as for osdn_paged_append; rows of a token that does not exist are zero, those of a sequence or page that is not there NaN
 *   k_out, v_out      [B,T,Hk,K] out
 */
int osdn_paged_read_mx(const osdn_norm_params *p, const osdn_cache_mx *cache, const int32_t *positions, const int32_t *seq,
                       const osdn_rows *k_out, const osdn_rows *v_out, void *stream);

/*
 * osdn_paged_decode over a cache in 4 bits: the same with the values that the codes stand for (io_dtype: of q and o).  Products are of bf16
 * numbers with fp32 sums: the cache's values are exact in bf16; with bf16 I/O weights are the sum of two such numbers, with fp32 I/O
 * queries and weights that of three, which hold all digits of a float.
 * How a call is cut, and whether codes are loaded past the caches, hangs on p->max_length, as lengths are not known to the host: a bound that is far above
 * them gives the same results in more time (512 sequences of 200 tokens, four heads: bounds of 200, 2048, 4096 and 131072 18.7, 18.8, 30.9 and 30.3 us).
 */
size_t osdn_paged_decode_mx_workspace_bytes(const osdn_decode_params *p);
int osdn_paged_decode_mx(const osdn_decode_params *p, const osdn_cache_mx *cache, const osdn_rows *q, const int32_t *lengths,
                         const int32_t *seq, const osdn_rows *o, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention over a few pages of a long cache, selected for each query and key head by a bound of their scores.
 */
typedef struct {
    int32_t B, Hq, Hk, K;           /* queries (bounds: sequences), their heads (bounds: not looked at), heads of the cache, width */
    int32_t io_dtype;               /* osdn_dtype of q, of the bounds, and of the cache unless that is in 4 bits */
    int32_t max_length;             /* select: no length is above it */
    int32_t max_new;                /* bounds: no sequence gets more new tokens (those beyond it are left out) */
    int32_t pages;                  /* select: pages for each key head, at most; at least first + last */
    int32_t first, last;            /* select: so many pages from the front (>= 0) and from the end (>= 1) are always among them */
} osdn_select_params;

/*
 * The smallest and the largest key of every page, for each head and element, kept up with what is appended: those of the pages that the
 * tokens cached[b] <= i < lengths[b] of sequence seq[b] stand in.  A page that had tokens before keeps their bounds, one that begins
 * with these tokens gets new ones.  NaN among the keys makes the element's bounds NaN.  B is at most 65535, B Hk at most 2^21, and that times the pages
 * that max_new tokens of a sequence may lie in (no more than max_pages) less than 2^31; the launch is sized by it.
 *   cache             the keys alone are looked at (v may be NULL)
 *   cached, lengths   [B] int32 (as osdn_paged_plan leaves them); nothing to do where cached >= lengths
 *   seq               [B] int32 or NULL (=> b).  No sequence twice
 *   bounds            [n_pages, Hk, 2, K] io_dtype, in and out, 16-byte aligned: the smallest, then the largest
 */
int osdn_page_bounds(const osdn_select_params *p, const osdn_cache *cache, const int32_t *cached, const int32_t *lengths,
                     const int32_t *seq, void *bounds, void *stream);
int osdn_page_bounds_mx(const osdn_select_params *p, const osdn_cache_mx *cache, const int32_t *cached, const int32_t *lengths,
                        const int32_t *seq, void *bounds, void *stream);

/*
 * The pages that a query reads.  For key head h and page g the score is sum over its query heads and the elements of
 *     max(q_i lo_i, q_i hi_i),
 * which no key of the page passes (computed in 64 bits, as sum of Q-_i lo_i + Q+_i hi_i, Q- and Q+ the sums over the query heads of min(q, 0) and
 * max(q, 0)).  Of the pages that the sequence has, the first `first`, the last `last` and those of the largest scores are chosen, p->pages in
 * all or as many as there are; equal scores: the earlier page.  A page that is not there, and one whose score is NaN, come before all
 * others; so does one with an infinite bound where its Q is zero.
 * B is at most 65535, B Hk at most 2^21, Hq at most 65535; p->pages and the pages of max_length tokens are at most 2^30 and, times B Hk, less than 2^31; p->pages
 * hold at most 2^31 - 256 tokens.  Who makes the scores hangs on max_length (64 sequences of 8192 tokens in pages of 16, one head of 64: bounds of 8192 and 131072 tokens 9.3
 * and 15.6 us).
 *   q                 [B,Hq,K] rows (token is not used)
 *   lengths, seq      as for osdn_paged_decode
 *   chosen            [B,Hk,pages] int32 out: page numbers in the order of their tokens, -1 behind the last (and for one that is not there)
 *   tokens            [B,Hk] int32 out: the tokens that they hold; 2^31 - 1 where osdn_paged_decode's results would be NaN
 *                     for the length or the sequence
 *   workspace         osdn_page_select_workspace_bytes(p) bytes, 256-byte aligned; may be NULL if that is 0
 */
size_t osdn_page_select_workspace_bytes(const osdn_select_params *p, int32_t page_size);
int osdn_page_select(const osdn_select_params *p, const osdn_pages *pages, const osdn_rows *q, const void *bounds, const int32_t *lengths,
                     const int32_t *seq, int32_t *chosen, int32_t *tokens, void *workspace, size_t workspace_bytes, void *stream);

/*
 * osdn_paged_decode over chosen pages: query head group h of entry b sees the first tokens[b][h] tokens of the pages chosen[b][h][...].
 *   p                 as for osdn_paged_decode; max_length: no entry of tokens is above it; window is 0; B Hk at most 65535
 *   cache             its table is not looked at
 *   chosen            [B,Hk,n_chosen] int32
 *   workspace         osdn_paged_decode_pages_workspace_bytes(p) (.._mx: of the cache in 4 bits) bytes
 */
size_t osdn_paged_decode_pages_workspace_bytes(const osdn_decode_params *p);
size_t osdn_paged_decode_pages_mx_workspace_bytes(const osdn_decode_params *p);
int osdn_paged_decode_pages(const osdn_decode_params *p, const osdn_cache *cache, const osdn_rows *q, const int32_t *chosen, int32_t n_chosen,
                            const int32_t *tokens, const osdn_rows *o, float *lse, void *workspace, size_t workspace_bytes, void *stream);
int osdn_paged_decode_pages_mx(const osdn_decode_params *p, const osdn_cache_mx *cache, const osdn_rows *q, const int32_t *chosen, int32_t n_chosen,
                               const int32_t *tokens, const osdn_rows *o, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Diagnostic query for tests: the decisions of the projection's derivative (Section 4.5,
 * reverse sweep through the projected affine recurrence) that osdn_bwd took, as it left them
 * in the workspace.  Returns the byte offset, inside a workspace of a plain (not packed) batch
 * that osdn_bwd has processed, of an array [B, H, ceil(T/64), K] of 64-bit words (low 32 bits
 * first): bit i of word (b, h, n, c) is set iff the unprojected update of coordinate c at
 * token 64 n + i landed inside the box [d_min, d_max], faces included.  Bits of tokens past T
 * are unspecified; with d_min > d_max (no projection) the array is not written.  Returns 0 for
 * invalid parameters.  Host-only: launches nothing.
 */
size_t osdn_debug_mask_offset(const osdn_params *p);

/*
 * Optional per-kernel timing (for benchmarks; off by default; not thread-safe -- this switch
 * and its event list are the only process-wide state of the library).  While enabled, every
 * kernel an entry point launches is bracketed by a pair of HIP events on the caller's stream.
 * osdn_profile_read() waits for the recorded events, returns for each kernel id the summed
 * duration in milliseconds and the number of launches since the previous read (arrays of
 * n >= osdn_profile_kernel_count() host elements), and forgets them.
 */
void osdn_profile_enable(int on);
int osdn_profile_kernel_count(void);
const char *osdn_profile_kernel_name(int id);
int osdn_profile_read(double *ms_sum, int *launches, int n);

#ifdef __cplusplus
}
#endif
#endif /* OSDN_H */
