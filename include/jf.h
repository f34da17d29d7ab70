/*
 * jf.h -- C ABI of libjf, a Jacobi-step engine for causal decoders on
 * AMD Instinct MI355X (gfx950).
 *
 * One call of jf_jacobi_step / jf_multiblock_step is ONE Jacobi iteration
 * (Jacobi Forcing, arXiv 2512.14681, Sec. 2.1, Eq. 3): a single forward pass
 * of the decoder over the draft rows, causal against an exact KV cache of the
 * committed prefix, a greedy argmax over the vocabulary for every row, and
 * acceptance of the longest prefix of draft rows that reached their fixed
 * point (Sec. 3.2; the acceptance step of App. A Alg. 1).
 * jf_commit_kv then keeps the accepted rows' K/V and drops the rest (the
 * cache-trim step of Alg. 1).
 *
 * Conventions
 *  - Pointers named d_* are DEVICE pointers; everything else is host memory.
 *  - The caller owns every buffer: weights, the packed-weight buffer, the KV
 *    cache, the workspace and all outputs.  libjf owns only the opaque host
 *    object jf_model, and never allocates device memory.
 *  - Device buffers need the alignment of what they hold: of their elements,
 *    and 8 bytes for the workspaces (64-bit words).  Weights, workspaces and
 *    activations that start on 16-byte boundaries, as every allocator returns
 *    them, are read faster in bf16 steps of 10 rows and more.
 *  - Every call validates its arguments on the host before enqueuing any
 *    work.  On error it returns a negative jf_status, enqueues nothing and
 *    sets jf_last_error() (thread-local).  No exception crosses the ABI and
 *    the library never aborts.  HIP runtime failures return JF_E_HIP with the
 *    HIP error string in jf_last_error().
 *  - Step and commit calls only enqueue work on `stream` (a hipStream_t).
 *    The committed length C lives on the device, so step -> commit -> step
 *    needs no host round trip.  Conditions that only the device can see
 *    (a token id outside [0, V)) are reported in jf_step_result.flags.
 *    The host keeps an upper bound of C (it grows by the rows of each
 *    committed step); a step that would pass max_ctx by that bound first
 *    reads C back (one stream synchronisation) and fails with JF_E_CAPACITY
 *    only if the exact length leaves no room.
 *  - One jf_model decodes one sequence (batch 1).  Calls on one model must
 *    not overlap (one stream, or external ordering).
 */
#ifndef JF_H
#define JF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  JF_OK = 0,
  JF_E_INVAL = -1,    /* null pointer, bad enum, bad value             */
  JF_E_SHAPE = -2,    /* shape not supported (see jf_config)           */
  JF_E_CAPACITY = -3, /* rows > max_rows, or C + rows > max_ctx        */
  JF_E_DTYPE = -4,    /* unsupported dtype                             */
  JF_E_HIP = -5,      /* HIP runtime error                             */
  JF_E_STATE = -6     /* call not valid in the model's current state   */
} jf_status;

/* JF_E4M3 (OCP 8-bit floating point, largest value 448) is a type of the paged
 * caches of jf_kv_append / jf_kv_read / jf_attention_kv8 only. */
typedef enum { JF_F32 = 0, JF_BF16 = 1, JF_E4M3 = 2 } jf_dtype;

/* Decoder shape: RMSNorm (gain), RoPE (rotate-half pairs i, i + head_dim/2,
 * inverse frequency rope_base^(-2i/head_dim)), grouped-query attention with
 * query head j reading KV head j / (n_heads / n_kv_heads), SwiGLU FFN,
 * untied LM head, no biases.
 * Limits: d_model, d_ffn multiples of 128, d_model <= 4096; head_dim in
 * {32, 64, 128};
 * n_heads * head_dim a multiple of 128; n_heads a multiple of n_kv_heads;
 * vocab a multiple of 16; 1 <= max_rows <= JF_MAX_ROWS; max_ctx a multiple of 64. */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab;
  float rope_base, rms_eps;
  int32_t dtype;     /* jf_dtype of the weights and the KV cache; all
                        activations are fp32 (see "activation planes")     */
  int32_t max_rows;  /* largest number of rows of any step / prefill chunk */
  int32_t max_ctx;   /* KV cache capacity in tokens                         */
} jf_config;

/* Activation planes: an activation tensor A[...] of a JF_BF16 model is kept
 * as two bf16 planes, hi = bf16(A) then lo = bf16(A - hi) (A ~= hi + lo to
 * about 16 significant bits); a JF_F32 model keeps one fp32 plane.  Either
 * way 4 bytes per element.  The component calls below take and return
 * activations in this form.
 *
 * GEMM-input layout: an activation matrix that feeds a projection, X[R][K]
 * (K a multiple of 128), is stored with R padded to Rp = 16 * ceil(R / 16)
 * rows as 16-row tiles, each a run of 128-column blocks; inside a 16 x 128
 * block, element (r, c) sits at j * 512 + lane * 8 + e, lane = r + 16 (c/32),
 * j = (c % 32) / 8, e = c % 8 (the matrix-core operand order, so one
 * fragment load is one contiguous 1 KB).  Element (row, col) of X is at
 *   ((row / 16) * (K / 128) + col / 128) * 2048 + that in-block offset,
 * and the lo plane follows the hi plane Rp * K elements later. */

/* One chain of rows in a multi-block step (the input-assembly step of App. A Alg. 1).
 * Rows first_row .. first_row+n_rows-1 form a chain; the first hangs under
 * attach_row (-1: a root, predicted by the last committed row) and every
 * other row under the row before it.  A row sees the committed prefix, its
 * ancestors and itself, and sits at position C + depth.  Rows
 * [first_row, first_row + verify_from) are context only; the rest are
 * verified against their parent's argmax (longest matching run).
 * Segment 0 must be the real-active draft: attach_row = -1, role JF_ROLE_RA,
 * verify_from = 1 (its root row is the pending token, always correct).
 * Segments tile rows 0..R-1 in order and attach backwards (a forest). */
typedef struct {
  int32_t first_row, n_rows, attach_row, role, verify_from;
} jf_segment;

enum { JF_ROLE_RA = 0, JF_ROLE_CAND = 1, JF_ROLE_PSEUDO = 2 };
#define JF_MAX_SEGMENTS 16
/* Rows of one step at most, and the u64 words of a row's in-step visibility
 * mask (bit j of word j / 64: in-step row j is visible). */
#define JF_MAX_ROWS 512
#define JF_VIS_WORDS 8

/* Result of one step, written on the device (16 bytes). */
typedef struct {
  int32_t accept;   /* tokens accepted = rows on the committed path (>= 1)  */
  int32_t winner;   /* segment that won (0: the Jacobi draft)               */
  int32_t pending;  /* argmax of the last accepted row: the next token      */
  int32_t flags;    /* JF_FLAG_* bits                                        */
} jf_step_result;

#define JF_FLAG_BAD_TOKEN 1 /* a token id was outside [0, V); read as 0       */
#define JF_FLAG_CAPACITY 2  /* C + rows exceeded max_ctx; cache writes dropped */
#define JF_FLAG_SYNC 4      /* a wait between the phases of a fused launch gave
                               up (the device did not run all its workgroups
                               at once); the step's outputs are invalid      */

#define JF_FLAG_BAD_PAGE 8 /* a page table entry was outside [0, n_pages); that
                              page was neither read nor written            */

typedef struct jf_model jf_model;
typedef void *jf_stream; /* hipStream_t; NULL is the null stream */

/* Bytes the caller must allocate (device memory) for a configuration.
 * packed: the weights in the kernels' layout; kv: the paged KV cache;
 * ws: workspace (activations, partial results, rope tables, page table). */
jf_status jf_query_sizes(const jf_config *cfg, size_t *packed_bytes,
                         size_t *kv_bytes, size_t *ws_bytes);

/* Bind buffers and pack the weights (Sec. 4.1: a pretrained causal decoder).
 * d_weights[n_weights]: device pointers in fixture order, each [out, in]
 * row-major of cfg->dtype:
 *   embed [V, d]; per layer l: attn_norm [d], wq [H*hd, d], wk [G*hd, d],
 *   wv [G*hd, d], wo [d, H*hd], ffn_norm [d], w_gate [F, d], w_up [F, d],
 *   w_down [d, F]; then final_norm [d], lm_head [V, d].
 * n_weights = 3 + 9 * n_layers.  After the call (and a stream sync) the
 * source tensors are no longer read.  The cache starts empty (C = 0).
 * KV cache layout (d_kv, cfg->dtype): [n_layers][max_ctx/64 pages] pages of
 * 64 tokens, page = K [G][64][hd] followed by V transposed [G][hd][64];
 * logical page p of every layer lives at physical page page_table[p]
 * (identity after load; see jf_kv_set_page_table). */
jf_status jf_model_load(const jf_config *cfg, const void *const *d_weights,
                        int32_t n_weights, void *d_packed, void *d_kv,
                        void *d_ws, jf_stream stream, jf_model **out);

/* Frees the host object only (device buffers stay the caller's). */
jf_status jf_model_free(jf_model *m);

/* Message of the last error on this thread ("" if none). */
const char *jf_last_error(void);

/* Run the prompt through the model in causal chunks of <= max_rows and
 * commit all of it (Sec. 2.1: prompt x; Eq. 1).  d_pending[0] receives the
 * argmax of the last prompt row: the first generated token. Requires C == 0
 * (host view) and n <= max_ctx. */
jf_status jf_prefill(jf_model *m, const int32_t *d_tokens, int32_t n,
                     int32_t *d_pending, jf_stream stream);

/* One Jacobi iteration on a linear draft (Eq. 3).  d_draft[n] holds the
 * draft at positions C..C+n-1; d_draft[0] must be the pending token.
 * Writes d_argmax[n] (g[i] = argmax of row i, lowest id on ties), d_result
 * (accept a = 1 + longest run of d_draft[k] == g[k-1], pending = g[a-1]) and
 * d_next_draft[n]: the Jacobi update g[a-1], g[a], ... ; mode 0 (block,
 * Eq. 4) leaves the n - a + 1 .. n tail unspecified (the next block step uses
 * n - a rows), mode 1 (running window) fills it with
 * pad_id(pad_seed, C + a + i) = splitmix64(pad_seed ^ (pos * 0x9E3779B97F4A7C15)) % V.
 * d_next_draft may equal d_draft.  d_logits (optional, may be NULL) receives
 * the fp32 logits [n][V].  The cache rows C..C+n-1 are overwritten with the
 * draft's K/V; jf_commit_kv keeps the accepted ones.  mode | JF_STEP_COMMIT
 * also commits them in the step (C += a, as jf_commit_kv(m, NULL, d_result,
 * 0, ...) would; no jf_commit_kv follows such a step).  The vocabulary
 * argmax reduction, the acceptance and that commit run in one launch. */
#define JF_STEP_COMMIT 2
jf_status jf_jacobi_step(jf_model *m, const int32_t *d_draft, int32_t n,
                         int32_t mode, uint64_t pad_seed, int32_t *d_argmax,
                         jf_step_result *d_result, int32_t *d_next_draft,
                         float *d_logits, jf_stream stream);

/* One multi-block / rejection-recycling iteration (Sec. 3.2, Alg. 1): R rows
 * d_tokens[R] arranged by segs[n_segs] (host array, n_segs <=
 * JF_MAX_SEGMENTS) into a forest, verified in one forward pass.
 * d_seg_accept[n_segs]: per segment, the longest run of verified rows that
 * match their parent's argmax.  The winner is the segment among 0 and the
 * JF_ROLE_CAND ones with the largest count (ties: segment 0, then the lowest
 * index); d_path[R] receives the committed path (rows from the root down to
 * the winner's last accepted row), d_result its length, winner and pending
 * token.  d_argmax[R] and d_logits (optional) as in jf_jacobi_step. */
jf_status jf_multiblock_step(jf_model *m, const int32_t *d_tokens, int32_t R,
                             const jf_segment *segs, int32_t n_segs,
                             int32_t *d_argmax, int32_t *d_seg_accept,
                             jf_step_result *d_result, int32_t *d_path,
                             float *d_logits, jf_stream stream);

/* Commit the accepted rows of the last step (cache-trim step of Alg. 1): the K/V
 * of path row i moves to position C + i, then C += accept (read from
 * d_result on the device), capped at max_commit if max_commit > 0.
 * d_path NULL means rows 0..accept-1 (a linear step: nothing moves).  Must
 * follow a step on the same model. */
jf_status jf_commit_kv(jf_model *m, const int32_t *d_path,
                       const jf_step_result *d_result, int32_t max_commit,
                       jf_stream stream);

/* Committed length C (synchronises the stream). */
jf_status jf_kv_length(jf_model *m, int32_t *out, jf_stream stream);

/* Drop committed tokens beyond new_len (rejected K/V removal of Alg. 1);
 * JF_E_STATE if new_len > C. Synchronises the stream. */
jf_status jf_kv_truncate(jf_model *m, int32_t new_len, jf_stream stream);

/* Replace the page table (max_ctx/64 entries, device memory copied in; each
 * entry a distinct physical page in [0, max_ctx/64)).  Checked on the host
 * from h_table, a host copy of the same table. */
jf_status jf_kv_set_page_table(jf_model *m, const int32_t *h_table,
                               int32_t n, jf_stream stream);

/* ---- measurement ---------------------------------------------------------
 * Kernel classes of one step; jf_profile_begin makes every following launch
 * of that class on this model bracketed by two HIP events on the launch
 * stream, jf_profile_end synchronises, returns the summed event time (ms)
 * and the number of launches, and stops recording. */
enum {
  JF_KERNEL_QKV = 1,    /* RMSNorm'd x times W_qkv, RoPE, K/V into the cache */
  JF_KERNEL_ATTN = 2,   /* attention + split combine                         */
  JF_KERNEL_O = 3,      /* O projection + residual                           */
  JF_KERNEL_GATEUP = 4, /* gate/up projection + SwiGLU                       */
  JF_KERNEL_DOWN = 5,   /* down projection + residual                        */
  JF_KERNEL_LMHEAD = 6, /* LM head + per-block argmax                        */
  JF_KERNEL_STEP = 7,   /* a whole jf_jacobi_step / jf_multiblock_step       */
  JF_KERNEL_ATTN_BLOCK = 8 /* QKV + attention + O of one layer in one launch
                              (bf16 steps of at most 16 rows)                  */
};
/* Options of a loaded model (host state; effective from the next call).
 * JF_OPT_FUSED_ATTENTION (default 0): 1 makes bf16 steps of at most 16 rows
 * run the QKV projection, the attention and the O projection of each layer
 * as one persistent launch (one workgroup per compute unit; the phases hand
 * over through device flags) instead of four launches.  Both compute the
 * same operation; on the 7B shape at 16 rows the fused launch measured
 * 44 us per layer against 40 us for the four launches, hence the default.
 * Returns JF_E_INVAL for an unknown option or value. */
enum { JF_OPT_FUSED_ATTENTION = 1 };
jf_status jf_model_set_option(jf_model *m, int32_t option, int32_t value);

jf_status jf_profile_begin(jf_model *m, int32_t kernel_class);
jf_status jf_profile_end(jf_model *m, double *total_ms, int32_t *launches);

/* ---- component calls (used by the attention and LM-head workloads) ---- */

/* Attention of one layer (the attention inside Eq. 3's forward pass):
 * q [R][n_heads][head_dim] activation planes, keys/values of positions
 * 0..C+R-1 in one layer's paged cache d_kv_layer (layout as in
 * jf_model_load; slots beyond C+R in a used page must hold finite values),
 * with the page table d_page_table.  Row r sees positions [0, C) and
 * in-step position C + j iff bit j of d_vis[r][JF_VIS_WORDS] is set (d_vis NULL:
 * j <= r, causal).  out: activation planes of the [R][n_heads * head_dim]
 * matrix in the GEMM-input layout (the O projection's input), Rp * n_heads *
 * head_dim elements per plane.  d_ws of at least jf_attention_ws_bytes(...). */
size_t jf_attention_ws_bytes(int32_t n_heads, int32_t head_dim, int32_t R);
jf_status jf_attention(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                       int32_t dtype, int32_t C, int32_t R, const void *d_q,
                       const void *d_kv_layer, const int32_t *d_page_table,
                       const uint64_t *d_vis, void *d_out, void *d_ws,
                       jf_stream stream);

/* LM head + greedy argmax + longest-prefix acceptance (Eq. 3; the
 * verification step of Alg. 1): x [R][d] activation planes in the GEMM-input layout
 * (Rp * d elements per plane) times lm_head^T (dtype), lm_head [V][d]
 * packed by jf_pack_matrix; g = argmax per row (lowest id on ties); accept as in
 * jf_jacobi_step against d_draft[R] (NULL: no acceptance, d_result unused).
 * d_ws of at least jf_lm_head_ws_bytes(R, V).
 * Packed weight layout (jf_pack_matrix): W[rows][cols] (rows % 16 == 0,
 * cols % 128 == 0) as 16 x 128 blocks in the same in-block order as the
 * GEMM-input layout (row r of the block = W row, c = W column); 16-row tiles
 * come in groups of P = 4 (rows % 64 == 0), else 2 (rows % 32 == 0), else 1,
 * and block (tile t, column block kc) is block number
 * ((t / P) * (cols / 128) + kc) * P + t % P. */
size_t jf_packed_matrix_bytes(int32_t rows, int32_t cols, int32_t dtype);
jf_status jf_pack_matrix(int32_t rows, int32_t cols, int32_t dtype,
                         const void *d_src, void *d_packed, jf_stream stream);
size_t jf_lm_head_ws_bytes(int32_t R, int32_t V);
jf_status jf_lm_head_accept(int32_t R, int32_t d, int32_t V, int32_t dtype,
                            const void *d_x, const void *d_w_packed,
                            const int32_t *d_draft, int32_t *d_argmax,
                            jf_step_result *d_result, float *d_logits,
                            void *d_ws, jf_stream stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * operation and outputs as jf_lm_head_accept, with no d_ws argument.  Its
 * scratch (per-block argmax keys and one zeroed word) is a fixed device array
 * inside libjf of JF_NOALLOC_SCRATCH_BYTES, one copy per GPU, held until the
 * process ends; the call performs no hipMalloc / hipFree and enqueues only
 * kernels.  R and V must satisfy jf_lm_head_ws_bytes(R, V) <=
 * JF_NOALLOC_SCRATCH_BYTES (e.g. R <= 64 at V = 152064), else JF_E_CAPACITY
 * and nothing is enqueued.  Every call on one GPU shares that GPU's array and
 * leaves its contents behind; calls that overlap on one GPU (other streams,
 * other threads) race and must be serialised by the caller.  The first call
 * on each device looks up the array's device address (hipGetSymbolAddress);
 * a failure there returns JF_E_HIP. */
#define JF_NOALLOC_SCRATCH_BYTES ((size_t)8 << 20)
jf_status jf_lm_head_accept_noalloc(int32_t R, int32_t d, int32_t V,
                                    int32_t dtype, const void *d_x,
                                    const void *d_w_packed,
                                    const int32_t *d_draft, int32_t *d_argmax,
                                    jf_step_result *d_result, float *d_logits,
                                    jf_stream stream);

/* ---- packed training sequences (forward only) -----------------------------
 * Sec. 3.1 (noise-aware causal attention) and App. C (sequence packing): a
 * training sequence interleaves, for each block i of a response, the noisy
 * block selected from its trajectory and its clean fixed point, so that one
 * forward pass gives the logits of both losses (Eq. 8 and the AR loss). */
enum {
  JF_MASK_NOISY_CONTEXT = 0, /* noisy block i sees the noisy blocks before it */
  JF_MASK_CLEAN_CONTEXT = 1  /* noisy block i sees the clean blocks before it */
};

/* One forward pass over d_tokens[R], R = 2 n_blocks n (R <= max_rows), laid
 * out [noisy_0, clean_0, noisy_1, clean_1, ...] in blocks of n, after the
 * committed prefix (the prompt, from jf_prefill).  Every row sees the
 * prefix and the earlier rows of its own block copy; beyond that a clean
 * block sees the clean blocks before it, and a noisy block sees the noisy
 * (JF_MASK_NOISY_CONTEXT) or the clean (JF_MASK_CLEAN_CONTEXT) blocks
 * before it.  Both copies of block i sit at positions C + i n + k.
 * Writes d_argmax[R] (lowest id on ties) and, if not NULL, the fp32 logits
 * d_logits[R][V].  The cache slots C .. C+R-1 are overwritten and nothing
 * is committed (a following jf_commit_kv fails with JF_E_STATE). */
jf_status jf_packed_forward(jf_model *m, const int32_t *d_tokens,
                            int32_t n_blocks, int32_t n, int32_t mask,
                            int32_t *d_argmax, float *d_logits,
                            jf_stream stream);

/* ---- trajectories (the data collection of Jacobi Forcing) -------------------
 * A block's Jacobi trajectory (Sec. 2.1) is the list of its iterates
 * y^(0), ..., y^(k), stopping at the first k with y^(k) = y^(k-1); y^(k) is
 * the fixed point.  Decoded in block mode (jf_jacobi_step mode 0, then
 * jf_commit_kv), a block of n tokens whose first n - rows positions are
 * accepted feeds its last `rows` tokens to a step, and the step's argmaxes
 * give the next iterate. */

/* Iterate y^(j+1) of an n-token block (Eq. 3) from y^(j) = d_prev[n] and the
 * argmaxes d_argmax[rows] of the step that fed y^(j)'s last rows tokens
 * (1 <= rows <= n):
 *   d_out[i] = d_prev[i]                     for i <= n - rows
 *   d_out[i] = d_argmax[i - (n - rows) - 1]  for i >  n - rows
 * (accepted positions and the pending token stay; each other position takes
 * the prediction made after its predecessor).  d_out may equal d_prev.
 * y^(0) is the caller's initial draft.  JF_E_SHAPE unless 1 <= rows <= n. */
jf_status jf_trajectory_record(const int32_t *d_prev, const int32_t *d_argmax,
                               int32_t n, int32_t rows, int32_t *d_out,
                               jf_stream stream);

/* Noise-schedule point selection (App. C with the schedule of Sec. 3.1,
 * Eq. 7).  d_traj[n_blocks][max_points][n]: block b's trajectory in its
 * first d_len[b] points, the last of them its fixed point y*; other points
 * are not read.  For each point, u = the number of positions that differ
 * from y* (unconverged tokens, Sec. 3.1).  Block b's target noise ratio is
 * t_b = (b mod w) / w (Eq. 7, blocks counted from 0), or d_t_num[b] / w
 * when d_t_num is not NULL (any other schedule on denominator w).
 * d_sel[b] = the point whose u / n is closest to t_b, the earliest on ties,
 * compared exactly in integers as |u w - t_num n| (t_num = b mod w or
 * d_t_num[b]); -1 when d_len[b] is outside
 * [1, max_points] (nothing of that block is read).  d_unconv (optional,
 * [n_blocks][max_points]) receives u per point, -1 beyond d_len[b].
 * n_blocks = 0 does nothing.  JF_E_SHAPE unless n, max_points, w >= 1. */
jf_status jf_trajectory_select(const int32_t *d_traj, const int32_t *d_len,
                               int32_t n_blocks, int32_t n, int32_t max_points,
                               int32_t w, const int32_t *d_t_num,
                               int32_t *d_sel, int32_t *d_unconv,
                               jf_stream stream);

/* ---- batches of sequences over a paged cache --------------------------------
 * Component calls for programs that decode many sequences: they append rows
 * to a paged cache (rotating them), attend over an 8-bit one and read it back.
 * A layer's cache is a pool of n_pages pages of 64 tokens, shared by all
 * sequences; one call works on one layer.
 *
 * Rows (queries, keys, values, outputs) of all sequences lie one after the
 * other: rows d_row_start[s] .. d_row_start[s + 1] - 1 belong to sequence s,
 * which has d_ctx[s] committed tokens, and row i of them has slot
 * d_ctx[s] + i.  Slot t is token t % 64 of physical page
 * d_page_table[s * table_stride + t / 64].  Rows before d_row_start[0] and
 * from d_row_start[n_seqs] on (padding) are neither read nor written.
 *
 * The three arrays stay on the device, so a captured call takes new lengths at
 * every replay; the host gives bounds: n_rows rows in the row tensors, at most
 * max_rows rows a sequence, at most max_ctx slots a sequence (committed and
 * rows; at most 64 table_stride).  What the device holds beyond these bounds
 * is not followed: such a sequence's rows are left as they were and
 * JF_FLAG_CAPACITY is raised (starts that decrease can leave sequences that fit
 * over each other: rows that two of them hold get values of no meaning); a page
 * table entry outside [0, n_pages) raises JF_FLAG_BAD_PAGE and its tokens
 * are skipped.  d_flags (optional, one int32) gets these bits ORed in; the
 * caller clears it.  n_seqs, n_rows or max_rows = 0 does nothing; n_pages = 0
 * otherwise is JF_E_CAPACITY.  n_seqs times the workgroups that max_rows and
 * max_ctx call for must stay within 2^22 (JF_E_CAPACITY). */
typedef struct {
  int32_t n_seqs, n_rows, max_rows, max_ctx, n_pages, table_stride;
  const int32_t *d_row_start;  /* [n_seqs + 1] */
  const int32_t *d_ctx;        /* [n_seqs] */
  const int32_t *d_page_table; /* [n_seqs][table_stride] */
} jf_batch;

/* Bytes of one page of one layer.  JF_F32 / JF_BF16: the page of
 * jf_model_load (K [G][64][hd], then V transposed [G][hd][64]), so such a pool
 * is also what jf_attention reads.  JF_E4M3: codes of the keys [G][64 hd] and
 * of the values [G][64 hd], then fp32 scales [G][2] (keys, values; powers of
 * two: a stored value is its code times its scale), padded to a multiple of
 * 128 bytes.  A head's codes are hd / 16 pieces of 64 lanes x 16 bytes, the
 * order in which the matrix cores take them: byte b of lane l is at
 * (b / 16) * 1024 + l * 16 + b % 16, and
 *   key of token t, dim i:   l = t % 16 + 16 (i / (hd / 4)),
 *                            b = (t / 16) (hd / 4) + i % (hd / 4)
 *   value of token t, dim i: l = i % 16 + 16 ((t / 4) % 4),
 *                            b = 16 (i / 16) + 4 (t / 16) + t % 4.
 * 0 for an unknown type, head_dim not in {32, 64, 128} or n_kv_heads < 1. */
size_t jf_kv_page_bytes(int32_t n_kv_heads, int32_t head_dim, int32_t kv_dtype);

/* Appends the rows' keys and values to the cache (type kv_dtype), and rotates
 * the queries.  d_k, d_v [n_rows][n_kv_heads * head_dim] and d_q (optional)
 * [n_rows][n_heads * head_dim] are rows of x_dtype (JF_F32 or JF_BF16), ld_*
 * elements apart (views into one fused projection, for instance).
 * Rotation: rope_base > 1 turns dims (i, i + head_dim / 2) of queries and keys
 * by p * rope_base^(-2 i / head_dim), p = d_pos[row] (rows of a tree share
 * positions) or, for d_pos NULL, the row's slot; rope_base 0 leaves them.
 * d_q_out gets the queries as activation planes [n_rows][n_heads][head_dim] of
 * act_dtype, as the attention calls take them.
 * JF_E4M3: the keys and the values of one head in one page share a scale.  A
 * call that appends into a page takes the smallest power of two that brings
 * the finite new values there to 448 or less (1 if they are all 0, 2^-100 at
 * least) or, where the page keeps earlier tokens (slots below d_ctx), the scale
 * it has if that is larger (not a scale of 1 over kept tokens that are all 0);
 * if the scale grows, the kept tokens' codes are rounded anew on it.  Codes
 * round to nearest, ties to even; infinities saturate at 448 times the scale
 * and NaN stays NaN.
 * Rows dropped by a verification need no call: the next append at the shorter
 * d_ctx overwrites them.  Their scale stays: but for kept zeros, a scale does
 * not shrink until the page is appended to from its first token on, so a draft
 * row with a large element leaves the tokens of its page on coarser codes.
 * Slots that no row names keep what they hold; in a JF_E4M3 page those past the
 * rows keep their codes, which stand for other values on another scale.
 * d_kv and d_q_out must start on 16-byte boundaries.  No page may be written
 * twice by one call (by two sequences, or at two places of one's table). */
jf_status jf_kv_append(const jf_batch *batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t kv_dtype,
                       int32_t x_dtype, int32_t act_dtype, const void *d_q, int64_t ld_q, const void *d_k,
                       int64_t ld_k, const void *d_v, int64_t ld_v, const int32_t *d_pos, double rope_base,
                       void *d_kv, void *d_q_out, int32_t *d_flags, jf_stream stream);

/* Reads slots d_ctx[s] .. d_ctx[s] + rows - 1 back as the values they hold:
 * d_k, d_v rows [n_rows][n_kv_heads * head_dim] of x_dtype, ld_* elements
 * apart (JF_BF16 holds an e4m3 value exactly).  d_kv must start on a 16-byte
 * boundary.  Rows whose page is bad stay as they were. */
jf_status jf_kv_read(const jf_batch *batch, int32_t n_kv_heads, int32_t head_dim, int32_t kv_dtype, int32_t x_dtype,
                     const void *d_kv, void *d_k, int64_t ld_k, void *d_v, int64_t ld_v, int32_t *d_flags,
                     jf_stream stream);

/* Attention over a JF_E4M3 cache that already holds the rows' keys and values:
 * row i of sequence s sees slots [0, d_ctx[s]) and in-step slot d_ctx[s] + j
 * iff bit j of d_vis[row][JF_VIS_WORDS] is set (d_vis NULL: j <= i).  A row
 * that sees nothing gets zeros; what a slot holds does not reach a row that
 * does not see it, NaN included.  d_q [n_rows][n_heads][head_dim] and d_out
 * are activation planes of act_dtype, d_out in the GEMM-input layout of
 * [n_rows][n_heads * head_dim] (a multiple of 128 columns), Rp * n_heads *
 * head_dim elements per plane with Rp = n_rows rounded up to 16; max_rows <=
 * JF_MAX_ROWS.  d_q, d_kv, d_out and d_ws must start on 16-byte boundaries;
 * d_ws holds jf_attention_kv8_ws_bytes(...) bytes, needs no clearing and may
 * be shared by calls that do not overlap.  The size is that of this batch: one
 * with fewer sequences or rows is cut into more parts and can need more. */
size_t jf_attention_kv8_ws_bytes(const jf_batch *batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);
jf_status jf_attention_kv8(const jf_batch *batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                           int32_t act_dtype, const void *d_q, const void *d_kv, const uint64_t *d_vis, void *d_out,
                           void *d_ws, int32_t *d_flags, jf_stream stream);

/* ---- log probabilities ------------------------------------------------------
 * Of logits d_logits [R][V] (JF_F32 as the steps and jf_packed_forward return
 * them, or JF_BF16), rows ld elements apart, with p = softmax of a row.  Each
 * output may be NULL:
 *   d_logprob[R]: log p of token d_tokens[row]; 0 where that is -1 (a row
 *     without a token), NaN for any other id outside [0, V);
 *   d_entropy[R]: -sum p log p;
 *   d_norm[R][2]: the row's maximum m and log sum e^(x - m), whose sum is the
 *     logarithm of the softmax's denominator (kept apart: no digits are lost
 *     at large offsets), which the gradient takes;
 *   d_top_ids, d_top_logprob [R][k], 0 <= k <= JF_MAX_TOP: the k largest
 *     logits' ids and log probabilities in order (ties: lowest id first).
 * A logit of -inf has p = 0 and is no alternative; places beyond the finite
 * logits get id -1 and -inf.  A row that is no distribution (all -inf, +inf or
 * NaN among its logits) gets ids -1 and NaN everywhere else, but for the 0 of a
 * row without a token.  d_ws, 16-byte
 * aligned, holds jf_token_logprobs_ws_bytes(R, V, k) bytes, which are enough
 * for fewer rows too, and needs no clearing.
 * R = 0 does nothing.  V <= 2^30, R <= 2^22. */
#define JF_MAX_TOP 32
size_t jf_token_logprobs_ws_bytes(int32_t R, int32_t V, int32_t k);
jf_status jf_token_logprobs(int32_t R, int32_t V, int32_t dtype, const void *d_logits, int64_t ld,
                            const int32_t *d_tokens, int32_t k, float *d_logprob, float *d_entropy, float *d_norm,
                            int32_t *d_top_ids, float *d_top_logprob, void *d_ws, jf_stream stream);

/* Gradient of sum(d_g_logprob * logprob + d_g_entropy * entropy) to the
 * logits, d_grad [R][V] of their type, rows ld_grad elements apart:
 *   g (1[j = token] - p_j) - h p_j (log p_j + entropy).
 * d_norm and d_entropy are those of jf_token_logprobs on the same logits.
 * d_g_logprob NULL: g = 0 (else d_tokens is needed); d_g_entropy NULL: h = 0
 * (else d_entropy is needed).  Rows with g = h = 0 get zeros, rows whose token
 * is -1 have g = 0.  d_grad may be d_logits (same ld): in place.  Writes only
 * columns [0, V). */
jf_status jf_token_logprobs_grad(int32_t R, int32_t V, int32_t dtype, const void *d_logits, int64_t ld,
                                 const int32_t *d_tokens, const float *d_norm, const float *d_entropy,
                                 const float *d_g_logprob, const float *d_g_entropy, void *d_grad, int64_t ld_grad,
                                 jf_stream stream);

/* ---- causal attention over packed sequences, with its gradient ---------------
 * Sequences lie one after the other in the row tensors: rows d_row_start[s] ..
 * d_row_start[s + 1] - 1 (device, [n_seqs + 1], not decreasing) belong to
 * sequence s, and each sees the rows of its own sequence up to itself.  Rows
 * before d_row_start[0] and from d_row_start[n_seqs] on (padding) are neither
 * read nor written.  A captured call takes new starts at every replay.  A
 * sequence whose start or end lies outside [0, n_rows], or whose end lies
 * before its start, is left as it was and JF_FLAG_CAPACITY is raised in
 * d_flags (optional, one int32, ORed; the caller clears it).  Of those that
 * remain, one that starts before an earlier one's end is left as it was too,
 * among up to 64 sequences; among more, others may be left as they were, and
 * rows that several hold get values of no meaning.
 * d_q, d_out [n_rows][n_heads * head_dim], d_k, d_v [n_rows][n_kv_heads *
 * head_dim] are rows of dtype (JF_F32 or JF_BF16), ld_* elements apart (views
 * into one fused projection, for instance); query head j reads KV head j /
 * (n_heads / n_kv_heads); scores are q k / sqrt(head_dim), head_dim in {32,
 * 64, 128}.  Rows that start on 16-byte boundaries are read faster.
 * d_lse (optional) [n_heads][n_rows] gets the logarithm of each row's sum of
 * e^score, which the gradient takes.  Scores, sums and statistics are fp32; in
 * JF_BF16 each weight is rounded to bf16 (2^-8 of it at most) for its product
 * with the values.  What a row does not see does not reach it, NaN included;
 * an infinity among the values that it sees gives an infinity, or NaN beside
 * another or where its weight is too small for fp32.  A row all of whose scores
 * are -inf gets zeros and -inf.  d_out must not overlap the inputs.  n_seqs or
 * n_rows = 0 does nothing. */
jf_status jf_attention_causal(int32_t n_seqs, int32_t n_rows, const int32_t *d_row_start, int32_t n_heads,
                              int32_t n_kv_heads, int32_t head_dim, int32_t dtype, const void *d_q, int64_t ld_q,
                              const void *d_k, int64_t ld_k, const void *d_v, int64_t ld_v, void *d_out,
                              int64_t ld_out, float *d_lse, int32_t *d_flags, jf_stream stream);

/* Gradient of sum(d_g_out * out) to the queries, keys and values, from what
 * jf_attention_causal was given and gave (d_out, d_lse).  The gradients of
 * keys and values are sums over the query heads that share them.  All row
 * tensors are of dtype; the gradients must overlap no input (but may be
 * columns of one tensor).  Nothing depends on the order in which workgroups
 * run.  Sums are fp32; in JF_BF16 weights and their gradients are rounded to
 * bf16 for the products, and a row's dot product of d_g_out and out is that of
 * the rounded d_out.  Weights are computed anew from d_lse, whose fp32 digits
 * leave them off by 2^-24 times the score (the factor e^0.06 at 2^20); however
 * large the scores are, they are at most 1.  An infinity or NaN among a
 * sequence's inputs may reach every gradient of that sequence, and none of
 * another's; a NaN score makes the gradients of its row's query and of the keys
 * and values that the row sees NaN.  d_ws, on a 16-byte boundary, holds
 * jf_attention_causal_grad_ws_bytes(...) bytes, which are enough for fewer
 * rows and sequences of these heads too, needs no clearing and may be shared
 * by calls that do not overlap. */
size_t jf_attention_causal_grad_ws_bytes(int32_t n_seqs, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads,
                                         int32_t head_dim);
jf_status jf_attention_causal_grad(int32_t n_seqs, int32_t n_rows, const int32_t *d_row_start, int32_t n_heads,
                                   int32_t n_kv_heads, int32_t head_dim, int32_t dtype, const void *d_q, int64_t ld_q,
                                   const void *d_k, int64_t ld_k, const void *d_v, int64_t ld_v, const void *d_out,
                                   int64_t ld_out, const float *d_lse, const void *d_g_out, int64_t ld_g_out,
                                   void *d_g_q, int64_t ld_g_q, void *d_g_k, int64_t ld_g_k, void *d_g_v,
                                   int64_t ld_g_v, void *d_ws, int32_t *d_flags, jf_stream stream);

/* ---- attention of a batch that shares prefixes --------------------------------
 * Groups of sequences that follow each other share their first pages: samples
 * of one prompt, requests behind one system prompt.  Sequences d_seq_start[g]
 * .. d_seq_start[g + 1] - 1 (device, [n_groups + 1], not decreasing) form
 * group g, and the first d_pages[g] entries of their rows of the page table
 * name the same pages (those of the group's first sequence are read).  Only
 * whole pages of committed tokens are shared: 64 d_pages[g] <= d_ctx of each.
 * Sequences of no group share nothing.  The host gives bounds: at most
 * max_rows rows of one group and max_pages (<= table_stride) shared pages.
 * What the device holds beyond these, a group that starts before an earlier
 * one's start, or a sequence with fewer committed tokens than it is said to
 * share or with rows outside its group's, raises JF_FLAG_CAPACITY, and the rows
 * of such a group or sequence are left as they were. */
typedef struct {
  int32_t n_groups, max_rows, max_pages;
  const int32_t *d_seq_start; /* [n_groups + 1] */
  const int32_t *d_pages;     /* [n_groups] */
} jf_prefix;

/* Attention over a cache of dtype JF_F32 or JF_BF16 (the pages of jf_kv_append)
 * that already holds the rows' keys and values: row i of sequence s sees
 * slots [0, d_ctx[s]) and in-step slot d_ctx[s] + j iff bit j of
 * d_vis[row][JF_VIS_WORDS] is set (d_vis NULL: j <= i), as if nothing were
 * shared; the shared pages are read once for all rows of a group.  A row that
 * sees nothing gets zeros; what a slot holds does not reach a row that does
 * not see it, NaN included (an infinity that it sees gives an output that is
 * not finite).  A page outside the pool raises JF_FLAG_BAD_PAGE and its
 * slots are seen by nobody.  d_q [n_rows][n_heads][head_dim] and d_out are
 * activation planes of dtype, d_out in the GEMM-input layout of [n_rows]
 * [n_heads * head_dim] (a multiple of 128 columns); the batch's max_rows <=
 * JF_MAX_ROWS.  d_q, d_kv, d_out and d_ws must start on 16-byte boundaries;
 * d_ws holds jf_attention_shared_ws_bytes(...) bytes (0: the call would be
 * refused), needs no clearing and may be shared by calls that do not overlap.
 * The size is that of this batch and prefix: one with fewer sequences, groups
 * or rows is cut into more parts and can need more, so a workspace for several
 * holds the largest of their sizes.  prefix NULL: nothing is shared. */
size_t jf_attention_shared_ws_bytes(const jf_batch *batch, const jf_prefix *prefix, int32_t n_heads,
                                    int32_t n_kv_heads, int32_t head_dim);
jf_status jf_attention_shared(const jf_batch *batch, const jf_prefix *prefix, int32_t n_heads, int32_t n_kv_heads,
                              int32_t head_dim, int32_t dtype, const void *d_q, const void *d_kv,
                              const uint64_t *d_vis, void *d_out, void *d_ws, int32_t *d_flags, jf_stream stream);

/* ---- policy loss ----------------------------------------------------------------
 * Clipped policy loss with a KL term over the tokens of sampled sequences, and
 * its gradient to the log probabilities and entropies of jf_token_logprobs,
 * as jf_token_logprobs_grad takes it (d_g_logprob, d_g_entropy).
 * Rows d_row_start[s] .. d_row_start[s + 1] - 1 (device, [n_seqs + 1], not
 * decreasing) belong to sequence s; a row with d_tokens[row] = -1 (d_tokens
 * NULL: none) has no token: its gradients are 0 and it counts nowhere.  What
 * rows outside all sequences hold counts nowhere, and no gradient is written
 * there.  For a row with
 * advantage A (d_advantage[row], or [sequence] for adv_rows 0):
 *   r = e^(logprob - old), policy = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A), 0 for A = 0
 *   k = ref - logprob, kl = e^k - k - 1 (d_ref_logprob NULL: 0)
 *   loss = scale * sum w (policy + kl_weight kl - entropy_weight entropy)   (d_entropy NULL: without it)
 * with w = 1 / tokens (JF_MEAN_TOKENS), 1 / (sequences with tokens * tokens of
 * the row's) (JF_MEAN_SEQS) or 1 (JF_SUM).  Clipped rows (A > 0 and r > 1 +
 * clip_high, or A < 0 and r < 1 - clip_low) have no gradient of the policy
 * term; a weight of 0 leaves its term out of loss and gradient, whatever its
 * value.  Differences and exponentials are computed in 64 bits; the order of
 * the sums is fixed.
 *   d_stats[JF_POLICY_STATS]: the loss, then sum w of policy, kl, entropy and
 *     clipped rows, then the number of tokens (no tokens: all 0);
 *   d_g_logprob, d_g_entropy [n_rows] (either may be NULL): the gradient.
 * Row starts that decrease or lie outside [0, n_rows] raise JF_FLAG_CAPACITY
 * in d_flags (optional): the statistics are NaN and no gradient is written.
 * n_seqs or n_rows = 0: statistics 0, no gradient.  n_rows, n_seqs <= 2^22.
 * d_ws, on a 16-byte boundary, holds jf_policy_loss_ws_bytes(...) bytes, needs
 * no clearing and may be shared by calls that do not overlap. */
enum { JF_MEAN_TOKENS = 0, JF_MEAN_SEQS = 1, JF_SUM = 2 };
#define JF_POLICY_STATS 6
typedef struct {
  double clip_low, clip_high;  /* 0 <= clip_low <= 1, clip_high >= 0 (may be infinite) */
  double kl_weight, entropy_weight, scale;
  int32_t mean;                /* JF_MEAN_TOKENS, JF_MEAN_SEQS or JF_SUM */
  int32_t adv_rows;            /* 0: one advantage a sequence, 1: one a row */
} jf_policy;
size_t jf_policy_loss_ws_bytes(int32_t n_seqs, int32_t n_rows);
jf_status jf_policy_loss(const jf_policy *policy, int32_t n_seqs, int32_t n_rows, const int32_t *d_row_start,
                         const int32_t *d_tokens, const float *d_logprob, const float *d_old_logprob,
                         const float *d_ref_logprob, const float *d_entropy, const float *d_advantage, float *d_stats,
                         float *d_g_logprob, float *d_g_entropy, void *d_ws, int32_t *d_flags, jf_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* JF_H */
