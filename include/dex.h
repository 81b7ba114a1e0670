/*
 * dex.h -- C ABI of the MI355X (gfx950) Depth Exploration Decoding library.
 *
 * One library context decodes `batch` independent sequences, each with its
 * own depth-position lattice, greedily, exactly as Algorithm 1 of the paper
 * ("Depth Exploration for LLM Decoding") describes:
 *   - dex_create    : a model with exit depths and an explored-depth set X
 *                     (Definition 3: d_0 < ... < d_{N-1} = L) go in;
 *                     stage k is the layer range (d_{k-1}, d_k] (Algorithm 1,
 *                     Require clause).
 *   - dex_prefill   : Algorithm 1's init -- the prompt's keys/values and the
 *                     first generated token (final-depth argmax at the last
 *                     prompt position).
 *   - dex_step      : one iteration of Algorithm 1's loop (expand, DECS,
 *                     insert, and when the anchor reaches the final depth
 *                     validate-and-commit then collapse) for every sequence;
 *                     commits at most one token per sequence.
 *   - dex_destroy   : frees everything the library allocated.
 *
 * The committed tokens equal greedy autoregressive decoding of the same
 * model (the lossless invariant of Section 3.2); with X = {L} and
 * width_cap = 1 each dex_step is one plain autoregressive step.
 *
 * Conventions
 *   - Every call returns dex_status; DEX_OK is 0, errors are negative.  No
 *     C++ exception crosses the ABI.  dex_last_error(ctx) gives a message
 *     (dex_last_error(NULL): the last dex_create failure of this thread).
 *   - Weights are passed as DEVICE memory, row-major; a projection matrix is
 *     [out_features][in_features].  dex_create repacks every projection
 *     matrix and the LM head into the library's own streaming layout, so a
 *     context holds a second, library-owned copy of those weights (one more
 *     model's worth of device memory: about 14.2 GB for a 32-layer d_model
 *     4096 model) until dex_destroy.  The caller's embedding table and norm
 *     gains stay borrowed: keep them alive and unchanged until dex_destroy
 *     (the caller's projection and LM-head arrays may be freed once
 *     dex_create has returned).  The library also owns the key/value caches,
 *     the lattice state and all scratch memory.  A context's first
 *     dex_prefill allocates prompt scratch (activations of about 8192 prompt
 *     rows at a time, or of one longer prompt: 0.65 GB at d_model 4096, d_ffn
 *     14336), and the context holds up to 1 GiB of it, with 1 MiB of pinned
 *     host memory, for further prompts until dex_destroy; a larger one is
 *     freed before dex_prefill returns.  Plan for it where several contexts
 *     share a GPU or memory is allocated after a prompt.
 *   - Host arrays passed in or out are caller-owned and only accessed during
 *     the call.
 *   - All device work is enqueued on config.hip_stream (NULL = the default
 *     stream).  dex_prefill and dex_step synchronise that stream before
 *     returning host results.  A context is not thread-safe.
 *   - Argument errors (DEX_E_INVAL), a prefill that could not allocate its
 *     scratch (DEX_E_NOMEM) and "every sequence is full" (DEX_E_CAPACITY
 *     before any work) leave the context as it was.  Any other failure
 *     inside an entry point -- a failed HIP call, a lattice capacity
 *     overflow found after the round's planning began, a host/device commit
 *     mismatch -- poisons it: later dex_prefill / dex_step calls return
 *     DEX_E_STATE; dex_destroy still frees everything.
 */
#ifndef DEX_H
#define DEX_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dex_ctx dex_ctx;

typedef enum {
  DEX_OK = 0,
  DEX_E_INVAL = -1,     /* bad argument (dims, explored set, sizes, null pointers) */
  DEX_E_NOMEM = -2,     /* device or host allocation failed */
  DEX_E_HIP = -3,       /* a HIP runtime call failed; message in dex_last_error */
  DEX_E_STATE = -4,     /* call out of order (step before prefill) or poisoned context */
  DEX_E_CAPACITY = -5   /* max_context or lattice capacity exhausted */
} dex_status;

typedef enum { DEX_F32 = 0, DEX_BF16 = 1 } dex_dtype;

/* Per-layer parameter order inside dex_model.layers. */
enum {
  DEX_P_ATTN_NORM = 0,  /* float [d]                    RMSNorm gain before attention */
  DEX_P_WQ = 1,         /* weight [H*hd][d]             query projection */
  DEX_P_WK = 2,         /* weight [Hkv*hd][d]           key projection */
  DEX_P_WV = 3,         /* weight [Hkv*hd][d]           value projection */
  DEX_P_WO = 4,         /* weight [d][H*hd]             attention output projection */
  DEX_P_FFN_NORM = 5,   /* float [d]                    RMSNorm gain before the FFN */
  DEX_P_W_GATE = 6,     /* weight [F][d]                SwiGLU gate projection */
  DEX_P_W_UP = 7,       /* weight [F][d]                SwiGLU up projection */
  DEX_P_W_DOWN = 8,     /* weight [d][F]                SwiGLU down projection */
  DEX_P_COUNT = 9
};

#define DEX_MAX_BATCH 64
#define DEX_MAX_EXPLORED 32
#define DEX_MAX_ROWS 256

/* "A model with exit depths": a decoder-only Llama-family backbone whose
 * shared final RMSNorm and LM head decode every explored depth (the paper's
 * inducing-adapter appendix: intermediate depths use the same final
 * normalisation and LM head).  Layer l (1-based) scales both residual
 * branches by residual_scale * l / L.  RoPE is rotate-half with base
 * rope_theta; attention scale 1/sqrt(head_dim); query head h reads key/value
 * head h / (n_heads / n_kv_heads).  `weight_dtype` is the element type of the
 * embedding, the projections and the LM head, and also of the key/value
 * cache and the activations fed to the matrix cores; norm gains are float.
 * Requirements: d_model a multiple of 16; head_dim 32, 64 or 128; n_heads
 * a multiple of n_kv_heads; n_heads/n_kv_heads <= 8 (DEX_E_INVAL from
 * dex_create otherwise).                                                   */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab;
  float rope_theta, rms_eps, residual_scale;
  int32_t weight_dtype;                 /* dex_dtype */
  const void *embed;                    /* device [vocab][d] */
  const float *final_norm;              /* device [d] */
  const void *lm_head;                  /* device [vocab][d] */
  const void *const *layers;            /* HOST array [n_layers * DEX_P_COUNT] of device pointers */
} dex_model;

/* "An explored-depth set" plus execution limits. */
typedef struct {
  const int32_t *explored;              /* host [n_explored], strictly increasing in [1, L], last == L */
  int32_t n_explored;                   /* N, 1 .. DEX_MAX_EXPLORED */
  int32_t width_cap;                    /* lattice rows per round per sequence; 0 = uncapped
                                           (the paper's binary lattice, needs 2^(N-1) rows) */
  int32_t decs;                         /* 1: DECS masked argmax (Algorithm 2, greedy); 0: plain argmax */
  int32_t batch;                        /* independent sequences, 1 .. DEX_MAX_BATCH */
  int32_t max_context;                  /* prompt length + generated tokens, per sequence */
  void *hip_stream;                     /* hipStream_t or NULL */
  int32_t stage_streams;                /* streams (lanes) a round's stages are spread
                                           over: the stages of one round read and write
                                           disjoint state, so they may run concurrently.
                                           0: the library default; 1: everything on
                                           hip_stream */
  float temperature;                    /* 0: greedy decoding.  > 0: Algorithm 2's sampling
                                           mode, every node decodes argmax(l / temperature
                                           + G) with G the Gumbel row of (sample_seed,
                                           sequence, position of the node's input token)
                                           (see dex_debug_gumbel below) */
  uint64_t sample_seed;
  int32_t adapter_dim;                  /* 0: no adapters.  Else m, the hidden width of the
                                           inducing adapters (Section 3.4 and its appendix):
                                           a node at a non-final explored depth k decodes
                                           h + dh_k(h), dh = alpha (W2 silu(W1 RMSNorm(h; g)
                                           + b1) + b2); the final depth is never adapted */
  const void *const *adapters;          /* [n_explored - 1][6] device pointers per non-final
                                           depth: g float[d], W1 [m][d], b1 float[m],
                                           W2 [d][m], b2 float[d], alpha float[1]; matrices in
                                           weight_dtype.  Borrowed: read at create (the
                                           library keeps repacked copies and alpha) */
  int32_t stage_grouping;               /* 0 (default) or 1: each lane takes a contiguous run
                                           of the round's stages and runs them in step, each
                                           kernel launched once per layer step for every
                                           stage of the run that has that step; -1: each
                                           stage's layers launched on their own, the stages
                                           dealt round-robin over the lanes.  The results
                                           are the same bits either way. */
} dex_config;

/* What one dex_step did (all host memory).  Rows are listed stage-major,
 * then by sequence, then in the lattice's priority order.                  */
typedef struct {
  int32_t n_rows;                       /* lattice nodes evaluated this round, all sequences */
  int32_t rows_per_stage[DEX_MAX_EXPLORED];
  int32_t layers_streamed;              /* layers of the stages that had >= 1 row */
  int32_t row_layers;                   /* sum over rows of the layers each row ran */
  int32_t q[DEX_MAX_BATCH];             /* FSM state (anchor's completed stages) at round start */
  int32_t kstar[DEX_MAX_BATCH];         /* shallowest matching depth index if committed, else -1 */
  int32_t row_seq[DEX_MAX_ROWS];
  int32_t row_slot[DEX_MAX_ROWS];       /* canonical slot index within its sequence's lattice */
  int32_t row_stage[DEX_MAX_ROWS];
  int32_t row_pos[DEX_MAX_ROWS];        /* absolute position of the row's input token */
  int32_t row_token[DEX_MAX_ROWS];      /* decoded candidate (DECS argmax) of the row */
  int64_t rounds_total;                 /* dex_step calls so far */
  double attn_bytes;                    /* algorithmic bytes of the round's attention: keys and
                                           values of every position up to each row group's
                                           deepest row, at every layer it ran, plus the
                                           queries read and the outputs written */
} dex_step_info;

/* Validate the model and X, derive the stages, allocate caches and scratch.
 * Errors: DEX_E_INVAL (dims, X not strictly increasing / not ending at L,
 * rows per round above DEX_MAX_ROWS), DEX_E_NOMEM, DEX_E_HIP.              */
dex_status dex_create(const dex_model *model, const dex_config *config, dex_ctx **out);

/* Algorithm 1's init.  prompts: host [batch][prompt_len] token ids in
 * [0, vocab).  Writes first_tokens[batch] (host): y_0 per sequence.  May be
 * called again to restart decoding with new prompts.
 * Errors: DEX_E_INVAL (ids, lengths), DEX_E_CAPACITY (prompt_len >= max_context). */
dex_status dex_prefill(dex_ctx *ctx, const int32_t *prompts, int32_t prompt_len, int32_t *first_tokens);

/* One round for every sequence.  committed (host [batch]): the token a
 * sequence committed this round, or -1.  info may be NULL.  A sequence whose
 * committed length reached max_context takes no further part.
 * Errors: DEX_E_STATE (no prefill yet / poisoned), DEX_E_CAPACITY (every
 * sequence is full, or the lattice outgrew its slot capacity), DEX_E_HIP.   */
dex_status dex_step(dex_ctx *ctx, int32_t *committed, dex_step_info *info);

/* Frees every library-owned allocation.  NULL-safe. */
void dex_destroy(dex_ctx *ctx);

const char *dex_last_error(const dex_ctx *ctx);

/* ---------------------------------------------------------------------------
 * Inspection taps for tests and the benchmark.
 * ------------------------------------------------------------------------- */

/* The work items the planner picks for one lattice state (host only: no
 * context and no GPU are needed).  Algorithm 1's expansion with the
 * eligibility of the one-explorer-per-device pipeline (a non-anchor slot
 * advances only when every ancestor has completed more stages) and the
 * width-cap priority (not in the paper, which names branch pruning as future
 * work): the anchor's advance first, then the width_cap - 1 other items of
 * lowest (hypothesis cost, path length, path), where a path is the string of
 * depth steps (a slot's stage k to k+1) and position steps (a slot's stage f
 * to the stage-0 node of the slot forked there) from the anchor's stage-0
 * node to the item's node, compared with the depth step first, and the
 * hypothesis cost is the sum of f + 1 over the fork stages f on it.
 *   slots      host [n_slots][4 + n_explored] int32, canonical order, slot 0
 *              the anchor: parent (-1 for slot 0, else an earlier slot),
 *              fork stage (< the parent's c, <= n_explored - 2; at most one
 *              child per (parent, stage)), c (completed stages), absolute
 *              position, then the candidates u[0..c-1] (the rest ignored)
 *   out        host [capacity][3] int32: kind (0 advance, 1 fork), slot,
 *              fork stage (-1 for advance), in priority order; *n_out = count
 * width_cap 0 = uncapped.  Malformed slots or too small a capacity:
 * DEX_E_INVAL (*n_out still receives the count in the latter case).        */
dex_status dex_debug_plan(int32_t n_explored, int32_t width_cap, int32_t decs, int32_t max_context,
                          const int32_t *slots, int32_t n_slots, int32_t *out, int32_t capacity, int32_t *n_out);

/* While enabled, every dex_step writes the float32 exit logits (before the
 * DECS mask) of each round row r to device_buf + r * vocab.  capacity_rows
 * must be >= the rows a round can have.  device_buf NULL disables.          */
dex_status dex_debug_set_logits_tap(dex_ctx *ctx, float *device_buf, int32_t capacity_rows);

/* Slot table of sequence `seq` in canonical order, each slot written as
 * stride = 5 + N int32: x, pos, parent (-1 for the anchor), fork stage, c,
 * then u[0..N-1] (-1 where not computed).  *n_slots receives the count.     */
dex_status dex_debug_lattice(dex_ctx *ctx, int32_t seq, int32_t *out, int32_t capacity_slots, int32_t *n_slots);

/* The last collapse of sequence `seq`: old canonical indices of the retained
 * slots (in order), whether the new anchor is fresh, and the committed
 * position the old anchor's keys/values went to.                            */
dex_status dex_debug_last_collapse(dex_ctx *ctx, int32_t seq, int32_t *map, int32_t capacity,
                                   int32_t *n_map, int32_t *fresh, int32_t *committed_pos);

/* Key/value cache layout: element (layer l, seq s, kv head g, entry e, dim i)
 * is at base + (((l * batch + s) * n_kv_heads + g) * entries + e) * head_dim + i
 * with entries returned in *entries.  Entry p < max_context is committed
 * position p; lattice slot j of seq s lives at entry lattice_entry(s, j)
 * (see dex_debug_slot_entry).                                                */
dex_status dex_debug_kv_layout(dex_ctx *ctx, void **k_base, void **v_base, int64_t *entries);
dex_status dex_debug_slot_entry(dex_ctx *ctx, int32_t seq, int32_t slot, int32_t *entry);

/* Kernel timing: while enabled, hipEvents bracket every launch of the layer
 * kernels on the context's stream.  dex_debug_kernel_times fills, for each
 * kernel class c < n (0 qkv, 1 attention, 2 attention combine, 3 o-proj,
 * 4 gate/up, 5 down, 6 lm-head, 7 other), the summed milliseconds and the
 * launch count since the last reset, and the algorithmic bytes moved by those
 * launches (weights + activations + keys/values they read or write).          */
dex_status dex_debug_set_kernel_timing(dex_ctx *ctx, int32_t enable);
dex_status dex_debug_kernel_times(dex_ctx *ctx, int32_t n, double *ms, int64_t *launches, double *bytes);

/* Round phases: while enabled, dex_step records events on the decode stream
 * at its boundaries.  dex_debug_round_times fills, summed over the rounds
 * since the last enable (*rounds of them), in milliseconds:
 *   ms[0] row-table upload           ms[1] stage sweep (all lanes joined)
 *   ms[2] exit head, verify/commit, the results' stores to the host
 *   ms[3] 0: those stores leave no copy to time
 *   ms[4] host commit handling and the collapse gather (from the exit's
 *         end to the collapse's end; one round fewer than *rounds)
 *   ms[5] the gap before a round: from the previous round's last device
 *         work to this round's upload (return to the caller, the caller's
 *         own work, the next call's planning; one round fewer)
 *   ms[6] host planning (dex_step entry to the upload, host clock)
 * n <= 7 entries are written.                                               */
dex_status dex_debug_set_round_timing(dex_ctx *ctx, int32_t enable);
dex_status dex_debug_round_times(dex_ctx *ctx, int32_t n, double *ms, int64_t *rounds);

/* Mean duration of one decode-step GEMM class (3 o-proj, 4 gate/up, 5 down,
 * 6 lm-head) at M rows: `reps` back-to-back launches on the context's stream
 * between two hipEvents, cycling through the layers' weights so that no
 * launch re-reads a matrix another launch just streamed.  Uses the context's
 * scratch buffers (the decode state is untouched).  *bytes_per_launch is the
 * algorithmic traffic of one launch (weights plus activations).            */
dex_status dex_debug_time_kernel(dex_ctx *ctx, int32_t cls, int32_t M, int32_t reps, double *avg_us,
                                 double *bytes_per_launch);

/* Stand-alone GEMM y[M][N] = x[M][K] * W[N][K]^T (float32 out).  M in
 * [1, 64] runs the skinny matrix-core kernel the decode step uses (tests of
 * batch invariance); M > 64 (bf16 only, N a multiple of 16) runs the M-tiled
 * kernel of the prompt prefill.  dtype: dex_dtype of W and x; K a multiple of
 * 8 (bf16) or 4 (fp32).  Device pointers.                                   */
dex_status dex_debug_gemm(int32_t dtype, const void *W, int32_t N, int32_t K, const void *x, int32_t M,
                          float *y, void *hip_stream);

/* Stand-alone decode attention (K4, the branch-masked attention of one
 * layer) with its split combine, launched exactly as a step launches them
 * for one stage.  Row r (sequence row_seq[r], absolute position row_pos[r],
 * committed length row_nc[r]) attends with every query head h to the
 * logical keys 0..row_pos[r] of kv head h / (n_heads / n_kv_heads): cache
 * entries 0..row_nc[r]-1 of its sequence, then entry chain[chain_off[r] + t]
 * for position row_nc[r] + t (its ancestor slots and its own slot), with
 * scale 1/sqrt(head_dim) and softmax over those keys.  Consecutive rows of
 * one sequence with equal row_nc form a row group as in a step.
 *   dtype      dex_dtype of the caches and of out (bf16: matrix-core kernel
 *              for head_dim 64 and 128)
 *   head_dim   32, 64 or 128; n_heads a multiple of n_kv_heads, at most 8
 *              query heads per kv head
 *   k_cache, v_cache  device [batch][n_kv_heads][kv_entries][head_dim]
 *   q          device float [n_rows][n_heads * head_dim] (RoPE applied)
 *   out        device [n_rows][n_heads * head_dim] of dtype
 *   row_*, chain_off, chain   host arrays (n_rows entries; chain_len)
 * Requires 0 <= row_seq < batch, 0 <= row_nc <= row_pos + 1 <= kv_entries,
 * at most 64 chain positions per row (row_pos - row_nc < 64), chain entries
 * in [0, kv_entries) and chain_off[r] + row_pos[r] - row_nc[r] < chain_len;
 * anything else returns DEX_E_INVAL before any launch.  Allocates and frees
 * its own tables and split partials; synchronises hip_stream.            */
dex_status dex_debug_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                               int32_t batch, int32_t kv_entries, const void *k_cache, const void *v_cache,
                               const float *q, int32_t n_rows, const int32_t *row_seq, const int32_t *row_pos,
                               const int32_t *row_nc, const int32_t *chain_off, const int32_t *chain,
                               int32_t chain_len, void *out, void *hip_stream);

/* dex_debug_attention for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): same arguments, same kernels and the same output bits, but
 * the row tables and split partials live in a fixed array of 64 MiB that
 * the library holds on every GPU it runs on until the process ends (the
 * first call on a device resolves that device's copy; the call runs on the
 * current device, which must own hip_stream).  No hipMalloc, hipFree or
 * other allocating routine is called.  Limits: n_rows <= DEX_MAX_ROWS,
 * chain_len <= 16384, and n_rows * n_heads * (max row_pos / 64 + 1) *
 * (head_dim + 2) * 4 bytes of split partials <= 63.75 MiB (at head_dim 128
 * and 32 heads: 8 rows up to 32128 keys each); beyond them
 * the call returns DEX_E_CAPACITY before any device work, with the reason
 * in dex_last_error(NULL).  Every call on one GPU shares that GPU's array:
 * calls that overlap on one GPU (other threads, other streams) race and must
 * be serialised by the caller.  Nothing in the array needs to start at zero
 * (every partial the combine reads is written by the same call).
 * Synchronises hip_stream.                                                  */
dex_status dex_debug_attention_noalloc(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                                       int32_t batch, int32_t kv_entries, const void *k_cache,
                                       const void *v_cache, const float *q, int32_t n_rows,
                                       const int32_t *row_seq, const int32_t *row_pos, const int32_t *row_nc,
                                       const int32_t *chain_off, const int32_t *chain, int32_t chain_len,
                                       void *out, void *hip_stream);

/* The Gumbel source of sampling mode (Algorithm 2 draws one Gumbel row per
 * sampling slot; here the row of a slot is a function of (seed, sequence,
 * position of the slot's input token), so plain autoregressive sampling at
 * the same position draws the same row and the committed tokens equal AR
 * sampling's).  With the SplitMix64 finaliser mix64 and gamma =
 * 0x9E3779B97F4A7C15 (Steele, Lea and Flood, OOPSLA 2014), all mod 2^64:
 *   key = mix64(seed ^ mix64(seq * 2^32 + pos)),
 *   z_v = mix64(key + (v + 1) * gamma),
 *   u_v = ((z_v >> 41) + 1/2) / 2^23      (exact in binary32),
 *   G_v = -ln(-ln u_v)                    (binary32 here).
 * dex_debug_gumbel writes G_0..G_{V-1} of one row to device memory `out`
 * (float32) on `hip_stream`, for tests of the generator.                    */
dex_status dex_debug_gumbel(uint64_t seed, int32_t seq, int32_t pos, int32_t V, float *out, void *hip_stream);

/* Plain device copy of `bytes` (multiple of 16) used to calibrate hardware
 * traffic counters against a kernel of known size.                          */
dex_status dex_debug_copy(void *dst, const void *src, int64_t bytes, void *hip_stream);

/* ---------------------------------------------------------------------------
 * Operators over a paged key/value cache, for programs that bring their own
 * layers: rotary positions and the cache write, attention of one new token,
 * page tables that fork, grow and compact, and beam selection.
 *
 *   - The cache is the caller's device memory: keys and values of a layer are
 *     [n_pages][n_kv_heads][page_size][head_dim] each (16-byte aligned), a
 *     pool of layers [n_layers] of those.  page_size is a power of two, 1 to
 *     1024.  Position p of sequence s is slot p % page_size of page
 *     table[s][p / page_size] (device int32 [n_seqs][max_pages]); an entry
 *     outside [0, n_pages), -1 by custom, is no page.  n_pages * n_kv_heads *
 *     page_size < 2^32 - 1, n_pages <= 2^30, max_pages * page_size <= 2^30.
 *   - All arrays are device memory unless they are called host arrays; all
 *     work is enqueued on hip_stream, which belongs to the current device, and
 *     nothing is allocated, copied to the host or waited for, so every call
 *     can be captured into a graph.  What a call reads on the device (lengths,
 *     tables, parents) may change between replays; its sizes may not.
 *   - Arrays are aligned to their type.  Elements of a strided output do not
 *     overlap each other, and an output overlaps no input unless the call says
 *     that it may.
 *   - Work memory is the caller's: the size that the matching _work function
 *     gives (0: may be NULL), 16-byte aligned, with any contents.  It is free
 *     for another use once the call's work is done; two calls that may overlap
 *     in time (two streams, two graphs) need one each.
 *   - Argument errors return DEX_E_INVAL before anything is launched, with
 *     the reason in dex_last_error(NULL).  Numbers on the device cannot be
 *     refused; each call says what it makes of those that do not fit, and
 *     none reads or writes outside its arrays for them.
 * ------------------------------------------------------------------------- */

/* Rotary positions: pair i of a head, i < rot_dim / 2, turns by position *
 * f_i, f_i = theta^(-2 i / rot_dim), and is scaled by `amplitude`; dimensions
 * from rot_dim on stay as they are.  Pairs are (i, i + rot_dim / 2), or
 * (2 i, 2 i + 1) where interleaved.  `turns` holds f_i / 2 pi in double.     */
typedef struct {
  const double *turns;                  /* device [rot_dim / 2] */
  int32_t rot_dim;                      /* even, 2 .. head_dim */
  int32_t interleaved;
  float amplitude;
} dex_rotary;

enum {
  DEX_ROTARY_PLAIN = 0,
  DEX_ROTARY_LINEAR = 1,                /* f_i / factor (positions interpolated) */
  DEX_ROTARY_BASE = 2,                  /* theta * factor^(rot_dim / (rot_dim - 2)) */
  DEX_ROTARY_BANDS = 3                  /* f_i where it makes at least `fast` turns over the
                                           original context, f_i / factor where at most
                                           `slow`, in proportion between */
};

/* The plan's turns (HOST double [rot_dim / 2]).  factor is read by every
 * scaling but PLAIN; original, slow and fast (0 <= slow < fast) by BANDS.    */
dex_status dex_rotary_turns(int32_t scaling, int32_t rot_dim, double theta, double factor, double original,
                            double slow, double fast, double *turns);

/* Turns queries and keys, or one of them (n_heads or n_kv_heads 0 and null
 * arrays): q_out[r][h] = R(pos[r]) q[r][h].  Element d of head h of row r lies
 * at row * row_stride + h * head_stride + d of its array, strides in elements
 * of dtype.  An output may be its input with the same strides, or memory that
 * overlaps no input.  inverse: turns back, R(-pos), which is also the
 * rotation's gradient (scaled by `amplitude` again, so the two undo each other
 * where that is 1).  Positions are any int32; the angle is formed in double.
 * n_rows * head_dim * (n_heads + n_kv_heads + 8) < 2^35.                     */
dex_status dex_rope(int32_t dtype, int32_t head_dim, const dex_rotary *rotary, int32_t inverse, int32_t n_rows,
                    const int32_t *pos, const void *q, int64_t q_row, int64_t q_head, int32_t n_heads, void *q_out,
                    int64_t q_out_row, int64_t q_out_head, const void *k, int64_t k_row, int64_t k_head,
                    int32_t n_kv_heads, void *k_out, int64_t k_out_row, int64_t k_out_head, void *hip_stream);

/* The cache write of one layer, with the rotation: row r's keys, turned, and
 * its values go to position row_pos[r] of sequence row_seq[r] (NULL: r), its
 * queries, turned, to q_out (n_heads 0 and null arrays: no queries).  rotary
 * NULL: nothing turns.  A row whose position is negative, whose sequence is
 * not in [0, n_seqs) or whose page is not there is left out altogether.  Rows
 * must not share a position of a sequence, nor sequences a page written to
 * (dex_pages_reserve sees to that).  Limits as dex_rope's, with the values'
 * heads.                                                                    */
dex_status dex_pages_append(int32_t dtype, int32_t head_dim, const dex_rotary *rotary, int32_t n_rows,
                            const int32_t *row_seq, const int32_t *row_pos, const void *q, int64_t q_row,
                            int64_t q_head, int32_t n_heads, void *q_out, int64_t q_out_row, int64_t q_out_head,
                            const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                            int64_t v_head, int32_t n_kv_heads, void *k_pages, void *v_pages, int32_t n_pages,
                            int32_t page_size, const int32_t *table, int32_t n_seqs, int32_t max_pages,
                            void *hip_stream);

/* Attention of one new token a row over one layer: row r (sequence
 * row_seq[r], NULL: r) with query head h attends to the keys j < row_len[r]
 * of kv head h / (n_heads / n_kv_heads), with a window only to the last
 * `window` of them (0: all), and only where the page is there:
 *   s_j = scale q.k_j,  out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m),
 *   lse = m + ln sum_j e^(s_j - m)   (float [n_rows][n_heads], or NULL).
 * A row that sees no key (row_len <= 0, a sequence outside [0, n_seqs), no
 * page) gets zeros and -inf.  No row_len exceeds max_len, which sizes the
 * work: a longer one counts as max_len, or as the table's width, for its window
 * too.  head_dim 32, 64 or 128; n_heads a multiple of n_kv_heads, at most 64
 * times it and 8192; q, out and the cache are of dtype, sums, weights and
 * statistics float.  Consecutive `group` rows whose leading pages are the same
 * (the beams of a request) have those read once for several of them: for 32 /
 * (n_heads / n_kv_heads) rows at a time, all of them with keys and with the same
 * first key, in whole steps of 256 keys, 512 past 6144 keys, 1024 past 12288 and
 * so on, the same for all (rows on both sides of such a length share nothing).
 * Any group gives the same bits: a row's depend on its own keys and query
 * alone.                                                                    */
int64_t dex_pages_attention_work(int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                 int32_t max_len, int32_t group);
dex_status dex_pages_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_rows,
                               const int32_t *row_seq, const int32_t *row_len, int32_t max_len, int32_t window,
                               int32_t group, float scale, const void *q, int64_t q_row, int64_t q_head,
                               const void *k_pages, const void *v_pages, int32_t n_pages, int32_t page_size,
                               const int32_t *table, int32_t n_seqs, int32_t max_pages, void *out, int64_t out_row,
                               int64_t out_head, float *lse, void *work, void *hip_stream);

/* Page tables.  ref[p] (int32 [n_pages]) counts the holders of page p: the
 * table rows that list it and any others the caller counts (a cached prefix);
 * 0 is free.  length[s] is the sequence's tokens.  Table entries behind a
 * sequence's pages are -1.  n_seqs <= 1024 and n_seqs * max_pages <= 2^30 for
 * fork and reserve.
 *
 * dex_pages_fork: sequence s becomes a copy of sequence parent[s], sharing its
 * pages, or empty where parent[s] is not in [0, n_seqs).  Sequences that are
 * nobody's parent lose their pages, which are free once ref is 0; so a call
 * with parent[s] = s for some and -1 for others frees the others.  Each output
 * may be its input.                                                         */
dex_status dex_pages_fork(const int32_t *table, const int32_t *ref, const int32_t *length, const int32_t *parent,
                          int32_t n_seqs, int32_t max_pages, int32_t n_pages, int32_t *table_out, int32_t *ref_out,
                          int32_t *length_out, void *hip_stream);

/* Room for n_new[s] >= 0 more tokens (below 0 counts as 0) of every sequence,
 * which may then write positions length[s] .. length[s] + n_new[s] - 1.  Pages
 * are taken lowest number first, for the sequences in order.  A partly filled
 * last page that others hold too is replaced by one of the sequence's own, and
 * (src, dst, tokens) says what dex_pages_copy has to copy before the next
 * write: its first `tokens` slots.  The last of several writers keeps the page
 * if no one else holds it.  Where that page is not there the sequence gets one
 * whose first slots hold whatever they held.  ref has to count every table row
 * that lists a page: one with count 0 is given out again.  Writes
 *   table, ref, length   updated (length[s] += n_new[s]);
 *   pos[s]     the first new position, or -1 (nothing asked, or not granted);
 *   src, dst, tokens     int32 [n_seqs], the copies first, then -1, -1, 0;
 *   state      int32 [4]: copies, pages taken, pages missing, 1 if a sequence
 *              that asks for tokens outgrows the table or has a length below 0.
 * Unless state[2] and state[3] are 0 nothing was granted: table, ref and length
 * stay, every pos is -1 and the list is empty.                              */
dex_status dex_pages_reserve(int32_t *table, int32_t *ref, int32_t *length, const int32_t *n_new, int32_t n_seqs,
                             int32_t max_pages, int32_t n_pages, int32_t page_size, int32_t *pos, int32_t *src,
                             int32_t *dst, int32_t *tokens, int32_t *state, void *hip_stream);

/* Moves the n pages in use (ref > 0) to pages 0 .. n - 1: the i-th of those at
 * or past n goes to the i-th free page before it.  map[p] (int32 [n_pages]) is
 * page p's new number, -1 for a free page; src and dst (int32 [n_pages / 2])
 * list the moves for dex_pages_copy, then -1; state as above: moves, n, 0, 0.
 * table_out and ref_out may be their inputs.                                */
dex_status dex_pages_compact(const int32_t *table, const int32_t *ref, int32_t n_seqs, int32_t max_pages,
                             int32_t n_pages, int32_t *table_out, int32_t *ref_out, int32_t *map, int32_t *src,
                             int32_t *dst, int32_t *state, void *hip_stream);

/* Copies pages of every layer of a pool: entry i, i < min(*count, capacity)
 * (count NULL: capacity), copies the first tokens[i] slots (NULL: all) of page
 * src[i] to page dst[i], keys and values.  An entry with a page outside
 * [0, n_pages) copies nothing.  No page may be a dst twice, or both src and
 * dst.  A head's row of head_dim elements is a multiple of 16 bytes.         */
dex_status dex_pages_copy(int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_pages, int32_t n_kv_heads,
                          int32_t page_size, void *k_pool, void *v_pool, const int32_t *src, const int32_t *dst,
                          const int32_t *tokens, const int32_t *count, int32_t capacity, void *hip_stream);

/* Beam search's selection.  Candidate (beam, token) of a request has total
 * score[beam] + logit - lse(the beam's logits); a finished beam (done, uint8
 * or NULL) has one candidate, (beam, eos) with its score as it is, the others
 * -inf.  A score that is not finite, and logits with a NaN, a +inf or nothing
 * but -inf, make all the beam's totals -inf.  Writes the n_out candidates of
 * largest total, largest first, equal ones by beam and token: parent (row
 * request * beams + beam, as dex_pages_fork takes it), token, score (the
 * total), done (the beam's, or token == eos; NULL: not wanted).  Within a beam
 * candidates are compared by their logits, across beams by totals in double,
 * whose lse is off by at most (9 + 2 E) 2^-24 (E the mean of maximum - logit
 * under the softmax; a few 2^-26 as a rule) and is the same for beams of the
 * same logits, so that these tie.  logits: [requests * beams][vocab] of dtype,
 * rows ld elements apart, any alignment.  beams and n_out 1 .. 64, n_out <=
 * beams * vocab, requests * beams <= 2^20, requests * beams * (vocab / 2048 + 2)
 * <= 2^25; eos in [0, vocab), or -1 (with done NULL): none.                  */
int64_t dex_beam_select_work(int32_t dtype, int32_t requests, int32_t beams, int32_t vocab, int32_t n_out);
dex_status dex_beam_select(int32_t dtype, const void *logits, int64_t ld, int32_t requests, int32_t beams,
                           int32_t vocab, const float *score, const uint8_t *done, int32_t eos, int32_t n_out,
                           int32_t *parent, int32_t *token, float *score_out, uint8_t *done_out, void *work,
                           void *hip_stream);

/* ---------------------------------------------------------------------------
 * Over the same cache: trees of drafted tokens, attention over chosen pages,
 * and eviction by accumulated attention weight.  What is said above of arrays,
 * streams, work memory and refusals holds here too.  head_dim of the attention
 * calls and of bounds and selection is 32, 64 or 128, n_heads a multiple of
 * n_kv_heads, at most 64 times it and 8192, rows * n_heads <= 2^30.  A launch
 * has fewer than 2^32 threads, and a call that would need more is refused: from
 * 2^24 pairs of a row or sequence and a kv head on, or from 2^22 where a pair has
 * 1024 threads or four workgroups.
 * ------------------------------------------------------------------------- */

/* Trees.  Node i < draft (1 to 256) of tree b is a drafted token, parent[b][i]
 * the node it continues: a number in [0, i), anything else makes it a root.
 * mask[b][i] (uint64 [ceil(draft / 64)]): bit j is set if j is node i or one of
 * its ancestors.  depth[b][i] (or NULL): how many ancestors it has.            */
dex_status dex_tree_mask(const int32_t *parent, int32_t n_trees, int32_t draft, uint64_t *mask, int32_t *depth,
                         void *hip_stream);

/* Which path of a tree the model agrees with: a node is accepted if its parent
 * is and its token is target[b][parent], what the model wants there; a root, if
 * its token is root[b] (root NULL: always).  Nodes from n_draft[b] on (NULL:
 * draft) are none.  path[b] lists the nodes from a root to the deepest accepted
 * one, the lowest number of equally deep ones, then -1; count[b] is their
 * number, next[b] the target of the last, root[b] (or -1) if there is none.   */
dex_status dex_tree_accept(const int32_t *parent, const int32_t *token, const int32_t *target, const int32_t *n_draft,
                           const int32_t *root, int32_t n_trees, int32_t draft, int32_t *path, int32_t *count,
                           int32_t *next, void *hip_stream);

/* Attention of the drafted tokens of trees over one layer.  Row b * draft + i is
 * node i of tree b, of sequence tree_seq[b] (NULL: b) with tree_len[b] keys
 * before the tree (a longer one counts as max_len, below 0 as 0); node j's key
 * and value are at position tree_len[b] + j (dex_pages_append puts them there;
 * its rotary position is tree_len[b] + depth, so turn it with dex_rope first;
 * where dex_pages_reserve granted nothing, pos -1, every row_pos of the tree is
 * -1 and its tree_draft 0).
 * The row sees the keys before the tree, and node j's if bit j of mask[b][i] is
 * set, j < tree_draft[b] (NULL: draft), each only where its page is there; the
 * mask may be any, and what it hides has no effect: large values, NaN and
 * infinity neither.  Softmax, out and lse as dex_pages_attention's, in all
 * attention below: a weight under 2^-126 of the row's largest may count as 0 (in
 * bf16 as 2^-132), and an infinite value with such a weight gives infinity or
 * NaN; sums are formed with weights up to 2^8, so values past 2^119 may give
 * infinity.  A row that sees nothing, and the rows from tree_draft[b] on, get zeros
 * and -inf.                                                                   */
int64_t dex_pages_tree_attention_work(int32_t dtype, int32_t n_trees, int32_t draft, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t head_dim, int32_t max_len);
dex_status dex_pages_tree_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_trees,
                                    int32_t draft, const int32_t *tree_seq, const int32_t *tree_len,
                                    const int32_t *tree_draft, int32_t max_len, float scale, const void *q, int64_t q_row,
                                    int64_t q_head, const uint64_t *mask, const void *k_pages, const void *v_pages,
                                    int32_t n_pages, int32_t page_size, const int32_t *table, int32_t n_seqs,
                                    int32_t max_pages, void *out, int64_t out_row, int64_t out_head, float *lse,
                                    void *work, void *hip_stream);

/* Moves tokens inside their sequences, in every layer of a pool: for j <
 * min(count[s], capacity), position first[s] + j (first NULL: 0) of sequence s
 * receives keys and values of its position first[s] + index[j], where index is
 * at index + layer * index_layer + s * index_seq + head * index_head (strides in
 * elements, 0 for what shares a list).  to_table NULL: in place, and an entry
 * with index[j] <= j copies nothing (index[j] = j is there already); otherwise
 * into the pages of to_table [n_seqs][to_pages], which the call does not read.
 * An entry below 0, or without a page on either side, copies nothing.  All reads
 * are of the old contents.  A page written to has no other holder, in the call's
 * table or out of it.  A head's row is a multiple of 16 bytes.                */
dex_status dex_pages_keep(int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_pages, int32_t n_kv_heads,
                          int32_t page_size, void *k_pool, void *v_pool, const int32_t *table, int32_t n_seqs,
                          int32_t max_pages, const int32_t *to_table, int32_t to_pages, const int32_t *first,
                          const int32_t *index, int64_t index_layer, int64_t index_seq, int64_t index_head,
                          int32_t capacity, const int32_t *count, void *hip_stream);

/* Pages behind a sequence's last token (length[s]; below 0 counts as 0) leave its
 * row of the table, whose entries there become -1, and lose a holder.  table_out
 * and ref_out may be their inputs.                                            */
dex_status dex_pages_trim(const int32_t *table, const int32_t *ref, const int32_t *length, int32_t n_seqs,
                          int32_t max_pages, int32_t n_pages, int32_t page_size, int32_t *table_out, int32_t *ref_out,
                          void *hip_stream);

/* Bounds of the keys of a page: bounds[p][h] (of dtype, [2][head_dim], 16-byte
 * aligned) is the least and the largest of its keys in every dimension, over the
 * tokens before length[s]; a NaN is passed over, and NaN alone gives NaN.  Writes
 * those of the pages that hold the last n_new tokens of each sequence (more than
 * it has: all), the others stay.  Sequences that share such a page hold the same
 * number of its tokens.                                                       */
dex_status dex_pages_bounds(int32_t dtype, int32_t head_dim, const void *k_pages, int32_t n_pages, int32_t n_kv_heads,
                            int32_t page_size, const int32_t *table, int32_t n_seqs, int32_t max_pages,
                            const int32_t *length, int32_t n_new, void *bounds, void *hip_stream);

/* The pages to read for each row and kv head h: of the columns of its sequence's
 * table that hold tokens (row_len as dex_pages_attention takes it) and a page,
 * the first `sinks`, the last `recent`, and those of largest score
 *   sum over h's query heads and dimensions of max(q_d least_d, q_d largest_d),
 * of equal ones the first, up to n_select in all.  columns[r][h] [n_select]
 * lists them ascending, then -1.  Scores are in double; a q_d of 0 adds 0, and a
 * score that is NaN counts as infinity.                                       */
int64_t dex_pages_select_work(int32_t n_rows, int32_t n_kv_heads, int32_t page_size, int32_t max_len);
dex_status dex_pages_select(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_rows,
                            const int32_t *row_seq, const int32_t *row_len, int32_t max_len, const void *q, int64_t q_row,
                            int64_t q_head, const void *bounds, int32_t n_pages, int32_t page_size, const int32_t *table,
                            int32_t n_seqs, int32_t max_pages, int32_t n_select, int32_t sinks, int32_t recent,
                            int32_t *columns, void *work, void *hip_stream);

/* dex_pages_attention over the listed columns alone: row r's heads of kv head h
 * see the tokens before row_len[r] of columns[r][h] [n_columns], in any order (a
 * column listed twice counts twice; one outside the table is none).  Of a row
 * only the first ceil(row_len / page_size) entries are read.                  */
int64_t dex_pages_sparse_attention_work(int32_t dtype, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads,
                                        int32_t head_dim, int32_t n_columns, int32_t page_size);
dex_status dex_pages_sparse_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t n_rows, const int32_t *row_seq, const int32_t *row_len, float scale,
                                      const void *q, int64_t q_row, int64_t q_head, const int32_t *columns,
                                      int32_t n_columns, const void *k_pages, const void *v_pages, int32_t n_pages,
                                      int32_t page_size, const int32_t *table, int32_t n_seqs, int32_t max_pages,
                                      void *out, int64_t out_row, int64_t out_head, float *lse, void *work,
                                      void *hip_stream);

/* dex_pages_attention of one new token a row that also adds up what each key was
 * given: weight_out[r][h][j] = weight[r][h][j] + the sum of the softmax weights of
 * key j over the query heads of kv head h, for j < row_len[r] (0 for a key whose
 * page is not there); what lies behind stays.  Rows [n_rows][n_kv_heads] of float,
 * weight_ld and weight_out_ld >= max_len elements apart; weight_out may be weight
 * with the same stride.                                                       */
int64_t dex_pages_weigh_work(int32_t dtype, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                             int32_t max_len);
dex_status dex_pages_weigh(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_rows,
                           const int32_t *row_seq, const int32_t *row_len, int32_t max_len, float scale, const void *q,
                           int64_t q_row, int64_t q_head, const float *weight, int64_t weight_ld, float *weight_out,
                           int64_t weight_out_ld, const void *k_pages, const void *v_pages, int32_t n_pages,
                           int32_t page_size, const int32_t *table, int32_t n_seqs, int32_t max_pages, void *out,
                           int64_t out_row, int64_t out_head, float *lse, void *work, void *hip_stream);

/* Which keys of each sequence and kv head stay: the first `sinks`, the last
 * `recent`, and the heaviest others (of equal ones the first; a NaN counts as
 * infinity), count[s] = min(length[s], capacity, budget) in all.  index[s][h]
 * [budget] lists them ascending, then -1, as dex_pages_keep takes it;
 * weight_out[s][h] [capacity] is their weights in that order, then 0.  weight_out
 * may be weight with the same stride.                                         */
dex_status dex_pages_evict(const float *weight, int64_t weight_ld, int32_t n_seqs, int32_t n_kv_heads, int32_t capacity,
                           const int32_t *length, int32_t budget, int32_t sinks, int32_t recent, int32_t *index,
                           int32_t *count, float *weight_out, int64_t weight_out_ld, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DEX_H */
