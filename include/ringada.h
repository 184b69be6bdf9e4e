/*
 * ringada.h -- C ABI of the RingAda per-stage hot path on AMD MI355X (gfx950).
 *
 * One ring client of RingAda (arXiv 2502.19864) hosts a contiguous run of
 * frozen transformer blocks (the Trm layers of Sec. III-A) each carrying two
 * bottleneck adapters h <- h + sigma(h W_down) W_up (Eq. (1)), one after the
 * attention sublayer and one after the feed-forward sublayer.  Per training
 * iteration the client
 *   - applies its blocks to the activations handed over by the previous
 *     client and passes the result on (Sec. II-B and Sec. III-B,
 *     "Forward and Backward Propagation");
 *   - relays the gradient handed back by the next client down through its
 *     frozen weights, producing weight gradients for unfrozen adapters only,
 *     and stops at the lowest unfrozen adapter (Alg. 1: the backward ends at
 *     the (L-d+1)-th adapter; Sec. III-B: the terminator);
 *   - updates its unfrozen adapters (Sec. III-B).
 * A client may not forward a new batch while the update of its unfrozen
 * adapters for the previous batch is pending (Sec. III-B: unfrozen clients keep
 * the one-forward-one-backward order; Sec. III-B "three-fold advantages": no
 * stale weights).
 *
 * Conventions used by every call
 *   - All tensor pointers are DEVICE pointers unless stated otherwise.
 *   - Activations are row-major [batch, seq, d_model] in the stage dtype
 *     (RINGADA_F32: float, RINGADA_BF16: bfloat16 bit patterns in uint16).
 *     Arithmetic accumulates in fp32 for both dtypes.
 *   - Weights are row-major [in, out]: a projection is x @ W, as in Eq. (1).
 *   - stream is a hipStream_t passed as void* (NULL = the null stream).  Calls
 *     enqueue kernels and return; they never synchronise the device, except
 *     ringada_stage_bind_block and ringada_prof_end as documented.
 *   - Errors are returned as a status; the message of the last failing call on
 *     the calling thread is available from ringada_last_error().  The library
 *     never aborts and never prints.
 *   - The library allocates no device memory, in any call.  Every device
 *     buffer is the caller's: frozen weights, adapter masters and gradients,
 *     the activation stash and scratch (ringada_stage_plan), and the regions
 *     that hold what the library derives from the weights
 *     (ringada_stage_plan_weights).
 */
#ifndef RINGADA_H
#define RINGADA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  RINGADA_OK = 0,
  RINGADA_E_INVALID = 1,     /* a NULL pointer, a size out of range, an unknown enum */
  RINGADA_E_STATE = 2,       /* call out of order: see the state machine below */
  RINGADA_E_WORKSPACE = 3,   /* stash or scratch smaller than ringada_stage_plan says */
  RINGADA_E_UNSUPPORTED = 4, /* a shape or option this build has no kernel for */
  RINGADA_E_HIP = 5          /* a HIP runtime call failed (message has the HIP error) */
} ringada_status;

enum {
  /* post-LN encoder block (BERT shape): bias on every projection, GELU FFN,
   * bidirectional attention, LayerNorm after each residual add */
  RINGADA_ARCH_POSTLN_GELU = 0,
  /* pre-RMSNorm decoder block (LLaMA shape): no biases, SwiGLU FFN, RoPE
   * (rotate-half pairs (i, i + d_head/2)), causal attention */
  RINGADA_ARCH_PRERMS_SWIGLU = 1
};
enum { RINGADA_F32 = 0, RINGADA_BF16 = 1 };
enum {
  /* two adapters per block: one on the attention sublayer's output, one on
   * the FFN sublayer's output, each before the block's residual add */
  RINGADA_PLACEMENT_HOULSBY = 0,
  /* the single serial adapter of Sec. II-A (Fig. 1): one adapter per block,
   * on the FFN sublayer's output; the attention sublayer carries none */
  RINGADA_PLACEMENT_FFN = 1
};

typedef struct {
  int32_t arch;       /* RINGADA_ARCH_* */
  int32_t dtype;      /* RINGADA_F32 or RINGADA_BF16 storage */
  int32_t n_blocks;   /* L, blocks held by this stage, >= 1 */
  int32_t d_model;    /* d; bf16 path: a multiple of 256 up to 1024, or of
                         1024 up to 4096 */
  int32_t n_heads;    /* d_head = d_model / n_heads; bf16 path: d_head 64 or 128 */
  int32_t d_ffn;      /* F; bf16 path: multiple of 64 */
  int32_t d_adapter;  /* m, the bottleneck of Eq. (1); bf16 path: 64 */
  int32_t max_batch;  /* upper bounds for batch and seq of later calls */
  int32_t max_seq;
  float norm_eps;     /* LayerNorm / RMSNorm epsilon (added to the variance) */
  float rope_theta;   /* RoPE base, pre-RMS arch only */
  int32_t placement;  /* RINGADA_PLACEMENT_*: where the adapters sit */
} ringada_stage_desc;

/* Frozen weights of one block, device pointers in the stage dtype, all
 * row-major [in, out].  Pointers marked (post-LN) must be NULL for the pre-RMS
 * arch and non-NULL for the post-LN arch.  The norm gains and shifts
 * (norm1_g, norm1_b, norm2_g, norm2_b) must be 16-byte aligned
 * (ringada_stage_bind_block returns RINGADA_E_INVALID otherwise).  The memory
 * is borrowed: it must stay valid and unchanged until ringada_stage_destroy. */
typedef struct {
  const void* w_qkv;   /* [d, 3d]; output columns are [Q | K | V], head h owns
                          columns [h*d_head, (h+1)*d_head) of each */
  const void* b_qkv;   /* [3d] (post-LN) */
  const void* w_o;     /* [d, d] */
  const void* b_o;     /* [d] (post-LN) */
  const void* norm1_g; /* [d] LN1 gamma (post-LN) or RMSNorm-1 gain (pre-RMS) */
  const void* norm1_b; /* [d] LN1 beta (post-LN) */
  const void* w_in;    /* post-LN: W_i [d, F]; pre-RMS: [d, 2F] = [W_gate | W_up] */
  const void* b_in;    /* [F] (post-LN) */
  const void* w_out;   /* [F, d] */
  const void* b_out;   /* [d] (post-LN) */
  const void* norm2_g; /* [d] LN2 gamma or RMSNorm-2 gain */
  const void* norm2_b; /* [d] LN2 beta (post-LN) */
} ringada_block_weights;

/* One adapter of Eq. (1) (no biases): fp32 master weights and fp32 gradient
 * accumulators, device, caller-owned, borrowed until ringada_stage_destroy.
 * The backward ADDS into g_down/g_up; ringada_adapter_step consumes and zeroes
 * them.  g_down and g_up must be 16-byte aligned (ringada_stage_bind_block
 * returns RINGADA_E_INVALID otherwise); the bf16 backward sums each gradient
 * element in a fixed order, so equal inputs give bitwise equal gradients.
 * Adapters of one stage may share g_down and g_up (the backward then adds every
 * one's gradient); ringada_adapter_step takes all four tensors of each adapter
 * as its own, so a stage that shares any updates them some other way. */
typedef struct {
  float* w_down; /* [d, m] */
  float* w_up;   /* [m, d] */
  float* g_down; /* [d, m] */
  float* g_up;   /* [m, d] */
} ringada_adapter;

typedef struct {
  int32_t kind; /* 0 = SGD: w <- w - lr * g (the only optimiser of this build) */
  float lr;
} ringada_optim;

typedef struct ringada_stage ringada_stage;

/* ---------------------------------------------------------------- planning */

/* Host only (no device call).  Bytes of the activation stash and of the
 * scratch workspace that a forward + backward of (batch, seq) with cut-off
 * lowest_unfrozen needs.  The stash holds, for blocks l >= lowest_unfrozen, only
 * the tensors the early-stopped backward reads (Alg. 1: nothing below the
 * cut-off is back-propagated, so nothing below it is kept); blocks below the
 * cut-off and a fully frozen stage (lowest_unfrozen >= n_blocks) stash nothing.
 * Either output pointer may be NULL.  lowest_unfrozen < 0 stashes every block. */
ringada_status ringada_stage_plan(const ringada_stage_desc* desc, int32_t batch,
                                  int32_t seq, int32_t lowest_unfrozen,
                                  size_t* stash_bytes, size_t* scratch_bytes);

/* Host only.  Maps the unfreezing depth of Alg. 1 to the lowest_unfrozen
 * argument of a stage holding 0-indexed global blocks
 * [first_block, first_block + n_local) of an n_tm-block model.  The backward
 * ends at the (n_tm - depth + 1)-th block (1-indexed); Sec. III-B: a client
 * whose last block lies below it is forward-only (returns n_local), the one
 * holding it is the terminator (returns its local index), clients above it
 * return -1 (cut-off upstream: they must produce the input gradient).
 * Returns INT32_MIN for invalid arguments. */
int32_t ringada_local_cutoff(int32_t n_tm, int32_t depth, int32_t first_block,
                             int32_t n_local);

/* ---------------------------------------------------------------- lifetime */

/* Host only.  Bytes of the caller memory that holds what the library
 * derives from the weights:
 *   block_bytes: per block, passed to ringada_stage_bind_block: a transposed
 *     copy of each frozen projection matrix ([out, in], so that both operands
 *     of every forward product are contiguous along the contraction; post-LN
 *     bf16 stages with d_head 64 keep the QKV rows, and a copy of the QKV
 *     bias, in per-head order [Q_h K_h V_h]; pre-RMS stages interleave the
 *     gate and up rows in 32-row groups) and the adapters' working copies in
 *     the stage dtype (W_down, W_up and their transposes, fragment-packed in
 *     bf16 stages), 4 d m elements per adapter;
 *   stage_bytes: per stage, passed to ringada_stage_create: the rotary
 *     (cos, sin) table of the pre-RMS arch, max_seq x d_head/2 float pairs
 *     (0 for the post-LN arch).
 * Either output pointer may be NULL. */
ringada_status ringada_stage_plan_weights(const ringada_stage_desc* desc,
                                          size_t* block_bytes, size_t* stage_bytes);

/* Validates desc and creates a handle on the current HIP device.  stage_mem:
 * device memory of at least the stage_bytes of ringada_stage_plan_weights
 * (may be NULL when that is 0), 256-byte aligned, owned by the caller and
 * borrowed until ringada_stage_destroy; the first ringada_stage_bind_block
 * fills it.  Allocates nothing; RINGADA_E_WORKSPACE if stage_mem is too
 * small. */
ringada_status ringada_stage_create(const ringada_stage_desc* desc, void* stage_mem,
                                    size_t stage_mem_bytes, ringada_stage** out);

/* Binds block `block` (0-indexed, local).  Frozen weights and the adapters
 * are borrowed; under RINGADA_PLACEMENT_FFN attn_adapter must be NULL (the
 * block has none), otherwise both are required.  block_mem: device memory of
 * at least the block_bytes of ringada_stage_plan_weights, 256-byte aligned,
 * owned by the caller, borrowed until ringada_stage_destroy; the library
 * writes into it the transposed projections (the frozen weights never
 * change, so the copies stay valid) and the adapters' working copies, which
 * every ringada_adapter_step refreshes.  Fills it on `stream` and
 * synchronises the stream before returning.  Allocates nothing;
 * RINGADA_E_WORKSPACE if block_mem is too small.  Binding a block again
 * replaces its bindings. */
ringada_status ringada_stage_bind_block(ringada_stage* st, int32_t block,
                                        const ringada_block_weights* frozen,
                                        const ringada_adapter* attn_adapter,
                                        const ringada_adapter* ffn_adapter,
                                        void* block_mem, size_t block_mem_bytes,
                                        void* stream);

/* Re-derives the adapter working copies from the fp32 masters (call after
 * writing the masters directly, e.g. when loading a checkpoint). */
ringada_status ringada_stage_sync_adapters(ringada_stage* st, void* stream);

/* Releases the handle (host memory only; every device buffer stays the
 * caller's). */
void ringada_stage_destroy(ringada_stage* st);

/* ---------------------------------------------------------------- options of a stage
 * Both are set on a handle after ringada_stage_create, hold for every later forward
 * and backward until they are set again, and return RINGADA_E_STATE while a forward
 * is pending its backward. */

/* Attention of every block with a sliding window, sinks and a relative position
 * bias; the fields are those of ringada_attn_desc and ringada_attn_tensors (no lengths: every
 * row of a batch counts, as in the plain attention).  One table
 * serves all blocks; g_table (NULL: a frozen table) is ADDED into by the backward,
 * over the blocks whose attention it passes.  The memory is borrowed until the
 * options are set again or the stage is destroyed. */
typedef struct {
  int32_t window, sinks;
  int32_t n_buckets, max_distance;
  const float* table;     /* [n_buckets, n_heads], NULL when n_buckets is 0 */
  const int32_t* bucket;  /* [2 max_distance + 1] */
  float* g_table;
  void* workspace;        /* at least the bytes of ringada_stage_plan_attention, 256-byte aligned */
  size_t workspace_bytes;
} ringada_stage_attention;

/* Host only.  Bytes of opt->workspace that a forward and backward of (batch, seq)
 * need; only the integers of opt and whether g_table is NULL are looked at. */
ringada_status ringada_stage_plan_attention(const ringada_stage_desc* desc,
                                            const ringada_stage_attention* opt, int32_t batch,
                                            int32_t seq, size_t* workspace_bytes);

/* opt NULL, or without a window and buckets: the plain attention.  A forward whose
 * (batch, seq) needs a larger workspace returns RINGADA_E_WORKSPACE. */
ringada_status ringada_stage_set_attention(ringada_stage* st, const ringada_stage_attention* opt);

/* Dropout with probability p (0: none) on each sublayer's output, before its
 * adapter and the residual add (ringada_dropout's masks, with site first_site + 2 l for
 * block l's attention sublayer and first_site + 2 l + 1 for its FFN).  The backward
 * reads rng again: {seed, offset} must stay as its forward found them until it has
 * run.  Forwards of a frozen stage drop too. */
ringada_status ringada_stage_set_dropout(ringada_stage* st, float p, const uint64_t* rng,
                                         uint32_t first_site);

/* ---------------------------------------------------------------- hot path */

/* Forward through all n_blocks blocks: y = blocks(x), x and y [batch, seq, d]
 * (x and y must not overlap).  lowest_unfrozen = c selects what is stashed
 * for the backward (see ringada_stage_plan); stash/scratch are caller buffers
 * of at least the planned sizes and must stay untouched until the matching
 * backward has been enqueued.
 * State machine: with c < n_blocks the handle becomes "pending" and every
 * further forward (a frozen one included) returns RINGADA_E_STATE until
 * ringada_stage_backward has been called; with c >= n_blocks (frozen stage)
 * nothing is left pending, so such forwards may follow each other. */
ringada_status ringada_stage_forward(ringada_stage* st, void* stream,
                                     const void* x, void* y, int32_t batch,
                                     int32_t seq, int32_t lowest_unfrozen,
                                     void* stash, size_t stash_bytes,
                                     void* scratch, size_t scratch_bytes);

/* Early-stopped backward of the pending forward.  dy [batch, seq, d] is the
 * gradient at the stage output.  For blocks l >= max(c, 0), from the top
 * down: activation gradients through the frozen weights (no frozen weight
 * gradient is formed) and the adapters' weight gradients, ADDED into their
 * g_down / g_up.  With 0 <= c < n_blocks the pass ends after the lowest
 * adapter of block c (its weight gradients are the last thing computed):
 * the attention adapter, or under RINGADA_PLACEMENT_FFN the FFN adapter, so
 * that block's FFN, norms and attention are not back-propagated at all;
 * with c < 0 the gradient w.r.t. the stage input is written to dx_in.
 * dx_in must be non-NULL iff c < 0.  c must be >= the forward's cut-off
 * (else RINGADA_E_STATE: the stash does not reach that deep), and < n_blocks.
 * Clears the pending state. */
ringada_status ringada_stage_backward(ringada_stage* st, void* stream,
                                      const void* dy, int32_t lowest_unfrozen,
                                      void* dx_in);

/* Update of the unfrozen adapters (blocks l >= max(c, 0)) from their
 * accumulated gradients (Sec. III-B: clients with unfrozen adapters update
 * them), then zero the gradients and refresh the working copies.  Returns
 * RINGADA_E_STATE while a forward is pending its backward (the backward
 * must see the weights the forward used). */
ringada_status ringada_adapter_step(ringada_stage* st, void* stream,
                                    int32_t lowest_unfrozen,
                                    const ringada_optim* opt);

/* ---------------------------------------------------------------- initiator helpers
 * Alg. 1: the initiator computes the loss on the last block's output and
 * updates the head; these produce the dy that enters the backward. */

/* Mean squared error over n elements: dy = 2 (y - target) / n, *loss = mean.
 * y, target, dy in `dtype`; loss is one device float (may be NULL).  dy may be
 * y or target itself; any other overlap with them returns RINGADA_E_INVALID.
 * In place the call runs on one compute unit: far slower for large tensors (3.1 M
 * bf16 elements: 200 us against 6).  While a call with a loss runs, the first 4 KB
 * of dy may hold partial sums. */
ringada_status ringada_loss_mse(void* stream, int32_t dtype, const void* y,
                                const void* target, int64_t n, void* dy,
                                float* loss);

/* Linear head on position 0 of each sequence + softmax cross-entropy, mean
 * over the batch.  y, dy: [batch, seq, d] in `dtype` (dy is fully written:
 * zero except position 0); w_h [d, n_classes] and b_h [n_classes] fp32;
 * labels [batch] int32 in [0, n_classes); the fp32 gradients g_wh, g_bh and
 * the mean loss (one device float, may be NULL) are ADDED into: zero them
 * before the first call of an accumulation.  n_classes <= 16; d a multiple of
 * 8; y, dy and w_h 16-B aligned.  dy may be y itself; any other overlap with
 * position 0 of a sequence of y returns RINGADA_E_INVALID.  In place one compute
 * unit forms all rows of position 0: slower (32 samples, d 768, two classes: 9 us
 * against 6; 128 samples, d 4096: 101 against 40, with 16 classes 3.9 ms against
 * 0.1).  Every sum runs over the samples in a fixed
 * order: the same inputs give the same bits. */
ringada_status ringada_head_ce(void* stream, int32_t dtype, const void* y,
                               int32_t batch, int32_t seq, int32_t d,
                               const float* w_h, const float* b_h,
                               int32_t n_classes, const int32_t* labels,
                               void* dy, float* g_wh, float* g_bh, float* loss);

/* w <- w - lr * g; g <- 0, over n fp32 values (the head update). */
ringada_status ringada_sgd_f32(void* stream, float* w, float* g, int64_t n,
                               float lr);

/* ---------------------------------------------------------------- block operators
 * Attention, dropout, norms, the rotary embedding and the vocabulary head as calls of
 * their own, for blocks and heads that are put together outside a stage;
 * ringada_stage_set_attention and ringada_stage_set_dropout use the same kernels inside one. */

/* A [batch, row, head, d_head] tensor: strides in elements, d_head contiguous.
 * bf16: strides multiples of 8 and data 16-byte aligned; f32: any alignment of a
 * float. */
typedef struct {
  void* data;
  int64_t batch, row, head;
} ringada_view;

typedef struct {
  int32_t dtype;          /* RINGADA_F32 or RINGADA_BF16 */
  int32_t batch;
  int32_t n_heads;        /* query heads, a multiple of n_kv_heads: head h reads */
  int32_t n_kv_heads;     /* key-value head h / (n_heads / n_kv_heads) */
  int32_t d_head;         /* bf16: 64 or 128; f32: 1 .. 128 */
  int32_t seq_q, seq_k;   /* rows per sequence in q / o and in k / v */
  int32_t causal;         /* 1: a query sees no key after its own position */
  int32_t window;         /* 0: none, else a query sees the keys less than this far away */
  int32_t sinks;          /* and, with a window, the first so many keys however far */
  float scale;            /* of q.k, > 0 */
  int32_t n_buckets;      /* relative position bias: 0 = none, else 1 .. 65535 */
  int32_t max_distance;   /* R, 0 .. 1024: distances beyond count as R */
} ringada_attn_desc;

/* Query row i of a sequence with len_q queries and len_k keys stands at position
 * p = len_k - len_q + i, key row j at j (a new token's query: at the end of its
 * cache).  With table, bucket[clamp(j - p, -R, R) + R] names the table row whose
 * entry for the head is added to the score.  A row that sees nothing, and one at or past
 * its length, gives zeros (and lse -inf).  Rows of k, v and gradients at or past the
 * lengths are not read into any result, whatever they hold.  An infinity or NaN within the
 * lengths of k, v, q or dout may reach rows of its sequence that do not see it (0 times it). */
typedef struct {
  ringada_view q, k, v;   /* [batch, seq_q, n_heads, d_head]; [batch, seq_k, n_kv_heads, d_head] */
  ringada_view o;         /* as q: written by the forward, read by the backward */
  float* lse;             /* [batch, n_heads, seq_q]: base-2 log-sum-exp of the scores, written by the
                             forward (may be NULL there), read by the backward */
  const int32_t* len_q;   /* device [batch], NULL: seq_q; values are taken into [0, seq_q] */
  const int32_t* len_k;   /* device [batch], NULL: seq_k; values are taken into [0, seq_k] */
  const float* table;     /* device [n_buckets, n_heads]; an entry of -1e30 or less hides its bucket.  Scores
                             are held in fp32: beside an entry of 1e6 they are good to 1/16 */
  const int32_t* bucket;  /* device [2 R + 1], values taken into [0, n_buckets) */
} ringada_attn_tensors;

typedef struct {
  ringada_view dout;        /* as o */
  ringada_view dq, dk, dv;  /* as q, k, v; written, zeros at and past the lengths */
  float* dtable;            /* [n_buckets, n_heads], ADDED into; NULL: the table is frozen */
} ringada_attn_grads;

/* Host only.  Bytes of the workspaces of one forward and one backward (0: none needed);
 * with_dtable: whether the backward forms the table's gradient.  Either pointer may be
 * NULL.  Calls that may run at the same time (other streams, other graphs) take
 * workspaces of their own. */
ringada_status ringada_attn_plan(const ringada_attn_desc* desc, int32_t with_dtable,
                                 size_t* forward_bytes, size_t* backward_bytes);

/* o = softmax(scale q k^T + bias, visible keys) v.  Sums and the softmax are held in fp32.  With
 * bf16 tensors P (here and in the backward) and dS are rounded to bf16 on their way into a
 * product, and the backward takes D = sum of dout o from the stored o unless it forms the
 * table's gradient; with fp32 ones nothing is rounded to fewer bits.  Outputs must not overlap inputs.
 * Workspaces are 256-byte aligned and overlap nothing else. */
ringada_status ringada_attn_forward(void* stream, const ringada_attn_desc* desc,
                                    const ringada_attn_tensors* t, void* workspace,
                                    size_t workspace_bytes);

/* Gradients of ringada_attn_forward with the same desc and tensors.  Every sum has
 * a fixed order: the same inputs give the same bits.  No gradient may overlap what is
 * read or another gradient. */
ringada_status ringada_attn_backward(void* stream, const ringada_attn_desc* desc,
                                     const ringada_attn_tensors* t, const ringada_attn_grads* g,
                                     void* workspace, size_t workspace_bytes);

/* Host only.  Fills map[2 max_distance + 1], indexed by key - query + max_distance, with
 * the usual buckets of learned relative positions: of the n buckets of a direction
 * (half of n_buckets each when bidirectional, the keys after the query in the second
 * half; else all for the keys before it, the keys after it in bucket 0), the first
 * n / 2 hold one distance each, the others distances spaced evenly in their
 * logarithm up to max_distance, which is in the last with everything beyond. */
ringada_status ringada_relpos_buckets(int32_t n_buckets, int32_t max_distance,
                                      int32_t bidirectional, int32_t* map);

/* y = [res +] dropout(x) over n <= 2^35 contiguous elements of `dtype`: an element is zeroed
 * with probability p (0 <= p < 1, in steps of 2^-16), else multiplied by 1 / (1 - p).
 * The mask is a function of (seed, offset, site, element) alone and is stored nowhere:
 * the backward is the same call on dy, without res.  rng: {seed, offset}, two
 * uint64 in device memory, read when the kernel runs, so a captured graph takes
 * a new mask from a new offset; site tells apart the calls that share them.  Element e
 * takes 16-bit half e % 2 (low first) of word e % 8 / 2 of Philox4x32-10 with key seed
 * and counter (e / 8, site, offset), and is dropped when that is below 65536 p.  res may be
 * NULL; y may be x or res; any other overlap returns RINGADA_E_INVALID. */
ringada_status ringada_dropout(void* stream, int32_t dtype, const void* x, const void* res,
                               void* y, int64_t n, float p, const uint64_t* rng, uint32_t site);

/* Rows of d elements, d contiguous; the stride in elements (of no account with one row). */
typedef struct {
  void* data;
  int64_t row;
} ringada_rows;

enum { RINGADA_NORM_LAYER = 0, RINGADA_NORM_RMS = 1 };
typedef struct {
  int32_t dtype; /* RINGADA_F32 or RINGADA_BF16 */
  int32_t kind;  /* RINGADA_NORM_* */
  int64_t rows;
  int32_t d;     /* 1 .. 16384 */
  float eps;     /* added to the variance (the mean square), >= 0 */
} ringada_norm_desc;

/* y = (s - mean(s)) rstd gain + shift with rstd = 1 / sqrt(var(s) + eps), or for RINGADA_NORM_RMS
 * y = s / sqrt(mean(s^2) + eps) gain + shift; s = x, or with res s = x + res rounded to `dtype` and written to
 * sum (res and sum are given together or both NULL).  gain [d] and shift [d] (NULL: none) in `dtype`; stats [rows, 2]
 * floats (NULL: not wanted), 8-byte aligned: mean (0 for RMS) and rstd, which the backward reads.  Any alignment of an
 * element and any stride; 16-byte aligned rows whose d and strides are multiples of 16 bytes are read
 * faster.  Squares of s are formed in fp32: s of 2^60 and more overflows them.  y and sum may each be x or res, not both the same tensor; any other overlap of an output is refused
 * (RINGADA_E_INVALID).  Arithmetic and sums in fp32, one rounding each of s and y.  A row with an infinity or NaN
 * gives NaN in that row alone. */
ringada_status ringada_norm_forward(void* stream, const ringada_norm_desc* desc, const ringada_rows* x,
                                    const ringada_rows* res, const ringada_rows* sum, const void* gain,
                                    const void* shift, const ringada_rows* y, float* stats);

/* Host only.  Bytes of the workspace of a backward that forms dgain or dshift (without them: none needed). */
ringada_status ringada_norm_plan(const ringada_norm_desc* desc, size_t* backward_bytes);

/* Gradients of ringada_norm_forward with the same desc, gain and stats; sum is what it normalised (x where there
 * was no res).  dx is the gradient of s, so of x and of res: the norm's, plus dskip (NULL: none), what reaches
 * s past the norm.  dgain and dshift [d] floats are ADDED into; NULL: frozen.  dx may be dy, dskip or sum; any other
 * overlap of an output is refused.  Every sum has a fixed order: the same inputs give the same bits. */
ringada_status ringada_norm_backward(void* stream, const ringada_norm_desc* desc, const ringada_rows* dy,
                                     const ringada_rows* dskip, const ringada_rows* sum, const void* gain,
                                     const float* stats, const ringada_rows* dx, float* dgain, float* dshift,
                                     void* workspace, size_t workspace_bytes);

typedef struct {
  int32_t dtype;       /* RINGADA_F32 or RINGADA_BF16 */
  int32_t batch, rows;
  int32_t n_heads;     /* of q, 1 .. 2048 */
  int32_t n_kv_heads;  /* of k; 0: there is no k */
  int32_t d_head;      /* 2 .. 1024 */
  int32_t n_axes;      /* 1 .. 4 */
  int32_t section[4];  /* pairs that each axis turns, P in all, 2 P <= d_head */
  int32_t inverse;     /* 1: by the opposite angles (the backward: the same call on the gradients) */
} ringada_rotary_desc;

/* Rotary embedding of q [batch, rows, n_heads, d_head] and k [batch, rows, n_kv_heads, d_head]: pair (i, i + P) of a head
 * turns by positions[axis of pair i][batch][row] * freq[i] radians (the pairs of the stages' RoPE);
 * dimensions from 2 P on are copied.  Axis 0 has the first section[0] pairs, axis 1 the next, and so on.
 * positions: int32 [n_axes, batch, rows], any values; freq: double [P]; both device.  Angles are formed in 64 bits, the
 * rotation in fp32 with one rounding.  q_out may be q and k_out may be k (the same data and
 * strides); any other overlap of an output is refused.  k and k_out are NULL when n_kv_heads is 0.  Pairs and d_head that
 * are multiples of 8 (f32: of 4), with 16-byte aligned data and strides, go 16 bytes at a time, others one element: six times
 * slower and more. */
ringada_status ringada_rotary(void* stream, const ringada_rotary_desc* desc, const ringada_view* q,
                              const ringada_view* k, const int32_t* positions, const double* freq,
                              const ringada_view* q_out, const ringada_view* k_out);

/* Host only.  The usual frequencies: theta^(-j / section) for the j-th pair of each axis, or with shared
 * theta^(-i / P) for pair i of all.  freq: double [P] host, P <= 512. */
ringada_status ringada_rotary_frequencies(int32_t n_axes, const int32_t* section, double theta, int32_t shared,
                                          double* freq);

typedef struct {
  int32_t dtype; /* RINGADA_F32 or RINGADA_BF16 */
  int32_t rows;  /* 1 .. 2^23 */
  int32_t d;     /* 1 .. 16384; bf16: a multiple of 8 */
  int32_t vocab; /* 1 .. 2^22 */
} ringada_vocab_desc;

/* h, dh [rows, d]; w, dw [vocab, d] in the stage dtype: a row per class, as in an embedding table, so that a tied one can be
 * passed (unlike the stages' [in, out] weights).  bf16: 16-byte aligned, strides multiples of 8; strides at most 2^22. */
typedef struct {
  ringada_rows h, w;
  const int32_t* labels; /* [rows]; a row with a label outside [0, vocab) does not count */
  float* loss;           /* [rows] */
  float* lse;            /* [rows] */
  const float* dloss;    /* [rows]: the gradient that arrives at each row's loss; NULL: no gradients */
  ringada_rows dh, dw;   /* written; data NULL: not wanted (a frozen head takes dh alone) */
} ringada_vocab_tensors;

/* Host only.  Bytes of the workspaces of ringada_vocab_ce without and with gradients, and of ringada_vocab_next.
 * The logits are held for a piece of the rows at a time, at most 2 GiB of them (or 256 rows), beside a copy of h, 8 bytes (ringada_vocab_next: 12)
 * for every 32 logits and 4 for every 16384, up to 64 MiB for sums that several workgroups share (over 2^18 classes or rows: one dh or dw in fp32 for each 2^18 of
 * them), and, for rows of more than one piece in bf16, 4 vocab d bytes.  Up to 32 rows of bf16 without gradients whose h fits the LDS (15 at
 * d 4096, 7 at 8192, 3 at 16384) take 4 KiB a row (ringada_vocab_next: 6) and no copy.  Any pointer may be NULL. */
ringada_status ringada_vocab_plan(const ringada_vocab_desc* desc, size_t* forward_bytes, size_t* train_bytes,
                                  size_t* next_bytes);

/* Softmax cross entropy of the logits s = h w^T, and its gradients in the same call:
 *   lse = log sum exp s,  loss = lse - s[label],  P = dloss (softmax(s) - onehot(label)),  dh = P w,  dw = P^T h.
 * A row that does not count has loss 0, lse 0 and a zero row in dh; its h and dloss are read into nothing, whatever they
 * hold.  Logits, softmax and sums are fp32.  With bf16 tensors:
 *  - the logits wait for their row's lse in fp16, as their distance to the largest of 64 or 128 (off by 2^-11 of it);
 *  - P is rounded to bf16 on its way into the products; of at most 64 rows that count in a piece, to two bf16, whose own error is 2^-16;
 *  - what a row of the stored P falls short of its sum, zero, is added at w[label] in fp32: its errors reach dh as
 *    their products with w - w[label], and what all classes have in common stays out;
 *  - P is in units of the first counted row's |dloss|, where that is within 2^-40 and 2^40: entries of dloss may be up to 2^80
 *    then.
 * An infinity or NaN in a row that counts gives NaN in it, and in dw.  A class whose logit is -infinity by an infinity in w is left
 * out; +infinity makes the row NaN, and dw; either leaves NaN or infinities in that column of dh.  No output may overlap
 * anything else.  Every sum has a fixed order: the same inputs give the same bits. */
ringada_status ringada_vocab_ce(void* stream, const ringada_vocab_desc* desc, const ringada_vocab_tensors* t,
                                void* workspace, size_t workspace_bytes);

/* The class of the largest logit of every row of h (of equal ones the lowest; NaN logits are passed over, and a row of
 * nothing else gives some class in range) and its log-probability, s[token] - lse, NaN where s[token] is infinite. */
ringada_status ringada_vocab_next(void* stream, const ringada_vocab_desc* desc, const ringada_rows* h,
                                  const ringada_rows* w, int32_t* token, float* logprob, void* workspace,
                                  size_t workspace_bytes);

/* ---------------------------------------------------------------- diagnostics */

/* Thread-local message of the last failing call ("" if none). */
const char* ringada_last_error(void);

/* Per-kernel timing with HIP events.  After ringada_prof_begin every launch
 * the handle makes is bracketed by two events on its stream; ringada_prof_end
 * synchronises those events and returns, per kernel name, the number of
 * launches, their summed duration and the summed algorithmic work (FLOPs of
 * the contraction; minimum HBM bytes read + written). */
typedef struct {
  char name[64];
  int32_t launches;
  double total_ms;
  double flops;
  double bytes;
} ringada_prof_entry;

ringada_status ringada_prof_begin(ringada_stage* st);
ringada_status ringada_prof_end(ringada_stage* st, ringada_prof_entry* out,
                                int32_t max_entries, int32_t* n_entries);

#ifdef __cplusplus
}
#endif
#endif /* RINGADA_H */
