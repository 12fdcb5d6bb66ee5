/*
 * lif.h - C ABI of the MI355X (gfx950) sparse-FFN hot path of "LLM in a flash"
 * (arXiv 2312.11514): per-token FFN inference over predicted-active neurons held
 * in an HBM neuron cache that is fed from pinned host memory (standing in for flash).
 *
 * One handle (lif_layer) = one FFN layer.  Per token (or per batch of tokens) the
 * caller issues, on one HIP stream and without any host synchronisation,
 *
 *     lif_predict -> lif_update_window -> lif_load_bundles -> lif_sparse_ffn
 *
 * All counts (added / removed neurons, rows in use) stay on the device, so the four
 * calls chain without a host round trip and can be captured into a HIP graph.
 *
 * Conventions
 *   - Plain C; every call returns a status (LIF_OK = 0).  No call blocks or
 *     synchronises except lif_get_state, lif_get_counters and lif_profile_collect.
 *   - "device" pointers are HBM addresses valid on the GPU that is current when
 *     lif_create is called; "host" pointers are CPU addresses.  Streams are passed
 *     as void* holding a hipStream_t (NULL = the default stream).
 *   - The library allocates no device memory: every array, including the scratch
 *     workspace, is owned by the caller and must outlive the handle.
 *   - Element type E is fp32 (LIF_F32) or IEEE fp16 (LIF_F16).  G = 2 vectors per
 *     bundle (up row | down column), G = 3 for gated layers (gate row | up row | down column).
 *   - Shape limits: d_model, rank multiples of 8 (fp16) or 4 (fp32); d_ffn a multiple
 *     of 8 and at most 65536; rank at most 2048; max_batch at most 8; window_k at most 256.
 *   - A device-detected error (capacity overflow, or a lost launch: see lif_state.error) sets a
 *     sticky flag: until lif_reset every hot call becomes a no-op on the device; lif_get_state
 *     reports the flag.
 *   - Calls on one handle must not overlap (one stream at a time).
 */
#ifndef LIF_H
#define LIF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lif_layer lif_layer;

enum lif_status {
    LIF_OK = 0,
    LIF_INVALID_ARG = 1,   /* null pointer, unsupported shape, batch > max_batch */
    LIF_BAD_STATE = 2,     /* calls out of order (see lif_update_window / lif_load_bundles) */
    LIF_CAPACITY = 3,      /* reported by lif_get_state: active set exceeded capacity_rows */
    LIF_HIP_ERROR = 4      /* a HIP runtime call failed; see lif_last_error_string (lif_state.error: a lost launch) */
};

enum lif_dtype { LIF_F32 = 0, LIF_F16 = 1, LIF_BF16 = 2 /* bfloat16: key-value caches only */ };

/* How lif_sparse_ffn reads the cache (Section 3.3, inference over the cached rows). */
enum lif_ffn_mode {
    LIF_FFN_SKIP_DEAD = 0, /* do not read the down column of rows whose activation is zero */
    LIF_FFN_FULL_BUNDLE = 1 /* read every cached bundle completely */
};

/* What decides which neurons are predicted active (step 1). */
enum lif_predictor {
    LIF_PRED_LOWRANK = 0,  /* low-rank predictor (x A) B + c > theta (Section 3.1, Fig. 3b)               */
    LIF_PRED_GATE = 1      /* the resident gate projection itself (Appendix, Llama 2, "Alternative         */
                           /* approaches"): mask_i = gate_i . x + b_i > theta, exact; bundles = up | down; */
                           /* y_t = sum_s relu(gate . x_t + b)_s * (up_s . x_t) * down_s; glu = 0; batches */
                           /* and passes of several tokens as with the low-rank predictor                  */
};

typedef struct lif_config {
    int32_t d_model;        /* d: length of the up row and of the down column              */
    int32_t d_ffn;          /* F: number of intermediate neurons of the layer              */
    int32_t rank;           /* r: rank of the low-rank predictor (Section 3.1, Fig. 3b)    */
    int32_t window_k;       /* k: sliding window in steps, current step included (Fig. 4b) */
    int32_t capacity_rows;  /* rows preallocated in the cache ("Req_i", Section 3.3)       */
    int32_t max_batch;      /* largest batch of tokens per step (1..8)                     */
    int32_t glu;            /* 0: bundle = up|down, 1: bundle = gate|up|down               */
    int32_t dtype;          /* enum lif_dtype: type of x, y, A, B and the bundles          */
    int32_t ffn_mode;       /* enum lif_ffn_mode                                           */
    int32_t shrink_window;  /* 1: dynamic window (Appendix, Persimmon / Phi-2): when the active  */
                            /* set would exceed capacity_rows the oldest masks leave the window  */
                            /* until it fits; 0: such a step is a LIF_CAPACITY error             */
    int32_t predictor;      /* enum lif_predictor                                          */
    float threshold;        /* theta: neuron i is predicted active iff logit_i > theta     */
} lif_config;

typedef struct lif_buffers {
    /* predictor (device, read-only): logits = (x A) B + c                               */
    const void* A;          /* LIF_PRED_LOWRANK: the first predictor matrix stored with the */
                            /* contraction dimension contiguous, [rank x d_model] row-major, E */
                            /* (row j = column j of the paper's d_model x rank matrix);     */
                            /* LIF_PRED_GATE: the gate projection [d_ffn x d_model]         */
                            /* row-major, E (row i = gate weights of neuron i)              */
    const void* B;          /* [rank x d_ffn] row-major, E; unused (may be NULL) with       */
                            /* LIF_PRED_GATE                                                */
    const float* c;         /* [d_ffn] per-neuron offset, fp32; may be NULL (= 0)         */
    /* bias of the ReLU'd projection per original neuron (device, read-only)             */
    const float* b;         /* [d_ffn] fp32                                               */
    /* bundle store: PINNED HOST memory (hipHostMalloc or equivalent), read-only         */
    const void* host_bundles; /* [d_ffn x G*d_model] E, row i = (gate_i |) up_i | down_i   */
    /* neuron cache (device, read-write; Section 3.3 "matrix", "pointers", "bias")       */
    void* matrix;           /* [capacity_rows x G*d_model] E                              */
    int32_t* pointers;      /* [capacity_rows] slot -> original neuron id                 */
    float* bias;            /* [capacity_rows] fp32                                       */
    /* scratch (device, read-write), at least lif_workspace_bytes(cfg) bytes, 256-aligned; it
     * also holds the window state ("last_k_active": the last window_k step masks) and the
     * device-resident counts                                                             */
    void* workspace;
    size_t workspace_bytes;
    /* optional second part of the bundle store (PINNED HOST memory, read-only), normally NULL.  If set, the store is
     * NOT bundled (the layout that Section 3.2's bundling replaces, kept for measuring what bundling buys):
     * host_bundles then holds only the activation vectors, [d_ffn x (G-1)*d_model] E (row i = (gate_i |) up_i), and
     * host_down the down columns, [d_ffn x d_model] E; every new neuron costs two reads.  The cache rows, and so
     * every result, are the same as with the bundled store. */
    const void* host_down;
} lif_buffers;

typedef struct lif_state {
    int32_t num_used;       /* rows of the cache in use                                   */
    int32_t step;           /* number of completed lif_update_window calls since reset    */
    int32_t error;          /* LIF_OK, LIF_CAPACITY or LIF_HIP_ERROR, sticky until lif_reset.  LIF_HIP_ERROR: workgroups of
                             * a lif_sparse_ffn call of one launch did not run for about a second while others of it
                             * waited for them.  That call's y is complete; later calls do nothing                */
    int32_t last_added;     /* |added| of the last lif_update_window                      */
    int32_t last_removed;   /* |removed| of the last lif_update_window                    */
    int32_t last_moved;     /* rows moved by the last deletion                            */
    int32_t window_len;     /* step masks in the window after the last update (<= window_k) */
} lif_state;

typedef struct lif_counters {
    uint64_t steps;         /* lif_update_window calls that committed                     */
    uint64_t added;         /* sum of |added|                                             */
    uint64_t removed;       /* sum of |removed|                                           */
    uint64_t rows_moved;    /* rows rewritten inside the cache by deletions               */
    uint64_t h2d_bytes;     /* bytes read from the host bundle store                      */
    uint64_t ffn_calls;     /* lif_sparse_ffn calls                                       */
    uint64_t ffn_rows;      /* sum over those calls of the rows in use                    */
    uint64_t ffn_active;    /* sum over those calls of the rows with a non-zero activation */
} lif_counters;

/* Kernels timed by the profiling hooks, in the order of lif_profile_collect's arrays. */
enum lif_kernel_id {
    LIF_K_PREDICT_XA = 0,   /* t = x A                                                    */
    LIF_K_PREDICT_MASK = 1, /* logits = t B + c, threshold, pack                          */
    LIF_K_WINDOW = 2,       /* window diff, added / removed ids, deletion plan            */
    LIF_K_LOAD = 3,         /* row moves + host-to-device bundle append                   */
    LIF_K_FFN_UP = 4,       /* activations of all cached rows                             */
    LIF_K_FFN_DOWN = 5,     /* y = sum of activation x down column; a call of one launch  */
    LIF_K_COUNT = 6
};

/* Bytes of scratch lif_create needs for this configuration (0 if cfg is invalid). */
size_t lif_workspace_bytes(const lif_config* cfg);

/*
 * Build a layer handle over caller-owned arrays (Section 3.3: everything is
 * preallocated once).  Validates shapes and alignment, records the device alias of
 * the pinned bundle store, and enqueues nothing: call lif_reset before the first step.
 * Errors: LIF_INVALID_ARG (null/unsupported), LIF_HIP_ERROR (bundle store is not
 * device-accessible pinned memory).
 */
int lif_create(const lif_config* cfg, const lif_buffers* buf, lif_layer** out);

/* Frees the host-side handle only (never the caller's arrays). NULL is accepted. */
int lif_destroy(lif_layer* layer);

/*
 * Empty the cache (Section 3.3: num_used starts at zero): num_used = 0, every
 * window empty, step = 0, error flag and counters cleared.  Enqueued on `stream`; does
 * not touch the matrix contents.
 */
int lif_reset(lif_layer* layer, void* stream);

/*
 * Step 1, low-rank predictor (Section 3.1 "Anticipating ReLU Sparsity", Fig. 3b;
 * active = positive output, Section 3.1 "The Sliding Window Technique").
 *   x_dev          [batch x d_model] E, device, read-only
 *   masks_dev      [batch x d_ffn/8] bytes, device, written: bit (i mod 8) of byte i/8
 *                  of row t is 1 iff ((x_t A) B)_i + c_i > threshold
 *   step_mask_dev  [d_ffn/8] bytes, device, 8-byte aligned, written: OR of the batch's masks;
 *                  may equal masks_dev when batch == 1
 * Sums are accumulated in fp64 so the decision does not depend on summation order
 * beyond ~1e-15 relative.  NaN logits compare false (inactive).
 */
int lif_predict(lif_layer* layer, const void* x_dev, int32_t batch,
                uint8_t* masks_dev, uint8_t* step_mask_dev, void* stream);

/*
 * Step 2, sliding window (Section 3.1 "The Sliding Window Technique", Fig. 4b).
 * With S_t = union of the last window_k step masks (this one included):
 *   added_dev    [d_ffn] int32, device, written: S_t \ S_{t-1}, ascending neuron id
 *   removed_dev  [d_ffn] int32, device, written: S_{t-1} \ S_t, ascending neuron id
 *   n_added_dev, n_removed_dev  [1] int32, device, written: the two counts
 * Records the mask in the window state and advances the step counter.  If |S_t| would exceed
 * capacity_rows: with shrink_window = 0 nothing is changed, both counts are written as 0 and
 * the sticky error flag is set to LIF_CAPACITY; with shrink_window = 1 the oldest masks are
 * dropped from the window for good, one by one, until the union fits (S_t = union of the
 * newest window_len masks, window_len maximal), and only a step mask that does not fit on
 * its own is a LIF_CAPACITY error.
 * Must alternate with lif_load_bundles (LIF_BAD_STATE otherwise): the cache has to
 * hold S_{t-1} when the window moves.
 */
int lif_update_window(lif_layer* layer, const uint8_t* step_mask_dev,
                      int32_t* added_dev, int32_t* n_added_dev,
                      int32_t* removed_dev, int32_t* n_removed_dev, void* stream);

/*
 * Step 2 for a verification pass of speculative decoding (Section 4.3 "Speculative Decoding";
 * Appendix, related work on speculative decoding: the window then moves by several tokens at once).
 *   masks_dev  [n_tokens x d_ffn/8] bytes, device, 8-byte aligned: the per-token masks of the
 *              pass (as written by lif_predict with batch = n_tokens); d_ffn % 64 == 0
 *   keep       0..n_tokens: the first `keep` tokens (those expected to be accepted; the paper's
 *              choice is about alpha * (lambda + 1) for acceptance ratio alpha) enter the window,
 *              one entry per token, exactly as if pushed one after the other; the masks of the
 *              remaining tokens are needed for this pass only and leave with the next update.
 * The cache must hold, for this pass, the union of the last window_k kept token masks and of
 * the transient masks: added / removed are the difference to what it holds now.  If that exceeds
 * capacity_rows: with shrink_window = 0 a LIF_CAPACITY error; with shrink_window = 1 the oldest window
 * masks leave for good, one by one, until the masks of the pass and the remaining window fit (only a
 * pass whose own masks do not fit is a LIF_CAPACITY error).  Alternates with
 * lif_load_bundles like lif_update_window; follow with lif_sparse_ffn(batch = n_tokens).
 */
int lif_update_window_tokens(lif_layer* layer, const uint8_t* masks_dev, int32_t n_tokens, int32_t keep,
                             int32_t* added_dev, int32_t* n_added_dev, int32_t* removed_dev,
                             int32_t* n_removed_dev, void* stream);

/*
 * Step 3, cache update (Section 3.3 items 1 and 2, Fig. 6; bundles per Section 3.2).
 * Deletion: with c = *n_removed_dev and n' = num_used - c, the rows whose neuron left
 * the window are overwritten by the last rows: the j-th lowest dead slot below n'
 * receives the j-th highest live slot at or above n' (matrix row, pointer and bias
 * move together; at most c rows move).  Insertion: the bundle of the j-th added
 * neuron a_j is read from host_bundles[a_j] and written to row n' + j, with
 * pointers[n'+j] = a_j and bias[n'+j] = b[a_j]; num_used = n' + *n_added_dev.
 * The arguments must be the arrays written by the preceding lif_update_window.
 * Adds |added| x bundle bytes to the h2d_bytes counter.  LIF_BAD_STATE if no
 * lif_update_window is pending.
 */
int lif_load_bundles(lif_layer* layer, const int32_t* added_dev, const int32_t* n_added_dev,
                     const int32_t* removed_dev, const int32_t* n_removed_dev, void* stream);

/*
 * Step 4, FFN over the cached rows (Section 3.3 item 3):
 *   y_t = sum_{s < num_used} relu(up_s . x_t + bias_s) * down_s
 *   gated:  y_t = sum_s relu(gate_s . x_t + bias_s) * (up_s . x_t) * down_s
 * over every row in use (the whole window union).  Products of E-typed values,
 * fp32 accumulation, y rounded once to E.
 *   x_dev  [batch x d_model] E, device, read-only
 *   y_dev  [batch x d_model] E, device, overwritten (zeros when the cache is empty)
 * The summation order is fixed (slot order within fixed strides), so results are
 * reproducible run to run bit for bit.
 */
int lif_sparse_ffn(lif_layer* layer, const void* x_dev, int32_t batch, void* y_dev, void* stream);

/*
 * lif_sparse_ffn for callers that cannot allocate and want no scratch of their own in the call: code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation.  Same arguments, same arithmetic
 * and bit-identical results; the activations and the partial outputs of the call (the scratch that
 * lif_sparse_ffn keeps in the layer's workspace if it takes more than one launch) live in a static device array
 * inside the library instead, of lif_static_scratch_bytes() = 5 MiB, which every GPU the library runs on holds until
 * the process ends.  The call allocates nothing and frees nothing.
 *   limit   256-byte-rounded 4 * batch * capacity_rows  +  4 * 32 * batch * d_model  <=  lif_static_scratch_bytes()
 *           (batch 8 at d_model 4096 fits up to 32768 rows, a single token at any shape); beyond it LIF_INVALID_ARG,
 *           nothing is launched
 *   errors  as lif_sparse_ffn; LIF_HIP_ERROR if the array's address could not be obtained on the layer's device
 * All layers on one GPU share the array: calls that overlap on one GPU (different streams, different layers)
 * race on it; calls on one stream are safe.  Nothing in the array has to be cleared between calls (every value a
 * call reads was written by that call), and its contents after a call are unspecified.
 */
int lif_sparse_ffn_static(lif_layer* layer, const void* x_dev, int32_t batch, void* y_dev, void* stream);

/* Size in bytes of the static scratch array behind lif_sparse_ffn_static. */
size_t lif_static_scratch_bytes(void);

/*
 * One whole step in one call: lif_predict, lif_update_window, lif_load_bundles and
 * lif_sparse_ffn on the same x, with the same arguments, results and error behaviour as the
 * four calls in sequence.  The cache update and the activation stage of the FFN share one
 * launch: the host-link gather keeps few compute units busy, the others compute the
 * activations of the resident rows meanwhile (Section 3.3 items 2 and 3 overlapped).  For
 * batch == 1 the predictor is part of that launch too; the loaders compute the activations of
 * the rows they write, with the same summation order.  y, masks, ids,
 * counts and the cache are bit-identical to the four-call sequence.
 */
int lif_step(lif_layer* layer, const void* x_dev, int32_t batch, void* y_dev, uint8_t* masks_dev,
             uint8_t* step_mask_dev, int32_t* added_dev, int32_t* n_added_dev, int32_t* removed_dev,
             int32_t* n_removed_dev, void* stream);

/*
 * One speculative verification pass in one call (Section 4.3): lif_predict on the n_tokens
 * consecutive tokens of x, lif_update_window_tokens with keep_tokens, lif_load_bundles and
 * lif_sparse_ffn, with the same arguments, results and error behaviour as those four calls in
 * sequence, and the same shared launches as lif_step.
 */
int lif_step_tokens(lif_layer* layer, const void* x_dev, int32_t n_tokens, int32_t keep_tokens, void* y_dev,
                    uint8_t* masks_dev, uint8_t* step_mask_dev, int32_t* added_dev, int32_t* n_added_dev,
                    int32_t* removed_dev, int32_t* n_removed_dev, void* stream);

/*
 * Performance hint: the number of rows the cache
 * typically holds (for example the mean num_used of an earlier run).  lif_sparse_ffn and the fused steps then
 * launch that many waves and let each request its first row before the device-side row
 * count has arrived.  0 removes the hint.  Results never depend on it.
 */
int lif_set_expected_rows(lif_layer* layer, int32_t rows);

/*
 * Performance knob of the bundle gather (Section 3.3 item 2) in lif_step, lif_step_tokens and lif_load_bundles: pairs of
 * loader waves, one bundle in flight per pair, 1..64; 0 restores the default.  The default comes from the bundle size,
 * as many pairs as keep so many bytes of host reads outstanding, and at least 5:
 *   a step of one token            320 KiB, at most 32 pairs; vectors of at most 2 KiB (a pair then has two bundles in
 *                                  flight): 256 KiB, at most 64 pairs; vectors of more than 12 KiB: 20 pairs
 *   a step or pass of several      768 KiB, at most 48 pairs
 *   lif_load_bundles               640 KiB, at most 32 pairs
 * Results never depend on it.
 */
int lif_set_loader_pairs(lif_layer* layer, int32_t pairs);

/*
 * Performance knob of the single-token lif_step and lif_sparse_ffn: workgroups of one launch hand values over to each
 * other, and a workgroup that has polled for a value this often without success computes it itself (0: it never
 * waits).  Results never depend on it.
 */
int lif_set_handoff_polls(lif_layer* layer, int32_t polls);

/* Synchronises `stream`, then copies the device-side state / counters to the host. */
int lif_get_state(lif_layer* layer, lif_state* out, void* stream);
int lif_get_counters(lif_layer* layer, lif_counters* out, void* stream);

/*
 * Per-kernel timing with HIP events recorded on the caller's stream around every
 * kernel of the hot calls.  lif_profile_begin(layer, max_launches) creates the events
 * (host objects only) and switches timing on; lif_profile_collect synchronises the
 * stream, adds up elapsed milliseconds and launch counts per enum lif_kernel_id into
 * ms[LIF_K_COUNT] / launches[LIF_K_COUNT], destroys the events and switches timing off.
 * Launches beyond max_launches are not timed.
 */
int lif_profile_begin(lif_layer* layer, int32_t max_launches);
int lif_profile_collect(lif_layer* layer, double* ms, int64_t* launches, void* stream);

/*
 * Bandwidth reference of the box, for the roofline figures of a benchmark (not part of the method): one launch of a
 * plain streaming-read kernel over [src_dev, src_dev + bytes) (16-byte loads, every byte read once, nothing
 * written unless the folded words hit one magic value: sink_dev, 4 bytes of device memory, is then written).
 * bytes = 0 launches an empty kernel (the launch floor).  src_dev 16-byte aligned, bytes a multiple of 16.
 */
int lif_profile_read(const void* src_dev, size_t bytes, void* sink_dev, void* stream);

/*
 * Cost reference of the box for a benchmark (not part of the method): what it costs to hand the results of all
 * workgroups of a kernel to one workgroup of the same launch instead of to a second launch.  One launch of 256
 * workgroups that read 16 KiB each and produce 8 bytes (the shape of the mask kernel of lif_predict).
 *   mode 0  no hand-off (the plain kernel)
 *   mode 1  every workgroup passes a device-scope fence and takes a ticket, the last to arrive reads the 2 KiB back;
 *           no workgroup waits
 *   mode 2  no fences: results go out as 64-bit words carrying `stamp`, by relaxed device-scope atomic stores, and
 *           workgroup 0 polls them with relaxed device-scope atomic loads; the wait is bounded (it gives up after
 *           20000 polls per word and counts that in the 32-bit word at scratch + 256 * 16384 + 4100)
 *   scratch_dev  device memory, 256-byte aligned, lif_profile_handoff_bytes() bytes, zeroed once before the first call;
 *                calls on one scratch must not overlap
 *   stamp        mode 2: a value no earlier launch on this scratch has used (and not 0)
 */
int lif_profile_handoff(void* scratch_dev, int32_t mode, uint32_t stamp, void* stream);
size_t lif_profile_handoff_bytes(void);

/*
 * ---- Attention beside the FFN: a paged key-value cache -----------------------------------------------------------------
 *
 * The attention weights stay resident (Section 3, selective persistence); what a decode step needs beside them is the
 * cache of keys and values.  One handle (lif_kv) = the cache of a stack of attention layers.  Per decode step the caller
 * issues, on one HIP stream and without any host synchronisation,
 *
 *     lif_kv_reserve  ->  for every layer:  lif_kv_append -> lif_kv_attend
 *
 * and lif_kv_truncate, lif_kv_fork, lif_kv_compact between steps.  Lengths, tables and counts stay on the device, every
 * launch has a geometry that does not depend on them, so a step can be captured into a HIP graph.
 *
 *   - A sequence is a slot 0..max_seqs-1.  Its tokens 0..lengths[slot]-1 lie in the pages table[slot][0..]; a page holds
 *     page_tokens tokens of all layers.  refs[page] counts the table entries that name a page; a page with none is free.
 *   - E is fp32, fp16 or bfloat16, n = 16 / sizeof(E) elements make 16 bytes.
 *       keys    [layers][pages][kv_heads][page_tokens][head_dim]          E
 *       values  [layers][pages][kv_heads][page_tokens / n][head_dim][n]   E   (n consecutive tokens of one dimension together)
 *   - The tokens of a step are the last fresh[slot] tokens of their sequence.  A call takes `batch` rows of up to n_tokens
 *     tokens; row i belongs to slot slots[i] (slots == NULL: slot i), its token t < fresh is at position length - fresh + t,
 *     its tokens t >= fresh are padding: their outputs are zeros.  A slot number outside 0..max_seqs-1 makes a row of padding.
 *     A slot must not appear in two rows of a lif_kv_append.
 *   - Shape limits: head_dim a multiple of 8, 8..256; heads a multiple of kv_heads; page_tokens 16, 32, 64, 128 or 256;
 *     pages at most 2^24; max_seqs at most 1024; max_pages at most 2^20; max_tokens at most 256.
 *   - A device-detected error (lif_kv_state.error) is sticky: until lif_kv_truncate (LIF_CAPACITY, LIF_INVALID_ARG) or
 *     lif_kv_reset (any) the other calls do nothing on the device, so a step that did not get its pages writes none.
 *   - The library allocates no device memory.  Calls on one handle must not overlap (one stream at a time).
 */
typedef struct lif_kv lif_kv;

enum lif_norm { LIF_NORM_NONE = 0, LIF_NORM_RMS = 1, LIF_NORM_LAYER = 2 };
enum lif_rotary { LIF_ROTARY_HALF = 0, LIF_ROTARY_INTERLEAVED = 1 };
/* Frequencies of the rotated pairs for contexts longer than the trained one (lif_rope_frequencies). */
enum lif_rope_scaling {
    LIF_ROPE_PLAIN = 0,    /* f_i = base^(-2i / rotary_dim)                                                          */
    LIF_ROPE_LINEAR = 1,   /* positions divided by `factor`: f_i / factor                                            */
    LIF_ROPE_BASE = 2,     /* the base raised so that the slowest pair turns `factor` times slower, the fastest as    */
                           /* before: base * factor^(rotary_dim / (rotary_dim - 2))                                  */
    LIF_ROPE_RAMP = 3      /* by the turns w_i = trained * f_i / 2 pi a pair makes over the trained length: pairs of at */
                           /* least `fast` turns keep f_i, of at most `slow` turns get f_i / factor, linear between   */
};

typedef struct lif_kv_config {
    int32_t layers;         /* attention layers that share the tables                            */
    int32_t heads;          /* query heads                                                       */
    int32_t kv_heads;       /* heads of keys and values; query head h reads head h / (heads / kv_heads) */
    int32_t head_dim;
    int32_t page_tokens;
    int32_t pages;
    int32_t max_seqs;
    int32_t max_pages;      /* pages of a sequence at most: the width of the table               */
    int32_t max_tokens;     /* new tokens per sequence and call at most                          */
    int32_t dtype;          /* enum lif_dtype: queries, keys, values, outputs                    */
    int32_t norm;           /* enum lif_norm: of every query and key head                        */
    int32_t rotary;         /* enum lif_rotary: pairs (i, i + rotary_dim / 2) or (2i, 2i + 1)    */
    int32_t rotary_dim;     /* the first rotary_dim dimensions turn: 0 (none) .. head_dim; a multiple of 16 (half), of 2 (interleaved) */
    float norm_eps;
    float rotary_scale;     /* factor on the rotated dimensions (1: a plain rotation)            */
    float scale;            /* of the scores, positive; 1 / sqrt(head_dim) as a rule             */
} lif_kv_config;

typedef struct lif_kv_buffers {
    void* k;                /* device, the layouts above, 16-byte aligned                        */
    void* v;
    int32_t* table;         /* device [max_seqs x max_pages]; -1 where no page is                */
    int32_t* lengths;       /* device [max_seqs]                                                 */
    int32_t* fresh;         /* device [max_seqs]                                                 */
    int32_t* refs;          /* device [pages]                                                    */
    const double* frequencies; /* device [rotary_dim / 2]: angle per position of a pair; NULL if rotary_dim is 0 */
    void* workspace;        /* device, lif_kv_workspace_bytes(cfg) bytes, 256-byte aligned       */
    size_t workspace_bytes;
} lif_kv_buffers;

typedef struct lif_kv_state {
    int32_t used_pages;
    int32_t error;          /* LIF_OK; LIF_CAPACITY: pages or table columns did not suffice (the call changed nothing); */
                            /* LIF_INVALID_ARG: a lif_kv_fork on slots that it cannot take (it changed nothing);        */
                            /* LIF_BAD_STATE: lif_kv_adopt found tables that do not fit the cache (reset it)            */
    int32_t moved_pages;    /* pages copied by the last lif_kv_fork, lif_kv_compact or lif_kv_reserve               */
} lif_kv_state;

/* Rows of a lif_kv_append: row r = i * n_tokens + t is token t of batch row i, its heads one after the other at r * stride. */
typedef struct lif_kv_rows {
    const void* q;          /* [heads x head_dim] E per row                                      */
    const void* k;          /* [kv_heads x head_dim] E per row                                   */
    const void* v;
    void* q_out;            /* [heads x head_dim] E per row, written                             */
    int64_t q_stride, k_stride, v_stride, q_out_stride;  /* elements between rows, multiples of 16 bytes */
    const float* q_weight;  /* [head_dim] fp32, device; NULL: ones.  Unused without a norm       */
    const float* q_bias;    /* [head_dim] fp32; NULL: zeros.  LIF_NORM_LAYER only                */
    const float* k_weight;
    const float* k_bias;
    const int32_t* positions; /* device [batch x n_tokens], angles of rotation; NULL: the position in the sequence */
    const int32_t* slots;   /* device [batch] or NULL                                            */
    int32_t batch;
    int32_t n_tokens;
} lif_kv_rows;

/* Rows of a lif_kv_attend, laid out the same. */
typedef struct lif_kv_query {
    const void* q;          /* [heads x head_dim] E per row                                      */
    void* out;              /* [heads x head_dim] E per row, written                             */
    float* lse;             /* [batch x n_tokens x heads] fp32, written: log of the sum of e^score (-inf: nothing visible); or NULL */
    int64_t q_stride, out_stride;
    const int32_t* slots;   /* device [batch] or NULL                                            */
    const int32_t* starts;  /* device [batch]: first visible position; NULL: 0                   */
    const uint64_t* tree;   /* device [batch x n_tokens], n_tokens <= 64: bit u of word t: new token t sees new token u;
                             * NULL: it sees those with u <= t                                   */
    int32_t batch;
    int32_t n_tokens;
    int32_t window;         /* positions more than window - 1 before a token's own are not visible to it; 0: all are */
} lif_kv_query;

/*
 * Bytes of scratch lif_kv_create needs for this configuration (0 if cfg is invalid).  Most of it is for the parts of lif_kv_attend's sums, and grows with
 * max_tokens * heads / kv_heads up to some 64 rows a workgroup: 32 heads of 128 on 8 take 4 MB for 1 token, 17 for 5, 38 for 64, 151 for 256.
 */
size_t lif_kv_workspace_bytes(const lif_kv_config* cfg);

/* As lif_create: validates, enqueues nothing; call lif_kv_reset (or write the tables and call lif_kv_adopt) first. */
int lif_kv_create(const lif_kv_config* cfg, const lif_kv_buffers* buf, lif_kv** out);
int lif_kv_destroy(lif_kv* kv);

/* No sequences, all pages free, no error.  The pages' contents are not touched. */
int lif_kv_reset(lif_kv* kv, void* stream);

/*
 * Takes over table, lengths and fresh as the caller has written them (a cache that was filled elsewhere): counts refs, finds
 * the free pages, writes -1 behind the pages in use.  Lengths, fresh counts (0..length) or pages out of range: LIF_BAD_STATE.
 */
int lif_kv_adopt(lif_kv* kv, void* stream);

/*
 * Pages for counts[slot] more tokens of every slot (device [max_seqs]; negative counts as 0): lengths grow, fresh[slot] =
 * counts[slot].  The lowest free pages are taken, by slot and then by position.  Where tokens are added to a partly filled
 * page that other sequences hold too (possible after a truncation into forked pages), the slot gets a copy of it first, in the
 * same order; a page that everyone has left that way is free after the call.
 * Too few pages, or more than max_pages for a sequence: LIF_CAPACITY, nothing changes.
 * All new tokens of a slot belong to the lif_kv_append and lif_kv_attend calls up to the next lif_kv_reserve; of more than a call's n_tokens the
 * first n_tokens are taken.
 */
int lif_kv_reserve(lif_kv* kv, const int32_t* counts_dev, void* stream);

/*
 * Shortens every slot to lengths[slot] tokens (device [max_seqs]; negative or beyond its length: unchanged; 0 ends the sequence).
 * Pages no longer named by any table entry are free again; fresh = 0 for all slots.  Clears LIF_CAPACITY and LIF_INVALID_ARG.
 */
int lif_kv_truncate(lif_kv* kv, const int32_t* lengths_dev, void* stream);

/*
 * Slot dst[i] becomes a copy of slot src[i], i < n <= max_seqs (device arrays): it shares the full pages (refs + 1) and gets a
 * copy of the partly filled last one, in the lowest free pages, by i.  fresh[dst] = 0.  A destination must be empty and named once;
 * sources are read as they were before the call.  Otherwise, or for numbers out of range: LIF_INVALID_ARG, nothing changes; too
 * few pages: LIF_CAPACITY, nothing changes.
 */
int lif_kv_fork(lif_kv* kv, const int32_t* src_dev, const int32_t* dst_dev, int32_t n, void* stream);

/*
 * Makes the pool dense: with U pages in use, the j-th lowest free page below U receives the j-th highest used page at or
 * above U (contents of all layers, refs, table entries).  Afterwards pages 0..U-1 are in use.
 */
int lif_kv_compact(lif_kv* kv, void* stream);

/*
 * Queries and keys: norm per head, then rotation (both in fp32, angle = position * frequency in fp64, rounded once to E); keys and values
 * go to their pages of `layer`, queries to q_out.
 *   RMS    x / sqrt(mean x^2 + eps) * weight            LAYER  (x - mean) / sqrt(var + eps) * weight + bias
 *   rotation by a of a pair (x, y): (x cos a - y sin a, x sin a + y cos a) * rotary_scale
 * q_out may be q itself with the same stride, and must not overlap it otherwise (LIF_INVALID_ARG), nor k or v.
 */
int lif_kv_append(lif_kv* kv, int32_t layer, const lif_kv_rows* rows, void* stream);

/*
 * Attention of the new tokens over their sequences' cached tokens (their own included):
 *   out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m),   s_j = scale * q . k_j,  over the visible positions j
 * position j of a sequence of n tokens, f of them new, is visible to new token t iff  starts <= j,  j > n - f + t - window (if a
 * window is given), and j < n - f or new token j - (n - f) is visible to t (tree, or causal).  Nothing visible: zeros.
 * Keys and values at positions that a token does not see never reach its output, whatever they hold.  out may be q itself with the same stride, and
 * must not overlap it otherwise (LIF_INVALID_ARG).
 * batch * kv_heads * steps of a full table row (128 positions of 16-bit elements, 64 of fp32) must stay below 2^31.
 * Scores, sums and outputs are accumulated in fp32 and rounded once to E; the weights e^(s_j - m) are rounded to E for the product with the
 * values.  Every sum has a fixed order for given lengths (and hint): results are reproducible bit for bit.
 */
int lif_kv_attend(lif_kv* kv, int32_t layer, const lif_kv_query* query, void* stream);

/*
 * Performance hint for lif_kv_attend: cached tokens of a sequence as a rule; 0 (the default): as many as a table row holds.  Decides in
 * which blocks rows and positions are taken where a key head has 4 rows or more (tokens times the query heads that share it), and with that
 * the order of their sums: results may differ in the last bits.  Worth setting where tables are much wider than sequences (5 tokens of 4 sequences of
 * 1000, 32 heads on 8, in tables for 32768: 11.5 us with it, 15.0 without).
 */
int lif_kv_set_expected_tokens(lif_kv* kv, int32_t tokens);

/* Synchronises `stream`, then copies the device-side state to the host. */
int lif_kv_get_state(lif_kv* kv, lif_kv_state* out, void* stream);

/*
 * Frequencies of the rotated pairs, host only: out[0 .. rotary_dim / 2).  rotary_dim a positive even number, base > 0; factor > 0 for the
 * scaled kinds (LIF_ROPE_BASE: rotary_dim > 2); LIF_ROPE_RAMP: trained > 0, fast > slow.
 */
int lif_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double trained, double slow, double fast,
                         double* out);

/*
 * ---- What stays resident beside them: norms with the residual's addition, and projections with weights in 4 bits -----------------
 *
 * The attention weights, the output head and the norms are not streamed (Section 3, selective persistence); weights in 4 bits leave the memory to the
 * neuron cache.  Per half of a layer the caller issues, on one HIP stream,
 *
 *     lif_add_norm  ->  lif_packed_multiply (queries, keys and values)  ->  lif_kv_append -> lif_kv_attend  ->  lif_packed_multiply  -> ...
 *
 *   - E is fp32, fp16 or bfloat16.  Rows lie at a stride in elements; rows of E begin at multiples of 16 bytes, rows of 8 bits at multiples of 8.
 *   - Neither call needs a workspace, blocks or synchronises, and all can be captured into a HIP graph.  lif_add_norm has no handle; calls of
 *     lif_packed_multiply and lif_packed_dequantize on one handle may overlap on several streams, lif_packed_quantize and lif_packed_pack with none.
 *   - Rows in 8 bits are whole numbers -127..127 with an fp32 scale for the row, or for each `group` of its elements (the last group may be
 *     shorter): element = code * scale.
 */

/* Rows of a lif_add_norm. */
typedef struct lif_norm_rows {
    const void* x;          /* [n_rows x width] E                                                */
    const void* residual;   /* [n_rows x width] E, added to x; NULL: none                        */
    void* total;            /* [n_rows x width] E, written: residual + x; NULL: not wanted.  May be the rows of x or of the residual */
    void* out;              /* [n_rows x width], written: E, or 8 bits if scales are given.  May be the rows of x or of the residual (E) */
    float* scales;          /* [n_rows] or [n_rows x ceil(width / group)] fp32, written; NULL: out is E */
    const float* weight;    /* [width] fp32; NULL: ones.  Unused without a norm                  */
    const float* bias;      /* [width] fp32; NULL: zeros.  LIF_NORM_LAYER only                   */
    int64_t x_stride, residual_stride, total_stride, out_stride;  /* elements between rows       */
    int32_t n_rows;         /* 1..2^19                                                           */
    int32_t width;          /* a multiple of 8, 8..65536                                         */
    int32_t dtype;          /* enum lif_dtype: E                                                 */
    int32_t norm;           /* enum lif_norm (LIF_NORM_NONE: the addition, the rounding to 8 bits) */
    int32_t group;          /* elements of a scale: 32, 64 or 128; 0: the row has one            */
    float eps;
} lif_norm_rows;

/*
 * h = residual + x, total = h rounded to E, and of h (not of the rounded total)
 *   NONE  h      RMS  h / sqrt(mean h^2 + eps) * weight      LAYER  (h - mean) / sqrt(var + eps) * weight + bias
 * rounded to E, or to 8 bits: scale = max |y| * (1 / 127), in fp32, rounded to 16 significant bits, code = y / scale rounded to the nearest whole number, of
 * two the even one (a step of 16 bits makes that exact).  Sums are fp64, rounded once; the rest is fp32 in the order written here, every operation
 * rounded: results do not depend on the number of rows, and are reproducible bit for bit.  Where the scale is below 2^-110 scale and codes are 0; where it
 * would be infinite or not a number the scale is not a number.  total, out and scales must not overlap each other, nor weight and bias, nor x and the residual in
 * another way than as the same rows (LIF_INVALID_ARG; of rows at different strides whose ranges meet, any).
 */
int lif_add_norm(const lif_norm_rows* rows, void* stream);

typedef struct lif_packed lif_packed;

typedef struct lif_packed_config {
    int32_t n_out;          /* rows of the matrix: 1..2^20                                       */
    int32_t n_in;           /* a multiple of 8, 8..65536                                         */
    int32_t group;          /* inputs that share a scale (and a zero point): 32, 64 or 128       */
    int32_t zeros;          /* 0: every zero point is 8; 1: each group has one                   */
    int32_t dtype;          /* enum lif_dtype: of full weights, rows and outputs                 */
} lif_packed_config;

typedef struct lif_packed_buffers {
    void* codes;            /* device, lif_packed_code_bytes(cfg) bytes, 16-byte aligned         */
    void* groups;           /* device, lif_packed_group_bytes(cfg) bytes, 16-byte aligned        */
    size_t code_bytes, group_bytes;
} lif_packed_buffers;

/* Rows of a lif_packed_multiply. */
typedef struct lif_packed_rows {
    const void* x;          /* [n_rows x n_in]: E, or 8 bits if x_scales are given               */
    const float* x_scales;  /* [n_rows] or [n_rows x ceil(n_in / x_group)] fp32; NULL: x is E    */
    const float* bias;      /* [n_out] fp32, or NULL                                             */
    void* out;              /* [n_rows x n_out] E, written; must not overlap x, x_scales, bias or the matrix */
    int64_t x_stride, out_stride;  /* elements between rows; that of out need not be a multiple of anything */
    int32_t n_rows;         /* 1..2^19                                                           */
    int32_t x_group;        /* 0: a scale for each row; else the group of the weights            */
} lif_packed_rows;

/* Bytes of the two arrays (0 if cfg is invalid): n_out rounded up to 16 times n_in rounded up to 128, half a byte each; 4 bytes for each group. */
size_t lif_packed_code_bytes(const lif_packed_config* cfg);
size_t lif_packed_group_bytes(const lif_packed_config* cfg);

/* As lif_create: validates (the two arrays must not overlap), enqueues nothing; call lif_packed_quantize or lif_packed_pack first (or fill the arrays
 * with those of an equal handle). */
int lif_packed_create(const lif_packed_config* cfg, const lif_packed_buffers* buf, lif_packed** out);
int lif_packed_destroy(lif_packed* packed);

/*
 * From full weights (device, [n_out x n_in] E, rows at `stride` elements, 16-byte aligned).  Of the weights w of a group
 *   zeros 0   scale = max |w| * (1 / 7), zero = 8      zeros 1   scale = (max(w, 0) - min(w, 0)) * (1 / 15), zero = -min(w, 0) / scale, nearest
 * scale in fp32, rounded to 16 significant bits;  code = w / scale + zero to the nearest whole number, of two the even w / scale, in 0..15.  A scale below 2^-110
 * counts as 0; groups with a weight that is not finite, or whose scale would not be, give weights that are not numbers.
 */
int lif_packed_quantize(lif_packed* packed, const void* weights, int64_t stride, void* stream);

/*
 * (Neither these arrays nor the full weights of the two other calls may overlap the arrays of the matrix.)
 * From codes (device, [n_out x n_in / 2], two in a byte, the lower input in the lower half), scales [n_out x ceil(n_in / group)] fp32, which are
 * rounded to 16 significant bits (fp16 and bf16 values are kept; those below the normal numbers to multiples of 2^-141; what is infinite, or would be, is
 * not a number), and zeros [n_out x ceil(n_in / group)], 0..255, NULL if the configuration has none.
 */
int lif_packed_pack(lif_packed* packed, const uint8_t* codes, const float* scales, const uint8_t* zeros, void* stream);

/* What the weights stand for, scale * (code - zero) rounded to E, [n_out x n_in] at `stride` elements, 16-byte aligned. */
int lif_packed_dequantize(lif_packed* packed, void* weights, int64_t stride, void* stream);

/*
 * out[t, n] = sum_k x[t, k] * scale[n, k / group] * (code[n, k] - zero[n, k / group]) + bias[n]
 * Weights are not rounded further: a group's sum is fp32 (whole numbers for rows in 8 bits), scaled, added up in fp32 and rounded once to E.  Sums have a
 * fixed order for a given number of rows.  x_stride is at most 2^22.  In bf16, fp32 and 8 bits by groups what lies below 2^-133 in x, in its products with
 * whole numbers and in an output may be lost.  A row that holds infinity or NaN, or meets a scale that does, gives infinity or NaN there; other rows do not
 * see it.
 */
int lif_packed_multiply(lif_packed* packed, const lif_packed_rows* rows, void* stream);

/* Message of the last LIF_HIP_ERROR / LIF_INVALID_ARG on the calling thread. */
const char* lif_last_error_string(void);

/* Library version, for the loader check. */
int lif_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LIF_H */
