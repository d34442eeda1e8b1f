/*
 * ead.h - C ABI of the B200 (sm_100a) library for the gate step of Entropy
 * Adaptive Decoding (EAD).
 *
 * One "gate step" is one pass through the loop body of the paper's
 * Algorithm 1 for a batch of B independent sequences: project the active
 * model's final hidden state through that model's LM head (the last stage of
 * "l <- M_t(x + y)"), take the softmax of the raw logits (Eq. 1) and its
 * Shannon entropy (Eq. 2), pick the greedy token (the temperature -> 0 limit
 * of the sampling lines), append the entropy to the sequence's window and
 * average the last w entries (Eq. 3 / "mean(W[-w:])"), count the token
 * (c <- c + 1) and apply the dwell + threshold rule (Eq. 4) that selects the
 * model for the next token.
 *
 * Conventions
 *   - Every function returns 0 (EAD_OK) or a negative EAD_E* code; nothing
 *     throws or aborts across this boundary.  ead_strerror names a code.
 *   - Pointers marked "dev" are device pointers on cfg.device, "host" are
 *     host pointers.  Weights, hidden states and outputs are BORROWED: the
 *     library never copies or frees them; they must stay valid until the work
 *     enqueued with them has finished.  All per-sequence state (window,
 *     dwell counter, model flag) is OWNED by the context.
 *   - bf16 matrices are row major; their base must be 16-byte aligned and
 *     H_small, H_large must be multiples of 8 (16-byte rows).
 *   - Work is enqueued on cfg.stream and is asynchronous with respect to the
 *     host unless stated otherwise.  Calls on one context must not overlap on
 *     the device (one stream); the context is not thread safe.
 *   - The library needs an sm_100 device and has no other code path:
 *     ead_create fails with EAD_EUNSUPPORTED_ARCH elsewhere.
 *   - Models are numbered 0 = small (M_S), 1 = large (M_L).
 */
#ifndef EAD_H_
#define EAD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EAD_OK                  0
#define EAD_EINVALID_ARG      (-1)  /* NULL where not allowed, size out of range            */
#define EAD_EALIGNMENT        (-2)  /* pointer not 16-byte aligned or H not a multiple of 8 */
#define EAD_ECUDA             (-3)  /* a CUDA runtime / driver call failed                  */
#define EAD_EUNSUPPORTED_ARCH (-4)  /* device is not sm_100                                 */
#define EAD_EDEVICE_FAULT     (-5)  /* the device status word reports a kernel-side error   */
#define EAD_ESTATE            (-6)  /* state blob of the wrong size or version              */
#define EAD_ELIMIT            (-7)  /* size beyond a fixed built-in limit (see EAD_STATIC_*)  */

/* Bits of the device status word (ead_status). */
#define EAD_STATUS_NONFINITE   0x1u /* some row saw a NaN / infinite logit (row gets H = NaN) */
#define EAD_STATUS_WAIT_EXPIRED 0x2u /* a bounded wait inside a kernel ran out                 */
#define EAD_STATUS_BAD_COUNT   0x4u /* row counts inconsistent (internal ones, or a step's new_start) */
#define EAD_STATUS_SHARD_MISMATCH 0x8u /* vocabulary shards disagree on the step or on a row's model */
#define EAD_STATUS_BAD_PAGE    0x10u /* paged cache: page index out of range, or position not below max_len */

typedef struct ead_ctx ead_ctx; /* opaque */

/* Hyper-parameters follow the "Require" line of Algorithm 1 (tau, w, d_min);
 * the paper's experiments use w = 5 and d_min = 10. */
typedef struct ead_config {
    int32_t B;           /* sequences in the batch, 1 .. 4096                                 */
    int32_t V;           /* vocabulary size shared by both heads, >= 1                        */
    int32_t H_small;     /* hidden size of M_S, multiple of 8, >= 8                           */
    int32_t H_large;     /* hidden size of M_L, multiple of 8, >= 8                           */
    int32_t w;           /* window length of Eq. 3, 1 .. 64                                   */
    int32_t d_min;       /* minimum tokens on a model before a switch (Eq. 4); <= 1 = none    */
    float   tau;         /* threshold of Eq. 4, compared with the rolling mean in `unit`      */
    int32_t unit;        /* 0: entropy in nats; 1: in bits (Eq. 2 as printed, log base 2)     */
    int32_t start_model; /* model of the first token; Algorithm 1 starts on 0 (small)         */
    int32_t device;      /* CUDA device ordinal                                               */
    void   *stream;      /* cudaStream_t to enqueue on (borrowed); NULL = legacy default      */
    float   temperature; /* T of Algorithm 1's sampling lines; 0 = greedy (arg max)           */
    uint64_t seed;       /* seed of the sampling random stream (used when temperature > 0)    */
    int32_t eos_token;   /* token that ends a sequence ("while not done"); < 0 = none         */
    int32_t V_large;     /* vocabulary of M_L if it differs from V (the paper allows models of
                            different architectures); 0 = same as V.  Tokens of a step are
                            indices into the vocabulary of the model that produced them      */
    int32_t shard_count; /* 0: this context holds the whole heads.  n >= 1: it holds one of n
                            vocabulary slices (see ead_shard_connect); V and V_large are then the
                            rows of its slices                                                   */
    int32_t vocab_offset_small; /* sharded: row of the full small head at which this slice starts,
                                   a multiple of 16; tokens are reported in full-head indices   */
    int32_t vocab_offset_large; /* the same for the large head                                  */
} ead_config;

/*
 * Creates a context: allocates the per-sequence state of Algorithm 1's
 * initialisation (empty window, c = 0, M_t = start_model) plus scratch, and
 * encodes the TMA descriptors of the two heads.
 *   W_small  dev, bf16 [V, H_small], one row per vocabulary entry (borrowed, read only)
 *   W_large  dev, bf16 [V_large or V, H_large]
 *   out      host, receives the context
 * Synchronises the device once.  Errors: EAD_EINVALID_ARG, EAD_EALIGNMENT,
 * EAD_EUNSUPPORTED_ARCH, EAD_ECUDA.
 */
int ead_create(const ead_config *cfg, const void *W_small, const void *W_large, ead_ctx **out);

/*
 * One gate step (one iteration of Algorithm 1's loop) for all B sequences.
 *   h_small     dev, bf16 [B, H_small]: final hidden state of M_S per sequence
 *   h_large     dev, bf16 [B, H_large]: the same for M_L
 *               Only the row of the model that is active for a sequence is read.
 *   tok         dev, int32 [B]: next token: with cfg.temperature = 0 the arg max (lowest index
 *               among equal maxima); with cfg.temperature = T > 0 a draw from softmax(l / T),
 *               realised as arg max of l_i / T + g_i with standard Gumbel g_i = -ln(-ln u_i),
 *               u_i = (2k + 1) / 2^24, k = top 23 bits of word (i mod 4) of
 *               Philox4x32-10(counter = {i / 4, step, row, 0}, key = seed), step = number of
 *               gate steps of the context since the last reset.  -1 for a row with
 *               non-finite logits
 *   H           dev, float [B]: entropy of Eq. 2 in cfg.unit
 *   Hbar        dev, float [B]: rolling mean of Eq. 3 after this token
 *   model_used  dev, uint8 [B]: model that produced this token
 *   next_model  dev, uint8 [B]: model selected for the next token (Eq. 4)
 * Any output pointer may be NULL to skip it.  Row b of every output belongs to
 * row b of the inputs.  Asynchronous.  Errors: EAD_EINVALID_ARG,
 * EAD_EALIGNMENT, EAD_ECUDA.
 */
int ead_step(ead_ctx *ctx, const void *h_small, const void *h_large, int32_t *tok, float *H,
             float *Hbar, uint8_t *model_used, uint8_t *next_model);

/*
 * T consecutive gate steps with the hidden states of all steps resident on
 * the device; step t reads h_*_seq[t] and writes row t of each output.  The
 * T-step loop is replayed from CUDA graphs; the result is bit-identical to T
 * calls of ead_step.  Continues from the context's current state.
 *   h_small_seq  dev, bf16 [T, B, H_small];  h_large_seq  dev, bf16 [T, B, H_large]
 *   outputs      dev, [T, B] each, as in ead_step; any may be NULL
 * Asynchronous.  Errors as ead_step.
 */
int ead_run(ead_ctx *ctx, int32_t T, const void *h_small_seq, const void *h_large_seq,
            int32_t *tok, float *H, float *Hbar, uint8_t *model_used, uint8_t *next_model);

/*
 * The same T steps as ead_run, but every buffer is a HOST pointer: hidden
 * states are copied to the device and results back through internal staging
 * buffers, in chunks that overlap with the computation.  Synchronous: returns
 * when the outputs are complete, and also when it fails: before an error is
 * returned every copy already enqueued to or from the caller's buffers has ended.
 * Any output may be NULL.  Pinned host memory makes the copies faster but is not required.
 */
int ead_run_host(ead_ctx *ctx, int32_t T, const void *h_small_seq, const void *h_large_seq,
                 int32_t *tok, float *H, float *Hbar, uint8_t *model_used, uint8_t *next_model);

/*
 * DIAGNOSTIC (measurement aid, not part of the gate step's interface; so are
 * ead_kernel_launches, ead_launch_info, ead_plan_split, ead_plan_units, ead_plan_chunk and
 * ead_kv_wait_limit below).
 * The same T steps as ead_run, launched kernel by kernel (no graph replay) with
 * CUDA events around every kernel on cfg.stream, to attribute device time.
 *   kernel_ms  host, float [3]: summed device time in milliseconds of the
 *              compaction, LM-head and merge+gate kernels over the T steps
 * Synchronous (waits for the stream).  Results are identical to ead_run; the
 * event records make it slower, so it is a measurement aid, not the fast path.
 */
int ead_run_timed(ead_ctx *ctx, int32_t T, const void *h_small_seq, const void *h_large_seq,
                  int32_t *tok, float *H, float *Hbar, uint8_t *model_used, uint8_t *next_model,
                  float *kernel_ms);

/* Back to Algorithm 1's initial state (empty window, c = 0, start model) and a
 * cleared status word.  Asynchronous. */
int ead_reset(ead_ctx *ctx);

/* Waits for the context's stream, then reports the device status word
 * (EAD_STATUS_* bits, sticky until ead_reset).  Returns EAD_EDEVICE_FAULT if
 * EAD_STATUS_WAIT_EXPIRED or EAD_STATUS_BAD_COUNT is set, EAD_ESTATE if
 * EAD_STATUS_SHARD_MISMATCH is set, else EAD_OK. */
int ead_status(ead_ctx *ctx, uint32_t *status_word);

/*
 * Checkpoint of the per-sequence state (window contents, dwell counters, model
 * flags, number of steps taken).  ead_state_size gives the blob size for this
 * context; ead_get_state copies device -> host, ead_set_state host -> device.
 * Both wait for the stream.  A blob is only valid for a context with the same
 * B and w; ead_set_state also rejects (EAD_ESTATE, nothing copied) a blob whose flags are
 * not 0 / 1 or whose dwell counters or window fill counts are negative.
 * Errors: EAD_EINVALID_ARG, EAD_ESTATE, EAD_ECUDA.
 */
size_t ead_state_size(const ead_ctx *ctx);
int ead_get_state(ead_ctx *ctx, void *host_blob, size_t size);
int ead_set_state(ead_ctx *ctx, const void *host_blob, size_t size);

/*
 * Done mask ("while not done" of Algorithm 1).  A sequence becomes done when it produces
 * cfg.eos_token, or when the caller marks it here.  From the next step on a done row takes no
 * part: no logits are computed for it, its outputs are token -1, NaN entropies and its
 * unchanged model in model_used / next_model, and its window, counters and model stay frozen.
 * ead_reset clears the mask.  Both calls wait for the stream.
 *   done  host, uint8 [B], each 0 or 1
 * Errors: EAD_EINVALID_ARG, EAD_ECUDA.
 */
int ead_set_done(ead_ctx *ctx, const uint8_t *done);
int ead_get_done(ead_ctx *ctx, uint8_t *done);

/*
 * Usage accounting since the last ead_reset (the paper's "large model usage" column and the
 * count of model switches), summed over the B sequences.  Rows with non-finite logits in a
 * step are not counted for that step.  Waits for the stream.
 *   counts  host, uint64 [3]: {tokens produced by M_S, tokens produced by M_L, switches}
 *   per_row host, uint32 [3 * B] or NULL: the same three counters per sequence, row major [3][B]
 * Errors: EAD_EINVALID_ARG, EAD_ECUDA.
 */
int ead_usage(ead_ctx *ctx, uint64_t *counts, uint32_t *per_row);

/*
 * The footnote of the paper's Table 1: average parameters per forward pass relative to the
 * large model, (alpha P_S + beta P_L) / P_L, with alpha = tokens_small / total and
 * beta = tokens_large / total.  Pure host arithmetic; returns NaN if both counts are 0.
 */
double ead_parameter_ratio(uint64_t tokens_small, uint64_t tokens_large, double P_small, double P_large);

/* DIAGNOSTIC.  Number of kernels the library has launched through this context so far
 * (graph replays count their kernel nodes). */
int64_t ead_kernel_launches(const ead_ctx *ctx);

/* DIAGNOSTIC.  Launch geometry chosen at creation, for reporting: fills up to n ints with
 * {CTAs of the LM-head kernel, pipeline stages, rows of the hidden-state TMA
 * box, dynamic shared memory bytes}.  For B > 128 the stage count is that of a single-block unit
 * (48 KiB stages); the kernel cuts the same ring into 64 or 72 KiB stages for units of two blocks
 * and into 40 KiB ones for a head of at most 64 rows. */
int ead_launch_info(const ead_ctx *ctx, int32_t *info, int32_t n);

/*
 * Vocabulary-sharded gate step (several GPUs, one sequence batch).  The softmax of Eq. 1 and
 * the entropy of Eq. 2 are sums over the vocabulary and the greedy / sampled token is a maximum
 * over it, so the vocabulary rows of both heads can be split over n GPUs: each computes the
 * statistics of its slice, the slices' statistics are exchanged (n x B records of 32 bytes:
 * the only traffic between the GPUs), and every GPU merges all of them in shard order and runs
 * the window / dwell / threshold part of Algorithm 1 itself.  All GPUs then hold identical
 * per-sequence state and identical outputs, bit for bit, without further communication.  The
 * paper describes one device; this split is the build's own.
 *
 * Each GPU creates a context with cfg.shard_count = n (<= 16), cfg.V / cfg.V_large = rows of its
 * slices, cfg.vocab_offset_* = where they start, and the slice pointers as W_small / W_large;
 * all other fields equal on all GPUs.  Every GPU gets the full hidden rows at every step.
 *
 * ead_shard_range: the slice [*begin, *end) of a head of V rows that shard `shard` of n_shards
 * takes when the rows are dealt out in whole tiles of 128 (host arithmetic, needs no GPU).
 * Errors: EAD_EINVALID_ARG (also when n_shards exceeds the number of tiles).
 *
 * The exchange can run in two ways.
 *
 * (1) Inside the kernels, over peer memory.  Every shard owns an exchange buffer of
 * ead_shard_exchange_bytes(B, n) bytes, zero-filled, 16-byte aligned, mapped into the address
 * space of every other shard's GPU (peer access, an IPC handle, symmetric memory).
 *     ead_shard_connect(ctx, shard, exchange)   exchange: host array [n]; entry d = shard d's
 *                                               buffer as addressable from this GPU (entry
 *                                               `shard` is this context's own, local buffer)
 * From then on ead_step / ead_run / ead_run_host work as on one GPU, called on every shard with
 * the same hidden states: after its cross-CTA merge each shard stores its B records straight
 * into all n exchange buffers (plain stores; the record's step word last, with release
 * semantics at system scope), and the thread that stored a row's record then waits until that
 * row's records of all n shards for this step have arrived in the local buffer and finishes
 * the row: a sharded step is the same three kernels as an unsharded one.  Buffers alternate with
 * the parity of the step, which suffices because a shard cannot run more than one step ahead
 * of another.  The wait is bounded (2 s): a shard that never delivers sets
 * EAD_STATUS_WAIT_EXPIRED, the rows are reported like non-finite rows, and later steps do not
 * wait again.  Waits for the stream; restarts the numbering of exchanged records, so all shards
 * connect (to zero-filled buffers) at the same point of their runs.  ead_reset, ead_set_state
 * and ead_set_done must be applied on all shards alike.
 * Errors: EAD_EINVALID_ARG, EAD_EALIGNMENT, EAD_ECUDA.  Before ead_shard_connect the stepping
 * calls return EAD_EINVALID_ARG on a sharded context; ead_run_timed always does.
 *
 * (2) By the caller, between two library calls (NCCL or any other all-gather that is ordered
 * on the context's stream); no peer mapping needed:
 *     ead_shard_partials(ctx, h_small, h_large, records);      // this GPU's [B] records
 *     <all-gather the n record arrays, in shard order, into all_records on every GPU>
 *     ead_shard_gate(ctx, all_records, n, tok, H, Hbar, model_used, next_model);
 *   records      dev, [B] x EAD_SHARD_RECORD_BYTES, 16-byte aligned: per sequence (caller's row
 *                order) {float m, s, t; int32 idx; float k; int32 ki; int32 model; int32 step1}:
 *                max, sum exp(z - m), sum exp(z - m)(z - m) log2 e and arg max of the slice's
 *                logits, the sampling candidate, the head they belong to, and 1 + the number
 *                of sharded steps this context has taken.  Rows of ended sequences are not
 *                written.
 *   all_records  dev, [n_shards][B] records, shard s at index s
 *   outputs      as in ead_step
 * Both calls are asynchronous on the context's stream.  On a connected context `records` and
 * `all_records` may be NULL: the two halves of a step of way (1), called apart.
 *
 * In both ways a record whose model or step number differs from this context's sets
 * EAD_STATUS_SHARD_MISMATCH and leaves the row's state untouched (outputs as for a non-finite
 * row).  Errors of (2): EAD_EINVALID_ARG (also: context not created with shard_count >= 1, or
 * n_shards not equal to it), EAD_EALIGNMENT, EAD_ECUDA.
 */
#define EAD_SHARD_RECORD_BYTES 32
#define EAD_SHARD_MAX 16
int ead_shard_range(int32_t V, int32_t n_shards, int32_t shard, int32_t *begin, int32_t *end);
size_t ead_shard_exchange_bytes(int32_t B, int32_t n_shards);
int ead_shard_connect(ead_ctx *ctx, int32_t shard, void *const *exchange);
int ead_shard_partials(ead_ctx *ctx, const void *h_small, const void *h_large, void *records);
int ead_shard_gate(ead_ctx *ctx, const void *all_records, int32_t n_shards, int32_t *tok, float *H,
                   float *Hbar, uint8_t *model_used, uint8_t *next_model);

/*
 * DIAGNOSTIC.  How the one-block LM-head kernel (the one behind ead_head_entropy_static) divides
 * one head among its CTAs (host-side replica of the rule
 * the kernel applies on the device; pure arithmetic, needs no GPU).  With n rows on a head
 * there are R = ceil(n / 128) row blocks; CTA `cta` of `G` serves row block out[1] and
 * vocabulary columns [out[3], out[4]) (multiples of 16; the end may exceed V by < 16).
 *   out  host, int32 [6]: {active, row_block, slot, col_begin, col_end, group_size}
 * Errors: EAD_EINVALID_ARG.
 */
int ead_plan_split(int32_t cta, int32_t G, int32_t n_rows, int32_t V, int32_t *out);

/*
 * DIAGNOSTIC.  The same for the kernel that serves B > 128, whose CTAs work in UNITS of row blocks
 * (host-side replica of the device rule; needs no GPU).  With two_blocks != 0 (heads with a hidden
 * size of 3072 and more) a unit is two consecutive 128-row blocks against one weight tile.  An odd
 * last block is a unit of its own.  A head of exactly three row blocks is different: if its last
 * block has at most 64 rows, the two-block unit takes it along as a thin third block (thin16 =
 * its rows rounded up to 16) and works on tiles of tile_n = 256 - thin16 columns; otherwise it is
 * served one block per unit, as is every head with two_blocks == 0.  Units get CTAs in
 * proportion to their cost (two blocks : one = 9 : 5); member `slot` of a unit's `group` CTAs takes
 * tile slot of every whole round k < rounds, then its piece [tail_col0, tail_col0 + tail_cols) of
 * what the whole rounds leave over (cut evenly in 16-column units; tail_cols may be 0).  The
 * tiles of the first n_hi rounds are w_hi columns wide, those of the other rounds w_lo (round k
 * begins where round k - 1 ends: at group * (min(k, n_hi) * w_hi + max(0, k - n_hi) * w_lo)).  With
 * more than eight whole rounds of full tiles, no rest, or single-block units on a head of at most
 * two row blocks, all are tile_n wide; otherwise a member's share is cut into pieces of nearly
 * equal width.
 *   out  host, int32 [13]: {active, two_blocks, first_row_block, slot, group, rounds, tail_col0,
 *                           tail_cols, thin16, tile_n, n_hi, w_hi, w_lo}
 * Errors: EAD_EINVALID_ARG (also: more row blocks than CTAs).
 */
int ead_plan_units(int32_t cta, int32_t G, int32_t n_rows, int32_t V, int32_t two_blocks, int32_t *out);

/* Waits for outstanding work and frees everything the context owns.  NULL is allowed. */
void ead_destroy(ead_ctx *ctx);

/*
 * Entropy and greedy token of one LM head for a dense batch, WITHOUT any allocation.
 * (The paper has no counterpart: this is a service entry point of the library; what it
 * computes per row is Eq. 1-2 and the arg max, exactly as one ead_step does for rows
 * that are on that head.)
 *
 * For callers that are not allowed to allocate device memory: code that runs while the
 * framework's allocator is frozen (inside a memory-planned inference engine, under a
 * fixed memory budget that has already been handed out, or in a latency-critical section
 * where cudaMalloc's implicit device synchronisation is unacceptable).  ead_create and
 * ead_run_host call cudaMalloc; this function calls neither cudaMalloc nor cudaFree nor
 * any allocating library routine.  Its scratch memory (per-CTA partial statistics, a
 * padded copy of the hidden rows, a control block) lives in one array compiled into the
 * library, about 2.4 MB, which every GPU that loads the library holds until the process
 * exits.  That fixes the limits:
 *     B <= EAD_STATIC_MAX_B (128),  H <= EAD_STATIC_MAX_H (8192),  H a multiple of 8.
 * Larger sizes are rejected with EAD_ELIMIT before anything is launched.
 *
 *   W        dev, bf16 [V, H] row major, 16-byte aligned (borrowed, read only)
 *   h        dev, bf16 [B, H] row major, 16-byte aligned: one hidden row per sequence
 *   tok      dev, int32 [B]: greedy token, lowest index among equal maxima (-1 for a row
 *            with non-finite logits); may be NULL
 *   H_out    dev, float [B]: entropy in nats (NaN for a row with non-finite logits); may be NULL
 *   status   dev, uint32 [1]: receives EAD_STATUS_* bits of this call; may be NULL
 *   device   CUDA device ordinal; made current by the call
 *   stream   cudaStream_t to enqueue on; NULL = legacy default stream
 *
 * Asynchronous: four kernels are enqueued on `stream` (status clear, staging of the hidden
 * rows, the LM-head contraction, the merge).  The first call on a device also
 * looks up the device address of the built-in array and the device's limits; make that
 * first call outside any stream capture.
 * Every call on a device uses the SAME array.  The call rewrites all of it that it later
 * reads (nothing of an earlier call leaks into the result), but two calls whose kernels
 * overlap on the GPU (different streams, no dependency) race on it: keep calls on one
 * device ordered.  Not thread safe with respect to other calls on the same device.
 * Errors: EAD_EINVALID_ARG, EAD_EALIGNMENT, EAD_ELIMIT, EAD_EUNSUPPORTED_ARCH, EAD_ECUDA.
 */
#define EAD_STATIC_MAX_B 128
#define EAD_STATIC_MAX_H 8192
int ead_head_entropy_static(const void *W, const void *h, int32_t B, int32_t V, int32_t H,
                            int32_t *tok, float *H_out, uint32_t *status, int32_t device,
                            void *stream);

/*
 * Decoder-side operators around the gate step: what M_S and M_L do between two gate steps with
 * their contexts.  (The paper defines none of them: "l <- M_t(x + y)" is one line of Algorithm 1.
 * A sequence that stays on its model brings one new token per step; one that was just switched
 * brings every token its new model has not seen, which is why attention takes a CHUNK of new
 * tokens per sequence, of a different length for every sequence of the batch.)
 *
 * Number formats.  EAD_FMT_BF16: bf16 values.  EAD_FMT_E4M3: 8-bit e4m3 codes, and for every 32
 * consecutive values (along the head dimension, or along a hidden row) one scale byte e that
 * stands for 2^(e - 127): value = code * 2^(e - 127).  The scale is the smallest power of two for
 * which no finite value of the block exceeds 448, limited to 2^-120 .. 2^119 (a block of zeros
 * has 2^-120; beyond 448 * 2^119 values saturate); codes are rounded to nearest, ties to even.  A block
 * with a NaN or an infinity in it gets scale byte 255 and codes 0x7F, and reads as NaNs.  All
 * other values are exact in bf16.  Code 0x7F does not occur under another scale byte; what is
 * read for it there is unspecified.
 *
 * All four calls only enqueue work on `stream` of `device` (which they make current), allocate
 * nothing and copy nothing to the host.  They own no state: every buffer is the caller's.
 * Row strides are in elements; rows, pools and strides must keep 16-byte alignment.
 */
#define EAD_FMT_BF16 0
#define EAD_FMT_E4M3 1
#define EAD_FMT_BLOCK 32               /* values per scale byte */

/*
 * One layer's paged key/value cache.  Token slot s of page p of head h is the head_dim values at
 * element p * page_stride + h * head_stride + s * slot_stride of k and of v (so pages may be laid
 * out head by head or token by token, and k and v may be halves of one allocation).
 */
typedef struct ead_kv_cache {
    int32_t format;          /* EAD_FMT_BF16 or EAD_FMT_E4M3                                    */
    int32_t heads_kv;        /* 1 .. 128                                                        */
    int32_t head_dim;        /* 64 or 128                                                       */
    int32_t page_size;       /* token slots per page: 8, 16, 32, 64, 128 or 256                 */
    int32_t n_pages;         /* pages in the pools                                              */
    int32_t reserved;        /* 0                                                               */
    int64_t page_stride, head_stride, slot_stride;   /* elements                                */
    void *k, *v;             /* dev pools                                                       */
    uint8_t *k_scale, *v_scale;   /* dev, EAD_FMT_E4M3 only: [n_pages, heads_kv, page_size,
                                     head_dim / 32] bytes, contiguous; NULL for EAD_FMT_BF16    */
} ead_kv_cache;

/*
 * The step's batch.  Sequence b brings the tokens new_start[b] .. new_start[b + 1] - 1 of the
 * step (possibly none); they are the LAST tokens of its context of kv_len[b] tokens, i.e. token
 * i of them has position kv_len[b] - n_b + i.  Position p lives in page
 * page_table[b * table_stride + p / page_size], slot p % page_size.
 * max_new and max_len are upper bounds of n_b and kv_len[b] known to the host; the arrays
 * themselves stay on the device (a captured graph replays with new contents).  Positions at or
 * beyond max_len have no place: no page table entry is read for them.
 */
typedef struct ead_kv_batch {
    int32_t B;               /* sequences, 1 .. 4096                                            */
    int32_t n_tokens;        /* new tokens of the step = new_start[B]; 0 .. 2^30                */
    int32_t max_new;         /* >= every n_b                                                    */
    int32_t max_len;         /* >= every kv_len[b], at most 2^30                                */
    const int32_t *new_start;    /* dev [B + 1], ascending, new_start[0] = 0                    */
    const int32_t *kv_len;       /* dev [B]                                                     */
    const int32_t *page_table;   /* dev [B, table_stride]; entries beyond a context are not read */
    int32_t table_stride;    /* entries per row, >= ceil(max_len / page_size)                   */
    int32_t reserved;        /* 0                                                               */
} ead_kv_batch;

/*
 * Writes the new tokens' keys and values into the cache, quantised where its format says so.
 *   k_new, v_new  dev, bf16 [n_tokens, heads_kv, head_dim]; new_stride elements between tokens
 *                 (heads of a token are contiguous), so both may be slices of one projection
 *   status        dev uint32 or NULL; EAD_STATUS_BAD_PAGE is OR-ed in when a token has no valid
 *                 place (its page index is out of range, its position negative or not below
 *                 max_len), EAD_STATUS_BAD_COUNT when new_start contradicts n_tokens or max_new (a token
 *                 at or behind new_start[B], or of a sequence that brings more than max_new or ends behind
 *                 n_tokens); such a token is not written
 * Two tokens of a step must not share a slot.  Errors: EAD_EINVALID_ARG, EAD_EALIGNMENT,
 * EAD_EUNSUPPORTED_ARCH, EAD_ECUDA.
 */
int ead_kv_write(const ead_kv_cache *cache, const ead_kv_batch *batch, const void *k_new, const void *v_new,
                 int64_t new_stride, uint32_t *status, int32_t device, void *stream);

/*
 * Reads tokens back as bf16.  Row new_start[b] + i of the outputs is position first[b] + i of
 * sequence b (first NULL: 0), for i < n_b; batch->kv_len is not used and may be NULL.
 *   k_out, v_out  dev, bf16 [n_tokens, heads_kv, head_dim], out_stride elements between tokens
 *   first         dev int32 [B] or NULL
 * A token without a valid place reads as zeros and sets EAD_STATUS_BAD_PAGE or EAD_STATUS_BAD_COUNT as above.
 * Errors as ead_kv_write.
 */
int ead_kv_read(const ead_kv_cache *cache, const ead_kv_batch *batch, const int32_t *first, void *k_out, void *v_out,
                int64_t out_stride, uint32_t *status, int32_t device, void *stream);

/*
 * Attention of the step's new tokens over the paged cache (which already holds them:
 * ead_kv_write comes first).  Query head hq reads cache head hq / (heads_q / heads_kv).  A query
 * at position p sees key j iff j <= p and (window == 0 or j > p - window or j < sinks):
 *   z_j = scale * q . k_j,  out = sum_j exp(z_j) v_j / sum_j exp(z_j),  lse = ln sum_j exp(z_j)
 * with sums and maxima in 32 bits; probabilities are rounded to bf16 (the type of the values
 * they weight) before the product with v.  That product is divided by the sum at the end, and probabilities relative
 * to the running maximum reach 2^8: values above 2^120 / (number of keys seen) can overflow on the way.  Sequences
 * of at most 16 rows (new tokens x query heads per cache head) over an 8-bit cache take q as f16 after a power of two
 * has brought the row's largest element to 1 .. 2: elements below 2^-17 of it are rounded to multiples of
 * 2^-24.  A query that sees nothing (its position is negative)
 * gets zeros and lse = -infinity.  Keys that no query of a sequence sees are not
 * read, nor are the page table entries of pages that hold only such keys.  A key that is not finite
 * touches only the queries that see it; a VALUE that is not finite and is seen by one query can also
 * reach the sequence's other queries of this call, in its cache head and dimension (a probability of 0 times
 * NaN is NaN, as in a matrix product with a masked softmax): a caller that has to tell them apart
 * calls once per token.
 *   q          dev, bf16 [n_tokens, heads_q, head_dim], q_stride elements between tokens
 *   heads_q    a multiple of heads_kv, at most 128 per cache head
 *   scale      of the logits, finite and > 0
 *   window     >= 0; 0 = all earlier tokens;  sinks  >= 0; used with a window
 *   out        dev, bf16 [n_tokens, heads_q, head_dim], out_stride elements between tokens
 *   lse        dev float [n_tokens, heads_q] or NULL
 *   workspace  dev, EAD_KV_WORKSPACE_BYTES bytes, 256-byte aligned, zero-filled ONCE by the caller;
 *              every call leaves it ready for the next one.  Calls that may overlap on the
 *              device need a workspace each
 *   status     dev uint32 or NULL.  EAD_STATUS_BAD_PAGE: a page index was out of range (its
 *              tokens count as zeros) or a context is longer than max_len (the rest is not
 *              seen); EAD_STATUS_BAD_COUNT: new_start contradicts max_new or n_tokens (the rows
 *              of such a sequence are not written; rows of no sequence, behind new_start[B], are not written
 *              either and not reported); EAD_STATUS_WAIT_EXPIRED: a bounded wait in a kernel ran out (the
 *              outputs are not valid, and the workspace has to be zero-filled again)
 * The result does not depend on the order in which blocks run: partial results are joined in a
 * fixed order.  Errors: EAD_EINVALID_ARG, EAD_EALIGNMENT, EAD_ELIMIT (B * heads_kv * max_len above 2^34 per SM), EAD_EUNSUPPORTED_ARCH,
 * EAD_ECUDA.
 */
#define EAD_KV_WORKSPACE_BYTES (64u << 20)
int ead_kv_attention(const ead_kv_cache *cache, const ead_kv_batch *batch, const void *q, int64_t q_stride,
                     int32_t heads_q, float scale, int32_t window, int32_t sinks, void *out, int64_t out_stride,
                     float *lse, void *workspace, uint32_t *status, int32_t device, void *stream);

/*
 * DIAGNOSTIC.  The limit of the bounded waits in ead_kv_attention's kernels, in nanoseconds, for calls of this process from now
 * on; negative: the default (2 s).  With a limit that is too short waits run out in sound calls: for tests of what then happens.
 */
int ead_kv_wait_limit(int32_t ns);

/*
 * DIAGNOSTIC.  How ead_kv_attention weighs one sequence for one cache head when it deals a call's chunks out to the SMs (the
 * rule the kernel applies on the device; pure arithmetic, needs no GPU).  A unit is up to two row tiles of
 * floor(128 / heads_per_kv) tokens; it costs 12, and per tile of 64 keys that any of its queries sees (at least
 * one tile) 2, or 1 if it has one row tile.  Sequences of so few rows that the other kernel takes them have no units.
 *   n_new, kv_len  of the sequence;  max_new, window, sinks  as in the call;  heads_per_kv = heads_q / heads_kv
 *   out            host, int64 [2]: {units, their cost}
 * Errors: EAD_EINVALID_ARG.
 */
int ead_plan_chunk(int32_t n_new, int32_t kv_len, int32_t max_new, int32_t heads_per_kv, int32_t window, int32_t sinks,
                   int64_t *out);

/*
 * Residual addition and root-mean-square norm of n_rows hidden rows of H elements:
 *   s = x + residual (32 bits),  residual_out = bf16(s),
 *   y = s / sqrt(mean(s^2) + eps) * weight,  out = y in `format`
 * The sum of squares is taken over the unrounded s.  With EAD_FMT_BF16 the output is what
 * ead_step takes as h_small / h_large.
 *   x             dev, bf16 rows, x_stride elements apart
 *   residual      dev, bf16 rows, residual_stride apart, or NULL (s = x)
 *   residual_out  dev, bf16 rows, residual_out_stride apart, or NULL; may be residual or x itself
 *   weight        dev, bf16 [H]
 *   out           dev, bf16 or e4m3 rows, out_stride apart; may be x itself for EAD_FMT_BF16
 *   out_scale     dev, uint8 [n_rows, H / 32], EAD_FMT_E4M3 only, else NULL
 *   H             multiple of 8 (of 32 for EAD_FMT_E4M3), 8 .. 16384
 * Errors: EAD_EINVALID_ARG, EAD_EALIGNMENT, EAD_ELIMIT (H), EAD_EUNSUPPORTED_ARCH, EAD_ECUDA.
 */
#define EAD_NORM_MAX_H 16384
int ead_add_rmsnorm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                    void *residual_out, int64_t residual_out_stride, const void *weight, float eps, int32_t n_rows,
                    int32_t H, int32_t format, void *out, int64_t out_stride, uint8_t *out_scale, int32_t device,
                    void *stream);

/* Static, NUL-terminated description of an EAD_E* code. */
const char *ead_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* EAD_H_ */
