/*
 * fademem.h -- C ABI of the FadeMem per-chunk cache step on one MI355X
 * (gfx950).  FadeMem: "Distance-Aware Memory Consolidation for
 * Autoregressive Video Diffusion", arXiv 2606.10671.
 *
 * The library keeps, per transformer layer, the bounded ordered memory of
 * Sec. 3.1 / Sec. 3.3 (at most M entries, each one representative KV block
 * plus its span s and temporal position mu), updates it with Algorithm S1
 * (append, power-law distance schedule, adjacent-pair consolidation,
 * first-frame anchor), and runs the attention of a chunk's queries over
 * [memory entries in order || current chunk] (Sec. 3.1, Sec. 4.1).
 *
 * Conventions shared by every call
 * --------------------------------
 * - Tensors are token-major and contiguous: a block, a query chunk, a
 *   current chunk and an output are [tokens][heads][head_dim], one batch.
 *   Element type is fp32 or bf16 as configured (dtype); LSE is fp32.
 * - Device pointers must be 16-byte aligned; the pool 256-byte aligned.
 * - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *   Every call except fademem_get_state, fademem_entry_kv, fademem_set_state,
 *   fademem_merge_log, fademem_merge_counts and fademem_verify is
 *   asynchronous on that stream and never waits for the device
 *   (fademem_stage and fademem_count only read host state).  One cache is
 *   used by one host thread and one stream at a time.
 * - Calls that implement a step of the method cite the passage that defines
 *   it; the plumbing around them (pool sizing, creation, readers,
 *   checkpointing, error strings) has no counterpart in the paper and cites
 *   none.
 * - Ownership: the caller allocates and owns the device pool and every
 *   Q/K/V/O/LSE buffer.  The library allocates no device memory, never
 *   frees caller memory and keeps only the pool pointer.  insert copies K
 *   and V, so the caller may reuse its buffers once the stream has passed
 *   the call.
 * - Errors: 0 (FADEMEM_OK) or a negative FADEMEM_E* code.  Arguments and
 *   state are validated before anything is enqueued, so a call that fails
 *   validation leaves the cache unchanged.  FADEMEM_EHIP reports a HIP
 *   launch or runtime failure (see fademem_last_hip_error).  No C++
 *   exception crosses this interface.
 * - Debugging: with the environment variable FADEMEM_SERIALIZE set (not
 *   "0") when a cache is created, every asynchronous call on it waits for
 *   its own work before returning and reports a failure of that work as
 *   FADEMEM_EHIP, so an error shows at the call that caused it.  Results
 *   are the same bits as without it.
 */
#ifndef FADEMEM_H
#define FADEMEM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  FADEMEM_OK = 0,
  FADEMEM_EINVAL = -1,     /* bad configuration, argument, pointer or size      */
  FADEMEM_ESTATE = -2,     /* call not allowed in the current memory state       */
  FADEMEM_ENOMEM = -3,     /* caller's pool smaller than fademem_pool_bytes      */
  FADEMEM_EHIP = -4,       /* HIP runtime or launch error                        */
  FADEMEM_EUNSUPPORTED = -5,/* valid request this build does not implement       */
  FADEMEM_EINTERNAL = -6,  /* host replay of the memory state disagrees with the
                              device (fademem_verify, serialize mode)           */
  FADEMEM_ESCRATCH = -7    /* request larger than the static scratch of an
                              allocation-free entry point                       */
};

enum { FADEMEM_F32 = 0, FADEMEM_BF16 = 1 };

/* Consolidation operators: the K, V rule of a merge (Sec. 3.3
 * "Consolidation operator"; the ablation of Sec. 4.3, Table 4).  The
 * metadata rule (spans add, mu span-weighted) and the anchor's branch are
 * the same for all.
 *   SQRT_SPAN      X = (sqrt(s_j) X_j + sqrt(s_j+1) X_j+1) / (sqrt(s_j) + sqrt(s_j+1)),
 *                  the paper's default, in fp64, one RNE rounding to the storage type;
 *   AVERAGE        the same with both weights 1/2 (unweighted average);
 *   SELECT_NEAREST the newer entry's K, V (representative selection; no
 *                  K/V bytes move: the merged entry takes the newer one's slot);
 *   MAX            elementwise max pooling; the newer value wins only when
 *                  strictly greater (equal values, -0 and +0 included, keep
 *                  the older entry's bits). */
enum {
  FADEMEM_MERGE_SQRT_SPAN = 0,
  FADEMEM_MERGE_AVERAGE = 1,
  FADEMEM_MERGE_SELECT_NEAREST = 2,
  FADEMEM_MERGE_MAX = 3
};

typedef struct fademem_config {
  int64_t budget;           /* M, the entry budget (Sec. 3.1); 2 <= M <= 1023.
                               M >= 2 keeps one pair eligible once the newest
                               entry is protected (Sec. 3.3).                  */
  int32_t heads;            /* H >= 1                                          */
  int32_t head_dim;         /* D, 64 or 128                                    */
  int64_t tokens_per_block; /* N >= 1, tokens of one generation unit (one
                               latent frame, supplementary Sec. S4)            */
  double beta;              /* exponent of u(d) = d^beta, 0 < beta <= 1
                               (Sec. 3.3); the paper's default is 0.3 (Sec. 4.1) */
  int32_t anchor;           /* 1: the first inserted block is a global anchor
                               (Sec. 3.3, Alg. S1), the paper's default; 0: off */
  int32_t merge_op;         /* FADEMEM_MERGE_* (default SQRT_SPAN)              */
  int32_t dtype;            /* FADEMEM_F32 or FADEMEM_BF16 for K, V, Q, O      */
  int32_t layers;           /* L >= 1 per-layer memories sharing one schedule.
                               The schedule depends only on positions, so every
                               layer makes the same decisions (Sec. 3.3).       */
  int32_t rope_pairs;       /* Temporal RoPE handling (Sec. 3.3 "Boundary and
                               positional handling"): 0 = off (keys are used as
                               stored).  P > 0: the first P interleaved pairs
                               (2i, 2i+1) of each head's dimension carry the
                               temporal rotary phase; 1 <= P <= D/2.  Blocks
                               are inserted without their temporal phase and
                               stored so; fademem_attend exposes memory entry
                               i (0 = oldest) at temporal index i, i.e. pair k
                               of its keys rotated by the angle i * w_k with
                               w_k = rope_theta^(-k/P), evaluated in fp64 and
                               rounded once to the storage type.  The caller
                               applies the same rotation to the current
                               chunk's queries and keys at indices n + f (n =
                               entries held, f = frame within the chunk).    */
  double  rope_theta;       /* rotary base (> 1), e.g. 10000; ignored if P = 0 */
  int32_t stage_frames;     /* 0..4: frames a chunk may stage for the
                               zero-copy update (fademem_stage); 0 = off.
                               The pool then holds M + max(1, stage_frames)
                               KV slots per layer.                            */
} fademem_config;

typedef struct fademem_cache fademem_cache; /* opaque host object */

/* Bytes of device pool a configuration needs: M + max(1, stage_frames) KV
 * slots per layer for K and V, the memory's metadata, the attention's
 * scratch for split work (bf16: partial results of split query tiles,
 * 70.3 MB at D = 128; fp32: partial results of key ranges, 512 x 64 x (D+2)
 * floats) and, with rope_pairs > 0, a re-indexed K view per layer (one K
 * block per slot).  Returns EINVAL for a bad config. */
int fademem_pool_bytes(const fademem_config* cfg, size_t* bytes);

/* Create a cache over a caller-owned device pool of `pool_bytes` bytes
 * (>= fademem_pool_bytes).  Enqueues the initialisation of the metadata on
 * `stream` (the pool's previous contents do not matter).  The memory starts
 * empty.  *out receives a host handle to destroy with fademem_cache_destroy.
 * Errors: EINVAL (config, NULL or misaligned pool), ENOMEM (pool too small),
 * EHIP. */
int fademem_cache_create(const fademem_config* cfg, void* dev_pool, size_t pool_bytes,
                         void* stream, fademem_cache** out);

/* Release the host handle.  The pool stays the caller's.  NULL is a no-op. */
int fademem_cache_destroy(fademem_cache* cache);

/* Append the block B_t = (K_t, V_t) at position t as the entry (K_t, V_t,
 * t, 1) -- first step of Alg. S1, Sec. 3.3 "Memory entries and insertion".
 * k[l], v[l] (host arrays of `layers` device pointers) are layer l's block,
 * [N][H][D].  Positions are integers that strictly increase (0-indexed by
 * convention; the first block inserted into an empty memory becomes the
 * anchor when the option is on), |t| < 2^40.
 * Errors: EINVAL (NULL/misaligned pointers, position out of range),
 * ESTATE (position not increasing, or M+1 entries already held: call
 * fademem_consolidate first), EHIP. */
int fademem_insert(fademem_cache* cache, const void* const* k, const void* const* v,
                   int64_t position, void* stream);

/* Rest of Alg. S1.  If the memory holds at most M entries this is a no-op
 * (and enqueues nothing).  Otherwise, on the device: d_i = t - mu_i with t
 * the newest position, u = d^beta, gaps |u(d_{i+1}) - u(d_i)| over the
 * adjacent pairs except the one holding the newest entry, j = the smallest
 * gap (gaps within a relative 1e-9 of the smallest count as tied and the
 * oldest such pair wins); the pair is replaced by its consolidation: spans
 * add, mu is span-weighted; K, V by the configured operator (default:
 * sqrt-span weighted average evaluated in fp64 and rounded once,
 * round-to-nearest-even, to the storage type); when the pair holds the
 * anchor its K, V and position are kept (Sec. 3.3, Alg. S1).  The decision
 * never crosses to the host.  Errors: EHIP. */
int fademem_consolidate(fademem_cache* cache, void* stream);

/* A chunk's F updates in one call: for f = 0..frames-1, append frame f at
 * position first_position + f, then consolidate when over budget -- the
 * F sequential Alg. S1 updates that follow a chunk's final denoising step
 * (Sec. 4.1; supplementary Sec. S4: one entry per latent frame).  State,
 * merge log and every stored K/V bit equal those of `frames` calls of
 * fademem_insert + fademem_consolidate.  Frames are taken in groups of up
 * to four; within a group each K/V block that changes is written once (a
 * chain of merges is evaluated in registers, each merge
 * rounded to the storage type as on its own), and frames that a merge of
 * the same call consumes are read from the caller's buffers, never copied
 * into the pool.  k[l], v[l] (host arrays of `layers` device pointers) are
 * layer l's chunk, [frames*N][H][D], frame f in rows f*N..(f+1)*N-1; the
 * caller may reuse them once the stream has passed the call.
 * Errors: EINVAL (NULL/misaligned pointers, frames < 1, positions out of
 * range), ESTATE (first_position not above the newest position, or M+1
 * entries held), EHIP. */
int fademem_update(fademem_cache* cache, const void* const* k, const void* const* v, int64_t frames,
                   int64_t first_position, void* stream);

/* Zero-copy insert (Alg. S1 "Append"; Sec. 4.1 and supplementary Sec. S4:
 * one entry per latent frame, the memory updated once the chunk is
 * generated).  With stage_frames > 0, the caller's projection can write a
 * chunk's K/V straight into free pool slots instead of its own buffers:
 * fademem_stage returns, for frame f < frames of layer l, the device
 * address of the K block k[l*frames + f] and of the V block
 * v[l*frames + f] ([N][H][D] each; the frames of a chunk are separate
 * blocks).  It reads host state only and enqueues nothing; the addresses
 * stay valid until the next insert, consolidate or update.
 * fademem_update_staged(frames, first_position) then runs the same F
 * Alg. S1 updates as fademem_update with frame f taken from its staging
 * slot: a frame that survives stays where the caller wrote it (no copy) and
 * one that a merge consumes frees its slot.  State, merge log and stored
 * K/V bits equal those of fademem_update on the same frames.
 * fademem_attend_staged attends over [memory || staged frames] (the
 * generator's final pass over a chunk, whose K/V become the update's).
 * The free slots are known on the host because the library replays every
 * update's schedule on the host copy of the integer metadata (the device
 * still makes the decisions; fademem_verify checks that both agree).
 * Limits: 1 <= frames <= stage_frames <= 4.  Errors: EINVAL (frames out of
 * range, NULL pointers, positions out of range), ESTATE (M+1 entries held,
 * position not above the newest), EHIP. */
int fademem_stage(fademem_cache* cache, int64_t frames, void** k, void** v);
int fademem_update_staged(fademem_cache* cache, int64_t frames, int64_t first_position, void* stream);
int fademem_attend_staged(fademem_cache* cache, int32_t layer, const void* q, int64_t q_tokens,
                          int64_t frames, float scale, void* out, float* lse, void* stream);

/* Attention of the chunk's queries over layer `layer`'s exposed cache:
 * O_h = softmax(scale * Q_h K_h^T) V_h per head, with the keys/values
 * [memory entries in memory order || current chunk] (Sec. 3.1, Sec. 4.1),
 * no mask.  q and out: [q_tokens][H][D]; k_cur, v_cur: [cur_tokens][H][D]
 * (cur_tokens may be 0 if the memory is not empty).  scale = 0 selects
 * 1/sqrt(D).  lse, if not NULL, receives [H][q_tokens] fp32 natural-log
 * sums of exponentials of the scaled scores.  Accumulation is fp32 (bf16
 * inputs use bf16 MFMA with fp32 accumulation).  q_tokens = 0 is a no-op.
 * Errors: EINVAL (layer out of range, NULL/misaligned pointers, no keys at
 * all, sizes out of range), EHIP. */
int fademem_attend(fademem_cache* cache, int32_t layer, const void* q, int64_t q_tokens,
                   const void* k_cur, const void* v_cur, int64_t cur_tokens, float scale,
                   void* out, float* lse, void* stream);

/* Number of entries currently held (host mirror; never waits). */
int fademem_count(const fademem_cache* cache, int64_t* count);

/* Copy the memory's metadata to host arrays of at least M+1 elements (any
 * of them may be NULL): first covered position, span s_i, pos_sum_i (the
 * integer with mu_i = pos_sum_i / s_i) and the newest position.
 * Synchronises `stream`.  Errors: EINVAL, EHIP. */
int fademem_get_state(fademem_cache* cache, int64_t* count, int64_t* first, int64_t* span,
                      int64_t* pos_sum, int64_t* newest, void* stream);

/* Device pointers of layer `layer`'s logical entry i (0 = oldest), valid
 * until the next insert/consolidate.  Synchronises `stream`. */
int fademem_entry_kv(fademem_cache* cache, int32_t layer, int64_t i, const void** k,
                     const void** v, void* stream);

/* Checkpoint / resume: put a saved memory into a cache that holds nothing
 * yet (just created, same configuration), so that it continues exactly as
 * the cache the state was saved from.  count (0..M) entries, oldest first:
 * first[i], span[i], pos_sum[i] as fademem_get_state returns them, and the
 * newest inserted position; k[l*count + i], v[l*count + i] (host arrays of
 * layers*count device pointers, [N][H][D] each) are entry i's K, V of layer
 * l, e.g. from fademem_entry_kv of the saved cache or the caller's copies of
 * them (the saved state holds nothing else: entry 0 is the anchor when the
 * option is on).  The merge log and counts start again from zero.  Copies
 * on `stream` and synchronises it.  Errors: EINVAL (NULL/misaligned
 * pointers, count > M, spans < 1, first not increasing by at least the
 * previous span, pos_sum outside [first*span, newest*span], newest below
 * the last covered position, positions out of range), ESTATE (the cache
 * already holds or has held entries), EHIP. */
int fademem_set_state(fademem_cache* cache, int64_t count, const int64_t* first, const int64_t* span,
                      const int64_t* pos_sum, int64_t newest, const void* const* k, const void* const* v,
                      void* stream);

/* Selected pair indices j of the consolidations run so far, oldest first.
 * *total receives how many have run; the most recent min(total, cap, 4096)
 * are copied into j[].  Synchronises `stream`. */
int fademem_merge_log(fademem_cache* cache, int32_t* j, int64_t cap, int64_t* total,
                      void* stream);

/* Counts of the consolidations run so far (Algorithm S1's merge step):
 * *total of them, *anchor of which merged the anchor's pair (no K/V work),
 * so total - anchor merges moved K/V bytes.  Either pointer may be NULL.
 * Unlike the log these counts are not capped.  Synchronises `stream`.
 * Errors: EINVAL (NULL cache), EHIP. */
int fademem_merge_counts(fademem_cache* cache, int64_t* total, int64_t* anchor, void* stream);

/* Distance-dependent spectral decay (Sec. 3.2; supplementary Sec. S2).
 * latents: device [clips][frames][height][width] fp32, channel-averaged
 * latent frames.  For every clip the orthonormal 2-D DCT-II of frames
 * 0..max_lag; for every radial band k < bands and lag the Pearson
 * correlation of band k's DCT coefficients of frame 0 and of frame lag;
 * corr (device, [bands][max_lag+1] fp64) receives the mean over clips.
 * band_of: device [height][width] int32, the band of DCT coefficient
 * (u, v) (any value outside [0, bands) leaves the coefficient out).
 * workspace: device, 256-byte aligned, at least
 * fademem_spectral_workspace_bytes (the DCT bases, the band order and the
 * per-clip band sums; for frames larger than 64 x 128 also room for the DCT
 * of the analysed frames, used where it is not kept on chip).  Limits:
 * height*width <= 40960 and, above 64 x 128, the frame, its transform and
 * both DCT bases within 160 KiB of LDS; max_lag < frames, max_lag < 65535;
 * 1 <= bands <= 1024.  Asynchronous on `stream`; the library allocates
 * nothing.  Every call with the same inputs gives the same bits.  A band
 * whose coefficients do not vary, or that holds none, gets NaN.
 * Errors: EINVAL (NULL/misaligned pointers, sizes out of range), ENOMEM
 * (workspace too small), EHIP. */
int fademem_spectral_workspace_bytes(int64_t clips, int64_t frames, int32_t height, int32_t width,
                                     int32_t bands, int64_t max_lag, size_t* bytes);
int fademem_spectral_corr(const float* latents, int64_t clips, int64_t frames, int32_t height,
                          int32_t width, const int32_t* band_of, int32_t bands, int64_t max_lag,
                          void* workspace, size_t workspace_bytes, double* corr, void* stream);

/* Synchronise `stream` and compare the host replay of the memory (spans,
 * positions, slot table) with the device's state.  Returns OK or
 * EINTERNAL (serialize mode runs the same check after every call).
 * Errors: EINVAL (NULL cache), EHIP. */
int fademem_verify(fademem_cache* cache, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * analysis as fademem_spectral_corr, with its workspace in a static scratch
 * array of the library (64 MiB per GPU, held by each GPU the library runs on
 * until the process ends) instead of a caller's buffer; the caller still
 * passes the inputs and corr.  The call allocates nothing.  Requests whose
 * workspace (fademem_spectral_workspace_bytes) exceeds 64 MiB return
 * FADEMEM_ESCRATCH before anything is enqueued (the 374-clip analysis of
 * supplementary Sec. S2 needs 38.2 MB).  All calls on one GPU share its
 * scratch: calls that overlap on one GPU (several streams or threads) race.
 * Errors: as fademem_spectral_corr, plus ESCRATCH. */
int fademem_spectral_corr_static(const float* latents, int64_t clips, int64_t frames, int32_t height,
                                 int32_t width, const int32_t* band_of, int32_t bands, int64_t max_lag,
                                 double* corr, void* stream);

/* Host steps of the spectral-decay analysis (Sec. 3.2; supplementary Sec.
 * S2) on small host arrays; they read and write host memory only, enqueue
 * nothing and need no device.  The paper gives the radial frequency, the
 * horizon as the onset of the near-flat regime after the main decay, and a
 * nonlinear least-squares fit of r*(t) = a t^(-b); the band edges, the
 * smoothing and the threshold are this library's readings.
 *
 * fademem_spectral_band_map: band_of (host int32 [height][width]) receives
 * the band of DCT coefficient (u, v): `bands` equal-width bins of
 * r = sqrt((u/H)^2 + (v/W)^2) over [0, max r], the last bin closed, the DC
 * coefficient -1 (left out); centres (host double [bands], may be NULL)
 * the bins' centre radii.  1 <= height, width <= 1024, 1 <= bands <= 1024.
 *
 * fademem_spectral_horizons: corr (host double [bands][lags], row k = band
 * k's C_k(lag)); each row is smoothed by a centred moving average over
 * `window` lags (shrinking at the ends); horizon[k] (host int64 [bands]) is
 * the first lag >= 1 at which the smoothed curve has made at least half of
 * its total decay and falls to the next lag by less than `drop` times its
 * steepest one-lag fall, or -1 (the defaults used here: window 5, drop 0.05).
 *
 * fademem_spectral_fit: (a, b) of r = a t^(-b) minimising sum (r_i - a
 * t_i^(-b))^2 over n >= 2 points with t_i, r_i > 0: Gauss-Newton from the
 * straight-line fit of log r on log t, at most `iters` steps.
 *
 * Errors: EINVAL (NULL pointers, sizes out of range, non-positive or
 * infinite points, a fit that does not converge to finite values), ENOMEM. */
int fademem_spectral_band_map(int32_t height, int32_t width, int32_t bands, int32_t* band_of, double* centres);
int fademem_spectral_horizons(const double* corr, int32_t bands, int64_t lags, int32_t window, double drop,
                              int64_t* horizon);
int fademem_spectral_fit(const double* t, const double* r, int64_t n, int32_t iters, double* a, double* b);

/* Rotary positions with several axes (time, height, width): the rotation a
 * caller applies to a chunk's queries and keys.  With fademem_config's
 * rope_pairs the memory turns its own keys by their entry index (Sec. 3.3
 * "Boundary and positional handling"); the time axis here is the same
 * rotation, by the same pairs and frequencies.  Both are evaluated in fp64, by
 * code of their own: an element of one may be the neighbour of the other's
 * where the fp64 value lies next to the border of a rounding.
 * Pair p of a head turns by the angle pos[row][axis of p] * freq[p]:
 * (x0, x1) -> (x0 cos - x1 sin, x0 sin + x1 cos), evaluated in fp64 and
 * rounded once to the storage type.  The first pairs[0] pairs follow axis 0
 * (time), the next pairs[1] axis 1 (height), the next pairs[2] axis 2 (width);
 * pairs behind them are copied.  layout: pair p is elements (2p, 2p+1)
 * (INTERLEAVED) or (p, p + head_dim/2) (HALVES). */
enum { FADEMEM_ROPE_INTERLEAVED = 0, FADEMEM_ROPE_HALVES = 1 };
enum { FADEMEM_ROPE_MAX_PAIRS = 128 };

typedef struct fademem_rope {
  int32_t head_dim;        /* multiple of 16, 16..256                          */
  int32_t layout;          /* FADEMEM_ROPE_*                                   */
  int32_t pairs[3];        /* >= 0 each, their sum 1..head_dim/2               */
  double freq[FADEMEM_ROPE_MAX_PAIRS]; /* radians per position, finite         */
} fademem_rope;

/* Fill `rope` (host memory): pair k of an axis with P pairs gets the
 * frequency theta^(-k/P).  A caller may change freq[] afterwards.
 * Errors: EINVAL (NULL, sizes out of range, theta not in (1, 1e300)). */
int fademem_rope_init(fademem_rope* rope, int32_t head_dim, int32_t layout, int32_t pairs_t, int32_t pairs_h,
                      int32_t pairs_w, double theta);

/* Rotate `rows` rows (at most 2^23) of `heads` heads: y[i][h] = x[i][h] turned to position
 * pos[i] (device int32 [rows][3]; any int32 values).  x and y: device, rows
 * x_stride / y_stride elements apart (>= heads * head_dim, a multiple of 16
 * bytes), heads and elements contiguous, dtype FADEMEM_F32 or FADEMEM_BF16.
 * y may be x (same stride); otherwise no row of y may overlap a row of x.
 * inverse = 1 turns by the negative angles: the gradient with respect to x is
 * the inverse rotation of the gradient with respect to y.  rows = 0 is a
 * no-op.  Asynchronous on `stream`, on the current device.
 * Errors: EINVAL (NULL/misaligned pointers, sizes, strides or overlap, a bad
 * rotation), EHIP. */
int fademem_rope_apply(const fademem_rope* rope, int32_t dtype, const int32_t* pos, int64_t rows, int32_t heads,
                       const void* x, int64_t x_stride, void* y, int64_t y_stride, int32_t inverse, void* stream);

/* Paged window memory: the comparison memory of Sec. 4 (the first frames as
 * sinks that stay visible, and a sliding window of the latest ones) for many
 * sequences at once.  K and V lie in pages of page_tokens tokens that all
 * sequences share; a table per sequence maps its tokens to pages.  A step
 * appends new tokens to every sequence:
 *   fademem_paged_plan    pages, slots and positions of the step, on the GPU;
 *   fademem_paged_insert  per layer: the step's K (rotated or not) and V into
 *                         the pages;
 *   fademem_paged_attend  per layer: attention of the step's queries.
 * All three take their lengths from device memory, so a captured graph of
 * them replays with other lengths; none waits for the device.
 *
 * Visibility.  Token p of a sequence lies in block b = p / block_tokens.  Its
 * query sees the sequence's held tokens of blocks <= b that are among the
 * first `sinks` blocks or the last `window` blocks up to b (window = 0: all
 * of them).  block_tokens = 1 is the causal mask of a language model;
 * block_tokens = a chunk's tokens lets the tokens of a chunk see each other
 * and a window of chunks.
 *
 * Rows.  A step's rows (of q, k, v, out) are the new tokens of sequence 0,
 * then of sequence 1, ...; row i of sequence s is row q_start[s] + i.  Rows
 * behind the last sequence's are neither read nor written.
 *
 * The pool, the calls' buffers and the stream are used as fademem_cache uses
 * its own: one store is used by one host thread and one stream at a time (its
 * plan and its scratch too: two captured graphs of one store must not replay
 * at the same time).  insert and attend belong to the plan before them; one that
 * finds a plan of other `rows` or `max_new` on the device (a graph of them alone
 * replayed after a different plan) does nothing.  Calls are made with the device current that was
 * current at creation (EINVAL otherwise).  FADEMEM_SERIALIZE works as above. */
typedef struct fademem_paged_config {
  int32_t seqs;          /* sequences, 1..1024                                  */
  int32_t layers;        /* 1..4096; all layers share tables and page numbers  */
  int32_t heads;         /* query heads, a multiple of kv_heads                */
  int32_t kv_heads;      /* >= 1                                               */
  int32_t head_dim;      /* 64 or 128                                          */
  int32_t dtype;         /* FADEMEM_F32 or FADEMEM_BF16 for K, V, Q, O         */
  int32_t page_tokens;   /* P, 1..65536.  Multiples of 64 are read fastest     */
  int32_t sinks;         /* S >= 0, first blocks that stay visible             */
  int64_t pages;         /* pages of the pool, 1..2^24                         */
  int64_t max_tokens;    /* tokens of one sequence at most, 1..2^30            */
  int64_t max_rows;      /* rows of one step at most, 1..2^23; with G = heads /
                            kv_heads, max_rows * G and (max_rows * G / 32 +
                            seqs) * kv_heads are at most 2^30                  */
  int64_t block_tokens;  /* B, 1..2^30                                         */
  int64_t window;        /* blocks; 0: everything held is visible              */
  int32_t grid_h;        /* token p's position is (p / (grid_h * grid_w),      */
  int32_t grid_w;        /* p / grid_w % grid_h, p % grid_w); 1 x 1: (p, 0, 0) */
} fademem_paged_config;

typedef struct fademem_paged fademem_paged; /* opaque host object */

/* Bytes of device pool: tables, the step's plan, the attention's scratch for
 * split work, and per layer [pages][K|V][kv_heads][page_tokens][head_dim]
 * (one page of K and V: 2 GiB at most).  Errors: EINVAL. */
int fademem_paged_bytes(const fademem_paged_config* cfg, size_t* bytes);

/* Create a store over a caller-owned pool (256-byte aligned); every sequence
 * empty, every page free.  Enqueues the initialisation on `stream`; the pages'
 * contents are left as they are.  Errors: EINVAL, ENOMEM, EHIP. */
int fademem_paged_create(const fademem_paged_config* cfg, void* dev_pool, size_t pool_bytes, void* stream,
                         fademem_paged** out);
int fademem_paged_destroy(fademem_paged* paged);

/* Plan a step: sequence s keeps its first kept[s] tokens (fewer than it
 * holds: it goes back, so that a chunk can be denoised again or rejected
 * tokens dropped; 0: it starts again) and appends added[s] tokens behind them.
 * kept, added: device int32 [seqs], read when the stream gets there.  rows:
 * rows of the step's buffers, at least the sum of added; max_new: the most
 * that any added[s] is (it chooses the attention kernel).
 * Pages that lie wholly between the sinks and the window of token kept[s], or
 * behind the new end, are given back; then the lowest free page numbers go to
 * the sequences in order.  The same call again changes nothing.
 * status[s]: OK; EINVAL: kept[s] < 0 or above what is held, added[s] < 0 or
 * > max_new, more than max_tokens or `rows` in all (nothing of s changes);
 * ESTATE: kept[s] is behind pages already given back (nothing changes);
 * ENOMEM: not enough free pages for it and the sequences before it (it keeps
 * its first kept[s] tokens; no later sequence gets pages either).  The rows
 * of such a sequence are not inserted (slot -1), and their attention is 0,
 * LSE minus infinity.
 * Errors: EINVAL (NULL, rows outside 0..max_rows, max_new outside 0..rows),
 * EHIP. */
int fademem_paged_plan(fademem_paged* paged, const int32_t* kept, const int32_t* added, int64_t rows, int64_t max_new,
                       void* stream);

/* Device arrays of the store, *count elements (NULL: not wanted): valid for
 * its lifetime, written by fademem_paged_plan (PAGES: by
 * fademem_paged_insert).  Reads host state only.
 * Errors: EINVAL (NULL, unknown array, layer out of range). */
enum {
  FADEMEM_PAGED_Q_START = 0,   /* int32 [seqs + 1]: first row of each sequence */
  FADEMEM_PAGED_SLOTS = 1,     /* int64 [max_rows]: page * P + offset, or -1;
                                  the step's rows are written               */
  FADEMEM_PAGED_POSITIONS = 2, /* int32 [max_rows][3], 0 where the slot is -1  */
  FADEMEM_PAGED_STATUS = 3,    /* int32 [seqs]                                 */
  FADEMEM_PAGED_HELD = 4,      /* int32 [seqs]: tokens held, with the new ones */
  FADEMEM_PAGED_TABLE = 5,     /* int32 [seqs][ceil(max_tokens / P)], -1: none */
  FADEMEM_PAGED_FREE = 6,      /* int32 [1]: free pages                        */
  FADEMEM_PAGED_PAGES = 7      /* dtype, the layer's pages as laid out above   */
};
int fademem_paged_array(const fademem_paged* paged, int32_t which, int32_t layer, void** ptr, int64_t* count);

/* Write the planned step's keys and values into layer `layer`'s pages, the
 * keys turned to their rows' POSITIONS by `rope` (host, NULL: as they are;
 * its head_dim is the store's).  k, v: [rows][kv_heads][head_dim], rows
 * k_stride / v_stride elements apart (multiples of 16 bytes).
 * Errors: EINVAL, ESTATE (no step planned yet), EHIP. */
int fademem_paged_insert(fademem_paged* paged, int32_t layer, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, const fademem_rope* rope, void* stream);

/* Attention of the planned step's queries over layer `layer`'s pages, the
 * step's own tokens among them (insert first): query head h of row i reads
 * key head h / (heads / kv_heads); O = softmax(scale Q K^T) V over the keys
 * that the row sees.  q, out: [rows][heads][head_dim], rows q_stride /
 * out_stride elements apart; out must not overlap q.  scale = 0 selects
 * 1/sqrt(D); negative scales are refused.  lse, if not NULL: [heads][rows]
 * fp32.  Keys that a row does not see do not reach it, whatever their values
 * (infinities and NaN too); rows whose result is not finite are worked out
 * again key by key, which takes far longer than a call without them.
 * FADEMEM_F32 holds 32 bits throughout.  FADEMEM_BF16: scores, row maxima, sums
 * and O in fp32, the softmax weights rounded to bf16 for the products with V,
 * weights below 2^-126 zero, O rounded once.
 * Errors: EINVAL, ESTATE (no step planned yet), EHIP. */
int fademem_paged_attend(fademem_paged* paged, int32_t layer, const void* q, int64_t q_stride, float scale, void* out,
                         int64_t out_stride, float* lse, void* stream);

/* hipError_t value of the last FADEMEM_EHIP on this store (0 if none). */
int fademem_paged_last_hip_error(const fademem_paged* paged);

/* hipError_t value of the last FADEMEM_EHIP on this cache (0 if none). */
int fademem_last_hip_error(const fademem_cache* cache);

/* Static description of an error code. */
const char* fademem_strerror(int code);

#ifdef __cplusplus
}
#endif

#endif /* FADEMEM_H */
