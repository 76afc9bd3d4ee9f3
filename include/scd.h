/*
 * scd.h -- C ABI of the MI355X (gfx950) library for the per-iteration
 * draft-and-verify pass of Speculative Coupled Decoding (SCD).
 *
 * What one iteration computes (appendix "Algorithms", Alg. SCD(pi_MC); Sec. 4.3
 * "Implementation Details"; Alg. 1 "Modified Rejection Sampling"):
 *   1. Evaluate: LM-head logits of the L window positions,
 *        logit[m, v] = sum_k h[m, k] * W[v, k]           (bf16 in, fp32 accumulate)
 *   2. logit post-processing, which defines p^(t) (Sec. 4.3, last sentence;
 *      Sec. 5.1 "Effect on CFG"; appendix "Experimental Details"):
 *        z = (1 + lambda) * c - lambda * u   (classifier-free guidance, C = 2 rows)
 *        ids outside [v_lo, v_hi) are masked out;  z <- z / tau
 *        keep the ids with z >= (K-th largest z);  p = softmax over the kept ids
 *   3. one Modified-Rejection-Sampling call per window position, no break:
 *        u ~ U(0,1);  accept iff  u * q(x) <= p(x)              (k = 1, y = x)
 *        else y ~ norm(max(0, p - q))                             (k = 0)
 *      q is the position's distribution from the previous iteration (uniform
 *      over the allowed ids if it was never evaluated), x its current draft.
 *   4. first rejection r: emit y[0..a), a = min(r + 1, Lw) (a = Lw if none);
 *      the y right of r are the coupled redraft = next iteration's drafts;
 *      slide the window by a and give the entering positions uniform drafts.
 * With coupling = SCD_COUPLING_GS (Alg. "GS(P, Q, G)", appendix Alg. SCD(pi_GS)) steps 1-3
 * and the emission are the same; the redraft of the positions right of r is instead the
 * shared-noise Gumbel-max draw from the position's new distribution,
 *        g = argmax_v (log p(v) + G_j(v)),  G_j(v) = -ln(-ln U_j(v)),
 * with noise that depends on the position j (and the id v) only, not on the iteration,
 * decided as the equivalent exponential race argmin_v -ln(U_j(v)) / p(v) in fp32.
 * With sjd_mix > 0 (alpha-coupling, Sec. 5.3 and appendix Alg. "alpha-Coupling
 * Implementation", alpha = 1 - sjd_mix): per redraft one uniform u (stream 4); if
 * u <= alpha (fp32, alpha = fl(1 - sjd_mix)) the coupled redraft above is taken, otherwise an
 * independent draw from p: the same race with noise keyed by position AND iteration (stream 5).
 *
 * Conventions
 *   - Every pointer named d_* is a DEVICE pointer owned by the caller.  The
 *     library allocates no device memory, frees nothing of the caller's and
 *     never synchronises the stream (scd_status is the one exception).
 *   - Every call returns SCD_OK (0) or a negative scd_error.  No exceptions,
 *     no errno, no global state (the one exception: the library remembers, per
 *     GPU, the address of the static scratch of scd_couple_draft_static).  Kernels are launched asynchronously on the
 *     HIP stream given to scd_create.
 *   - A context is not thread-safe; distinct contexts are independent.
 *   - "Allowed ids" A = [v_lo, v_hi), n = |A|.  Tokens in x / y / the state are
 *     OFFSETS into A (0..n-1); emitted tokens (out) are real ids v_lo + offset.
 *     Processed logits z hold only the n allowed columns.
 *   - Rows of up to 65536 allowed ids support every option.  Longer rows are supported with
 *     top-k and the maximal coupling only; Gumbel sharing, sjd_mix > 0, top_p and diagnostics on
 *     such rows are refused by scd_create with SCD_EUNSUPPORTED.
 *   - Window order: row s of a [B, L, ...] array belongs to position pos0[b]+s.
 *     Lw_b = min(L, N - pos0[b]) rows are live; the rest are ignored on input
 *     and written as y = -1, k = 1 on output.
 *   - Random numbers: Philox4x32-10, key = (seed low 32, seed high 32),
 *     counter = (vocab offset >> 2 or 0, position, iteration, b << 8 | stream),
 *     lane = vocab offset & 3 (lane 0 for scalar draws); streams 0 = initial
 *     draft, 1 = accept uniform, 2 = residual race, 3 = Gumbel noise (iteration
 *     word 0), 4 = alpha-coupling switch, 5 = independent redraft.
 *     u = ((bits >> 9) + 0.5) * 2^-23.
 */
#ifndef SCD_H
#define SCD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct scd_ctx scd_ctx; /* opaque, host memory, owned by the library */

typedef struct scd_config {
  int32_t B;           /* sequences decoded together, >= 1                         */
  int32_t L;           /* Jacobi window length, 1..256                              */
  int32_t N;           /* tokens to generate per sequence, >= 1                     */
  int32_t V;           /* vocabulary size = rows of W                               */
  int32_t d;           /* hidden size, multiple of 8; 0 => no LM head (logits given) */
  int32_t v_lo, v_hi;  /* allowed ids [v_lo, v_hi), 0 <= v_lo < v_hi <= V;
                          L * (v_hi - v_lo) must stay below 2^31                    */
  int32_t top_k;       /* 0 => off; K = min(top_k, n)                               */
  float temperature;   /* tau > 0                                                   */
  float cfg_lambda;    /* 0 => no guidance (C = 1); else C = 2, z = (1+l)c - l u    */
  int32_t coupling;    /* scd_coupling: 0 = maximal coupling (MRS), 1 = Gumbel sharing */
  float sjd_mix;       /* 1 - alpha of the alpha-coupling (Sec. 5.3): probability that a
                          redraft is an independent draw from p instead of the coupled one;
                          0 = SCD (default), 1 = vanilla SJD; must be in [0, 1]          */
  float top_p;         /* nucleus filter (appendix "Experimental Details", video setting
                          p = 0.8), applied to the distribution that top-k leaves: of the ids
                          in order of decreasing probability the shortest prefix whose mass
                          reaches top_p is kept, ids tied with its last member included;
                          0 or 1 => off; must be in [0, 1]; needs v_hi - v_lo <= 65536.
                          Decided on 2^-40 fixed-point masses of expf(z - max), exactly:
                          mass above an id * 2^24 < round(top_p * 2^24) * total mass          */
  int32_t diagnostics; /* 1 => every scd_step also writes the per-position statistics of the
                          paper's analysis (Sec. 3: acceptance rate beta = 1 - D_TV(p, q),
                          Prop. "SJD Collision Probability": C = sum_v p_v q_v and the two
                          sums its Renyi-2 bound needs) to SCD_F_DIAG and the number of changed
                          drafts (Hamming distance between the drafts 1, 2 and 3 iterations
                          apart, Sec. 5.3 "Multi-Step Behavior") to SCD_F_HAMM;
                          0 => off; needs v_hi - v_lo <= 65536                               */
  uint64_t seed;
} scd_config;

typedef enum scd_coupling {
  SCD_COUPLING_MC = 0,   /* survivors' next drafts = their MRS outputs (Sec. 4.1)            */
  SCD_COUPLING_GS = 1    /* survivors' next drafts = shared-noise Gumbel-max draws; needs
                            v_hi - v_lo <= 65536                                             */
} scd_coupling;

typedef enum scd_error {
  SCD_OK = 0,
  SCD_EINVAL = -1,       /* bad argument or configuration                       */
  SCD_EWORKSPACE = -2,   /* workspace pointer null / misaligned / too small      */
  SCD_EHIP = -3,         /* a HIP runtime call or kernel launch failed           */
  SCD_ENUMERIC = -4,     /* a logit row had no finite value or a NaN (scd_status) */
  SCD_EUNSUPPORTED = -5, /* valid request this build does not implement          */
  SCD_ESCRATCH = -6      /* scd_couple_draft_static: the configuration needs more than
                            SCD_STATIC_SCRATCH_BYTES of scratch                   */
} scd_error;

/* Fields of the device-resident decode state, for scd_state_field. */
typedef enum scd_field {
  SCD_F_POS = 0,      /* int32 [B]       accepted-prefix pointer i_b                   */
  SCD_F_ITER = 1,     /* int32 [B]       iterations done t_b (= NFE)                   */
  SCD_F_X = 2,        /* int32 [B, L]    draft token offsets, ring slot = position % L */
  SCD_F_AGE = 3,      /* int32 [B, L]    earlier evaluations of the slot's position    */
  SCD_F_OUT = 4,      /* int32 [B, N]    emitted token ids, -1 where not yet emitted   */
  SCD_F_ACCEPT = 5,   /* int32 [B]       tokens emitted by the last step               */
  SCD_F_Y = 6,        /* int32 [B, L]    last step's MRS outputs, window order         */
  SCD_F_K = 7,        /* uint8 [B, L]    last step's accept bits, window order         */
  SCD_F_PX = 8,       /* float [B, L]    last step's p(x), window order                */
  SCD_F_QX = 9,       /* float [B, L]    last step's q(x), window order                */
  SCD_F_THR = 10,     /* float [2, B, L] smallest kept logit (top-k / nucleus threshold; -inf when
                                         neither filters) per parity (t & 1) and slot  */
  SCD_F_LSE = 11,     /* float [2, B, L] log normaliser per parity and slot            */
  SCD_F_NKEPT = 12,   /* int32 [2, B, L] size of the kept set per parity and slot      */
  SCD_F_Z = 13,       /* float [2, B, L, n] processed logits per parity and slot       */
  SCD_F_FLAGS = 14,   /* int32 [4]       [0] numeric-fault bits                        */
  SCD_F_VERIFIED = 15,/* int32 [B]       window positions verified so far (sum of Lw)  */
  SCD_F_TICKET = 16,  /* int32 [B]       internal arrival counters, zero between steps */
  SCD_F_G = 17,       /* int32 [B, L]    last step's Gumbel-sharing / independent redraft draws,
                                         window order; -1 where the row drew none (written
                                         under SCD_COUPLING_GS or sjd_mix > 0 only)      */
  SCD_F_DIAG = 18,    /* float [B, L, 4] last step, window order (diagnostics = 1 only):
                                         [0] beta = sum_v min(p_v, q_v) = 1 - D_TV(p, q)
                                         [1] C = sum_v p_v q_v
                                         [2] sum_v p_v^2 = exp(-H_2(p))   [3] sum_v q_v^2
                                         (C <= sqrt([2] * [3])); p = this iteration's
                                         distribution of the position, q = the one its draft
                                         came from (uniform for a first evaluation); rows that
                                         are not live hold zeros                             */
  SCD_F_S2 = 19,      /* float [2, B, L] internal: sum_v p_v^2 per parity and slot            */
  SCD_F_HAMM = 20,    /* int32 [B, 6]    last step (diagnostics = 1 only): for n = 1, 2, 3 the pair
                                         (differing, compared) of Hamm(t + 1 - n, t + 1): the
                                         window's drafts after the step against the drafts n
                                         iterations earlier, over the positions in both windows
                                         (n = 1: the surviving positions whose draft changed)  */
  SCD_F_XHIST = 21,   /* int32 [3, B, L] internal: drafts at the start of the last 3 iterations */
  SCD_F_PHIST = 22,   /* int32 [3, B]    internal: window starts of those iterations            */
  SCD_F_COUNT = 23
} scd_field;

/* Bytes of caller-provided device scratch a context needs; 0 on a bad config.  Nothing in it outlives
 * a call.  scd_couple_draft writes it, and so do scd_select, scd_step, scd_step_quantized, scd_step_fp8 and scd_step_logits where a
 * top-k of up to 3072 filters rows of more than 16384 ids; those calls must not overlap in time on
 * the GPU with others that were given the same workspace. */
size_t scd_workspace_bytes(const scd_config* cfg);

/* Bytes of the device-resident decode state; 0 on a bad config.  The fields of scd_field come first;
 * behind them, where scd_step deals the LM head's k over workgroups (short rows, few of them), lie
 * that step's partial sums, up to 4 MiB of which nothing outlives the step. */
size_t scd_state_bytes(const scd_config* cfg);

/* Validates cfg, copies it, remembers the workspace (256-byte aligned device
 * memory of >= scd_workspace_bytes, kept by the caller until scd_destroy) and
 * the HIP stream (a hipStream_t passed as void*, NULL = default stream).
 * *out is set only on SCD_OK. */
int scd_create(scd_ctx** out, const scd_config* cfg, void* d_workspace, size_t workspace_bytes,
               void* hip_stream);

/* Frees the host-side context.  Touches no device memory. */
int scd_destroy(scd_ctx* ctx);

/* Initialises a state buffer (256-byte aligned, >= scd_state_bytes): i_b = 0,
 * t_b = 0, the first min(L, N) positions get uniform initial drafts, out = -1.
 * Asynchronous. */
int scd_reset(scd_ctx* ctx, void* d_state);

/* Host-only address arithmetic: pointer and size of one field inside d_state. */
int scd_state_field(const scd_ctx* ctx, void* d_state, int field, void** d_ptr, size_t* bytes);

/* Step 1+2a (Evaluate + CFG + mask + temperature) for all B*L window rows.
 *   d_h  bf16 bits [B, C, L, d] row-major (C = 2: cond rows then uncond rows of
 *        each sequence);  d_W bf16 bits [V, d] row-major; only rows
 *        [v_lo, v_hi) are read;  d_z fp32 [B, L, n] window order, written.
 * Requires cfg.d > 0. */
int scd_lm_head(scd_ctx* ctx, const uint16_t* d_h, const uint16_t* d_W, float* d_z);

/* Step 2b (top-k threshold + softmax normaliser) for rows of processed logits.
 *   d_z fp32 [rows, n];  outputs per row: d_thr (K-th largest value, -inf if
 *   top-k is off or K >= n), d_lse (log of the sum of exp over the kept ids),
 *   d_nkept (size of the kept set).  p_v = [z_v >= thr] * exp(z_v - lse). */
int scd_select(scd_ctx* ctx, const float* d_z, int32_t rows, float* d_thr, float* d_lse,
               int32_t* d_nkept);

/* Step 3: vectorised MRS = speculative verification and maximal-coupling
 * redraft in one call (Alg. 1; Alg. SCD(pi_MC) parallel-for).
 *   d_z_cur, d_z_prev fp32 [B, L, n] processed logits of this / the previous
 *   iteration, window order;  d_x int32 [B, L] draft token offsets;
 *   d_fresh uint8 [B, L], nonzero = never evaluated (q uniform; the d_z_prev row
 *   must be readable, its values decide nothing), may be NULL = none fresh;  d_pos0 int32 [B];  iter = iteration
 *   index used in the random-number counters;
 *   outputs d_y int32 [B, L], d_k uint8 [B, L]. */
int scd_couple_draft(scd_ctx* ctx, const float* d_z_cur, const float* d_z_prev,
                     const int32_t* d_x, const uint8_t* d_fresh, const int32_t* d_pos0,
                     int32_t iter, int32_t* d_y, uint8_t* d_k);

/* scd_couple_draft for callers that cannot allocate device memory -- code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels,
 * same results; the scratch that scd_couple_draft keeps in the context's workspace (per-row
 * thresholds / normalisers / kept counts of both logit arrays and the rows' candidate
 * lists) lives in a static device array of SCD_STATIC_SCRATCH_BYTES inside the library instead
 * (one copy per GPU, held until the process ends).  The call allocates and frees nothing and
 * does not touch the context's workspace.  Returns SCD_ESCRATCH when the configuration needs
 * more: 24 bytes per window row (B * L rows, each of the six arrays rounded up to 256 bytes),
 * plus 51200 bytes per window row when top-k filters rows of 16385..65536 ids with
 * top_k <= 3072 (their candidate lists), i.e. up to 163 such rows.  Longer rows take
 * the lists while they fit; beyond that they are read whole, and their normalisers, summed in
 * another order, may differ from scd_couple_draft's in the last bits.
 * All calls on one GPU share that array and it keeps the last call's contents (nothing in it has
 * to start at zero): calls that overlap in time on one GPU -- different streams or contexts --
 * race.  The array's address is looked up once per GPU, in scd_create when a GPU is present,
 * else in the first call. */
#define SCD_STATIC_SCRATCH_BYTES (8u << 20)
int scd_couple_draft_static(scd_ctx* ctx, const float* d_z_cur, const float* d_z_prev,
                            const int32_t* d_x, const uint8_t* d_fresh, const int32_t* d_pos0,
                            int32_t iter, int32_t* d_y, uint8_t* d_k);

/* Step 4 without the slide: first rejection per sequence, accept length and
 * emitted tokens (Alg. SCD(pi_MC), "find first rejection index").
 *   d_k, d_y [B, L] from scd_couple_draft; d_pos0 [B];
 *   d_accept_len int32 [B] written; d_out int32 [B, N]: entries
 *   [pos0, pos0 + accept_len) written with v_lo + y. */
int scd_verify(scd_ctx* ctx, const uint8_t* d_k, const int32_t* d_y, const int32_t* d_pos0,
               int32_t* d_accept_len, int32_t* d_out);

/* One whole iteration (steps 1-4 incl. window slide) on the device-resident
 * state.  d_h as in scd_lm_head for the CURRENT windows (row s <-> position
 * i_b + s; rows past the sequence end are ignored but must be readable).
 * Finished sequences cost nothing and change nothing.  Requires cfg.d > 0.
 * On rows of up to 4096 ids, if they are few, the logits are added up over k in another order than
 * scd_lm_head's: the two may differ in the last bits there, and so may a decision that hangs on
 * them.  On all other shapes the logits are the same. */
int scd_step(scd_ctx* ctx, const uint16_t* d_h, const uint16_t* d_W, void* d_state);

/* Optional instrumentation for benchmarks: while both events are non-NULL,
 * scd_step, scd_step_quantized and scd_step_fp8 launch the LM-head kernel with the two events attached to the
 * dispatch (hipExtLaunchKernel): ev_start takes the kernel's start time, ev_stop
 * its stop time, on the context's stream; no other packet enters the stream
 * (hipEvent_t passed as void*, owned by the caller).  NULL, NULL turns it off.
 * Host-only call. */
int scd_set_lm_head_events(scd_ctx* ctx, void* ev_start, void* ev_stop);

/* For reports: writes the name of the LM-head kernel that scd_step / scd_lm_head launch
 * for this context's sizes, NUL-terminated, into host_buf[0..cap).  Template arguments:
 * lm_head_tile_kernel<1 + CFG, h rows, columns, stages, W past the caches>,
 * lm_head_splitk_kernel<row blocks, 1 + CFG, wavefronts>,
 * lm_head_kernel<row blocks, 1 + CFG, wavefronts, W past the caches>.
 * Where the two launch different kernels (scd_step deals k over workgroups of a tile kernel, and
 * its row kernel adds the parts up) both names are written, "scd_step's / scd_lm_head's"; scd_step's
 * alone if cap does not hold both (95 characters always do).
 * Returns SCD_OK, or SCD_EINVAL (NULL argument, cfg.d == 0, or cap too small).
 * Host-only call. */
int scd_lm_head_kernel_name(scd_ctx* ctx, char* host_buf, size_t cap);

/* The same iteration with the processed logits supplied by the caller
 * (d_z fp32 [B, L, n], window order) instead of computed by the LM head. */
int scd_step_logits(scd_ctx* ctx, const float* d_z, void* d_state);

/* ---- the LM head over 4-bit weights -----------------------------------------------------------
 *   W[v, k] = s[v, k / group] * (q[v, k] - o[v, k / group]),   q in 0..15, o = 8, or a zero point of 0..15.
 * group: weights of a row that share a scale, a multiple of 32 up to 65536 (the last group of a row may be shorter), at most 256
 * groups per row.  Row-major arrays, as a checkpoint holds them: d_codes uint8 [V, d / 2], even k in the low half of a
 * byte (4-byte aligned); d_scales bf16 [V, G] and d_zeros uint8 [V, G] (NULL: o = 8), G = ceil(d / group).  The steps read
 * them in another layout, made once by scd_pack_quantized.  All need cfg.d in 8 .. 2^20. */
typedef struct scd_quantized {
  const void* d_packed;   /* written by scd_pack_quantized for this configuration's allowed ids and d */
  int32_t group;
  int32_t zeros;          /* 1: with zero points, 0: without                                           */
} scd_quantized;

/* Bytes of the layout; 0 on a bad configuration or group. */
size_t scd_quantized_bytes(const scd_config* cfg, int32_t group, int32_t zeros);

/* Quantises W bf16 [V, d] (finite): codes and scales, and zero points unless d_zeros is NULL.  Without them s = max(largest / 7,
 * -smallest / 8) of a group, with them s = (largest - smallest) / 15 over a range that holds 0, rounded to bf16; the
 * codes are the nearest. */
int scd_quantize(scd_ctx* ctx, const uint16_t* d_W, int32_t group, uint8_t* d_codes, uint16_t* d_scales, uint8_t* d_zeros);

/* Lays the allowed rows out: d_packed, scd_quantized_bytes(cfg, group, d_zeros != NULL) bytes, 256-byte aligned.  Zero points above 15
 * count as 15. */
int scd_pack_quantized(scd_ctx* ctx, const uint8_t* d_codes, const uint16_t* d_scales, const uint8_t* d_zeros, int32_t group,
                       void* d_packed);

/* scd_lm_head and scd_step with these weights in the place of W.  The products are exact and summed in fp32: no weight is
 * rounded to bf16.  Meant for few rows on large tables, in groups of 64 or more; batches of some hundred rows, and groups of 32 with zero
 * points, take longer than over W in bf16. */
int scd_lm_head_quantized(scd_ctx* ctx, const uint16_t* d_h, const scd_quantized* W, float* d_z);
int scd_step_quantized(scd_ctx* ctx, const uint16_t* d_h, const scd_quantized* W, void* d_state);

/* scd_lm_head_kernel_name of these two, which launch the same kernel:
 * lm_head_quantized_kernel<QuantCfg<1 + CFG, blocks of 32 rows, rows of a block that are loaded, column tiles of a wavefront, wavefronts,
 * of which share k, KB of LDS, of which share columns>, k of a scaling / 16, zero points> (127 characters hold it). */
int scd_lm_head_quantized_kernel_name(scd_ctx* ctx, int32_t group, int32_t zeros, char* host_buf, size_t cap);

/* ---- the vocabulary table at the model's other end, and what it learns -------------------------
 * The same table W, bf16 bits [V, d] row-major, all pointers 16-byte aligned (d_ids, d_targets and the
 * float arrays 4-byte).  All of them need cfg.d > 0 (up to 2^24); of the rest of the configuration they use what is
 * named below, so a context with B = L = N = 1 serves a program that decodes nothing.  `rows` = 0 is allowed (arrays of
 * no elements may then be NULL), up to 2^25 ids (the gradient of more than 2^20 takes a time that grows with their square) or 2^20 rows
 * of the loss.  Workspaces are the caller's, 256-byte aligned, of the size that the
 * query gives for the same arguments (0 for bad ones); nothing in one outlives the call.  Calls on different
 * streams, contexts or in different recorded graphs must not share one if they may overlap in time. */

/* Type of a gradient of W. */
typedef enum scd_grad_type {
  SCD_GRAD_BF16 = 0,
  SCD_GRAD_F32 = 1
} scd_grad_type;

/* x[r] = scale * W[id_r], rounded once.  d_ids int32 [rows], ids of the whole vocabulary (not offsets); an id outside
 * [0, V) (padding) gives zeros.  d_x bf16 [rows, d], written. */
int scd_embed(scd_ctx* ctx, const int32_t* d_ids, int32_t rows, const uint16_t* d_W, float scale, uint16_t* d_x);

/* The same for the drafts in the decode state, as the model reads them before the next scd_step: d_x bf16
 * [B, C, L, d] as d_h there, row s of a sequence <-> position i_b + s, zeros for rows past the sequence's end; with
 * guidance the uncond rows get the same. */
int scd_embed_window(scd_ctx* ctx, const void* d_state, const uint16_t* d_W, float scale, uint16_t* d_x);

/* Gradient of scd_embed with respect to W: d_dW[v] = scale * sum of d_dx[r] over the rows with id_r = v, added up in 32
 * bits in an order that depends on the ids alone (the same call gives the same bits), rounded once.
 *   d_dx bf16 [rows, d];  d_dW [V, d] of type grad_type: with accumulate = 0 every row is written (zeros where no id
 * points), with accumulate = 1 the sum is added to the rows that occur, the others are left alone. */
size_t scd_embed_backward_workspace_bytes(const scd_config* cfg, int32_t rows);
int scd_embed_backward(scd_ctx* ctx, const int32_t* d_ids, int32_t rows, const uint16_t* d_dx, float scale, void* d_dW,
                       int32_t grad_type, int32_t accumulate, void* d_workspace, size_t workspace_bytes);

/* Softmax cross entropy of hidden rows over the allowed ids, without forming the logits in memory:
 *   z = h W^T / tau (allowed rows of W),  lse = log sum exp(z),  loss = lse - z[target].
 * top_k, top_p and the decode options do not enter; cfg_lambda must be 0 (SCD_EUNSUPPORTED otherwise).
 *   d_h bf16 [rows, d];  d_targets int32 [rows], OFFSETS into the allowed ids; a negative one leaves the row out (loss 0,
 * no gradient, whatever the row holds), one of n or more is not an allowed id (loss +inf, gradient of the normaliser alone);
 *   d_loss, d_lse fp32 [rows], written.  rows * allowed ids up to 2^38, allowed ids up to 2^30, d up to 2^21, tau
 * such that log2(e) / tau is finite (SCD_EUNSUPPORTED beyond). */
size_t scd_cross_entropy_workspace_bytes(const scd_config* cfg, int32_t rows);
int scd_cross_entropy(scd_ctx* ctx, const uint16_t* d_h, const uint16_t* d_W, const int32_t* d_targets, int32_t rows,
                      float* d_loss, float* d_lse, void* d_workspace, size_t workspace_bytes);

/* Its gradient.  d_lse from scd_cross_entropy on the same arguments; d_weight fp32 [rows], the gradient of the result with
 * respect to each row's loss, NULL = 1 (1 / rows for a mean).  The logits are made again, a piece of the vocabulary at a
 * time.  d_dh bf16 [rows, d] and d_dW [V, d] of type grad_type, of which the allowed rows alone are written, or added to
 * with accumulate = 1 (in 32 bits, rounded once); either may be NULL (not wanted).  The same call gives the same bits.
 *   The gradient's products add up in fp32, on operands of 16 bits: the gradients of the logits have 11 bits, down to 2^-28 (of the largest
 * weight for d_dW; steps of 2^-38 below, so that what is smaller than 2^-39 counts as 0).  For an fp32 d_dW alone they have 22 bits and end
 * at 2^-50.  W and the rows of h stand under one power of two each: elements below 2^-31 of the largest finite one (of all
 * allowed rows of W, or of all rows of h that are not left out) lose bits, and those below 2^-39 of it count as 0. */
size_t scd_cross_entropy_backward_workspace_bytes(const scd_config* cfg, int32_t rows, int32_t grad_type);
int scd_cross_entropy_backward(scd_ctx* ctx, const uint16_t* d_h, const uint16_t* d_W, const int32_t* d_targets, int32_t rows,
                               const float* d_lse, const float* d_weight, uint16_t* d_dh, void* d_dW, int32_t grad_type,
                               int32_t accumulate, void* d_workspace, size_t workspace_bytes);

/* For reports: the kernels of both calls' matrix products for `rows` rows, gemm_kernel<rows of a tile, columns of a tile, use>, and how many
 * ids the gradient takes at a time (the last piece may have fewer), NUL-terminated, in host_buf[0..cap): "gemm_kernel<.., kLoss>; pieces of
 * N: gemm_kernel<.., kGradient>, gemm_kernel<.., kRows> in K parts, gemm_kernel<.., kTable or kTableTwoTerms>" (255 characters
 * hold it).  SCD_OK, or SCD_EINVAL / SCD_EUNSUPPORTED as the calls.  Host-only call. */
int scd_cross_entropy_kernel_names(scd_ctx* ctx, int32_t rows, int32_t grad_type, char* host_buf, size_t cap);

/* ---- around the model's last norm, and what it leaves of the gradients ---------------------------
 * The norm that the hidden rows pass before the LM head, the LM head over 8-bit rows and weights, and the norm of the gradients that
 * these calls and the caller's own leave.  Pointers to rows, gains and tables are 16-byte aligned, float arrays and scales 4-byte.  Of the
 * configuration the norms use d (in 8 .. 2^24), the calls on gradients nothing. */

/* Type of a residual stream, a gain, a tensor. */
typedef enum scd_type {
  SCD_BF16 = 0,
  SCD_F32 = 1
} scd_type;

/* Root-mean-square norm with the residual's addition, rows of d:
 *   s = x + r,  inv = 1 / sqrt(mean(s^2) + eps),  y = s * inv * gain        (in fp32; each result rounded once)
 *   d_x bf16 [rows, d];  d_residual [rows, d] of type stream_type, or NULL (s = x);  d_gain [d] of type gain_type;  eps > 0;
 *   d_y bf16 [rows, d];  d_sum [rows, d] of type stream_type: s (NULL: not wanted, and without a residual);  d_inv fp32 [rows], for
 * the gradient (NULL: not wanted).  d_sum may be d_residual, d_y may be d_x; nothing else may overlap.  rows = 0 is allowed (arrays of no
 * elements may then be NULL), up to 2^25. */
int scd_norm(scd_ctx* ctx, const uint16_t* d_x, const void* d_residual, int32_t stream_type, const void* d_gain, int32_t gain_type, float eps,
             int32_t rows, uint16_t* d_y, void* d_sum, float* d_inv);

/* The same with y in 8 bits: d_codes e4m3 (4 exponent and 3 mantissa bits, no infinities) [rows, d] and d_scales fp32 [rows, ceil(d / 128)],
 *   scale = max |y| / 448 over 128 of a row,  code = y / scale (the quotient in fp32), rounded to the nearest, to the even one of two.
 * 128 values of which none reaches 448 * 2^-126 count as zeros (scale and codes 0); with an infinity among them the scale is infinite,
 * with a NaN a NaN.  (scd_lm_head_fp8 reads rows of a multiple of 16 columns, this call writes any that the configuration allows.) */
int scd_norm_fp8(scd_ctx* ctx, const uint16_t* d_x, const void* d_residual, int32_t stream_type, const void* d_gain, int32_t gain_type, float eps,
                 int32_t rows, uint8_t* d_codes, float* d_scales, void* d_sum, float* d_inv);

/* Gradient of both (of y as it is before its rounding) with respect to the rows and the gains:
 *   dx = inv * (a - s * inv^2 * mean(a * s)) + ds,  a = gain * dy;   dgain = sum over the rows of dy * s * inv
 * Behind a bf16 stream s is the rounded sum and inv that of the sum before: dx's second term and the terms of dgain then carry the stream's
 * rounding (up to 2^-8 of |s|), whatever types they are stored in; an fp32 stream keeps it out.
 *   d_sum (s: without a residual x, with stream_type SCD_BF16) and d_inv as scd_norm left them;  d_dy bf16 [rows, d];  d_dsum [rows, d] of
 * type grad_type: the gradient that reaches s from elsewhere, or NULL;  d_dx [rows, d] of type grad_type: the gradient of x and of the
 * residual alike; it may be d_dsum, or d_dy if it is bf16;  d_dgain [d] of type gain_grad_type, or NULL, added to with accumulate = 1 (in 32 bits,
 * rounded once).  The same call gives the same bits.  The workspace is the caller's, 256-byte aligned, of the size that the query gives
 * (0 for bad arguments); nothing in it outlives the call, and calls that may overlap in time must not share one. */
size_t scd_norm_backward_workspace_bytes(const scd_config* cfg, int32_t rows);
int scd_norm_backward(scd_ctx* ctx, const void* d_sum, int32_t stream_type, const void* d_gain, int32_t gain_type, const float* d_inv,
                      const uint16_t* d_dy, const void* d_dsum, int32_t grad_type, int32_t rows, void* d_dx, void* d_dgain,
                      int32_t gain_grad_type, int32_t accumulate, void* d_workspace, size_t workspace_bytes);

/* The LM head over e4m3 rows and weights with a scale for each block of 128:
 *   logit[m, v] = sum over the blocks b of k of  sh[m, b] * sw[v / 128, b] * sum over k in b of h[m, k] * W[v, k]
 *   d_h e4m3 [B, C, L, d] and d_h_scales fp32 [B, C, L, G], as scd_norm_fp8 writes them;  d_W e4m3 [V, d] and d_W_scales fp32
 * [ceil(V / 128), G], G = ceil(d / 128), as scd_quantize_fp8 writes them (blocks of 128 ids from id 0 on, the last block of a row or of the
 * table may be smaller).  Only rows [v_lo, v_hi) of W are read.  Products are exact and added up in fp32.  d a multiple of 16 up to 2^20, at most
 * 2^30 allowed ids (SCD_EUNSUPPORTED beyond). */
int scd_quantize_fp8(scd_ctx* ctx, const uint16_t* d_W, uint8_t* d_codes, float* d_scales);
int scd_lm_head_fp8(scd_ctx* ctx, const uint8_t* d_h, const float* d_h_scales, const uint8_t* d_W, const float* d_W_scales, float* d_z);
int scd_step_fp8(scd_ctx* ctx, const uint8_t* d_h, const float* d_h_scales, const uint8_t* d_W, const float* d_W_scales, void* d_state);

/* scd_lm_head_kernel_name of these two, which launch the same kernel: lm_head_fp8_kernel<Fp8Cfg<1 + CFG, blocks of 32 window rows, columns,
 * wavefronts along the columns, along the rows, stages, parts of k, W past the caches>, groups of 128 ids may end among a wavefront's columns> (127 characters
 * hold it). */
int scd_lm_head_fp8_kernel_name(scd_ctx* ctx, char* host_buf, size_t cap);

/* Norm of many gradients together, sqrt(sum of all elements' squares) (added up in 64 bits, stored as fp32), and clipping,
 *   out = g * min(1, max_norm / norm): the factor is rounded to fp32, the product to fp32 and from there to the output's type.
 * Arrays of `count` tensors in HOST memory, read during the call; a tensor's d is aligned to its elements, n >= 0 (up to 2^40; d may be NULL
 * for n = 0), type a scd_type.  d_norm fp32, one element: written by scd_gradient_norm, read by scd_clip_gradients, which takes any norm that
 * the caller puts there (of several machines' gradients together, say).  out[i] has the elements of grads[i], in either type; it may be
 * the same tensor (of the same type: left alone where norm <= max_norm); otherwise nothing may overlap.  A norm that is infinite leaves
 * zeros (NaN where the gradient is infinite), one that is NaN makes all NaN.  max_norm >= 0; infinite: finite norms leave the gradients as they are.  Workspace as in scd_norm_backward. */
typedef struct scd_tensor {
  void* d;
  int64_t n;
  int32_t type;
} scd_tensor;
size_t scd_gradient_norm_workspace_bytes(const scd_tensor* grads, int32_t count);
int scd_gradient_norm(scd_ctx* ctx, const scd_tensor* grads, int32_t count, float* d_norm, void* d_workspace, size_t workspace_bytes);
int scd_clip_gradients(scd_ctx* ctx, const scd_tensor* grads, const scd_tensor* out, int32_t count, float max_norm, const float* d_norm);

/* Synchronises the stream and reports: host_flags[0] = numeric-fault bits,
 * host_flags[1] = 1 if every sequence has emitted N tokens, host_flags[2] =
 * largest t_b, host_flags[3] = 0.  Returns SCD_ENUMERIC if a fault bit is set. */
int scd_status(scd_ctx* ctx, void* d_state, int32_t host_flags[4]);

const char* scd_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SCD_H */
