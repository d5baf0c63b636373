/*
 * rpd.h -- C ABI of the MI355X (gfx950) commit step of Reliable Parallel
 * Decoding (RPD).
 *
 * One call performs one decoding iteration's commit step (Sections 2.2, 3.1
 * and 3.2 of the paper; Appendix A.6 "Layerwise projection"): every masked
 * canvas position is projected through the unembedding at each of the final
 * K layers, each layer's full-vocabulary softmax is reduced to its argmax,
 * top probability and entropy (Eq. 1), layerwise stability is scored
 * (persistence Eq. 2, confidence drop Eq. 3, stability Eq. 4), candidates
 * are formed (Eq. 5), and the candidates whose cumulative upstream entropy
 * stays within the budget are committed, with the progress fallback
 * (Section 3.2).
 *
 * Conventions for every entry point:
 *  - Pointers marked "device" are HIP device (or managed) memory on the
 *    current device; "host" pointers are read during the call only.
 *  - The caller owns every buffer. The library allocates no device memory (a
 *    call that waits for a count has it stored in one page of pinned host
 *    memory, allocated by the process's first such call; rpd_score_commit_noalloc
 *    never uses it),
 *    keeps no pointer after it returns, and never writes its inputs.
 *  - Work is enqueued asynchronously on `stream` (a hipStream_t; NULL = the
 *    default stream). Results are valid once the stream has completed.
 *  - Arrays are dense and row-major in the shapes given. The final layer of
 *    the window is layer K-1.
 *  - Errors: every argument is validated on the host before anything is
 *    enqueued, so a status other than RPD_OK and RPD_ERR_HIP means nothing
 *    was enqueued and the outputs are untouched. RPD_ERR_HIP reports a HIP
 *    runtime call or launch that failed part-way: the work enqueued before
 *    it stays enqueued and may have written the outputs and the workspace
 *    in part, so the outputs are then undefined (and the stream may be in
 *    an error state, as HIP reports it). rpd_last_error() describes the
 *    failure (thread-local). No C++ exception crosses this interface.
 *  - Calls on distinct streams with distinct workspaces may overlap.
 */
#ifndef RPD_H
#define RPD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RPD_ABI_VERSION 3

/* element types: `hidden` and `w_u` of the commit step are RPD_DTYPE_BF16 or
 * RPD_DTYPE_F32 (both the same); RPD_DTYPE_F16 exists in the operators that name it */
enum { RPD_DTYPE_BF16 = 0, RPD_DTYPE_F32 = 1, RPD_DTYPE_F16 = 2 };

typedef enum rpd_status {
  RPD_OK = 0,
  RPD_ERR_NULL_POINTER = 1,        /* a required pointer is NULL */
  RPD_ERR_BAD_SHAPE = 2,           /* a dimension is out of range */
  RPD_ERR_BAD_PARAM = 3,           /* a hyperparameter is out of range or NaN */
  RPD_ERR_WORKSPACE_TOO_SMALL = 4, /* workspace_bytes < the required size */
  RPD_ERR_UNSUPPORTED = 5,         /* dtype / alignment / size not supported */
  RPD_ERR_HIP = 6                  /* a HIP runtime call or launch failed */
} rpd_status;

/* bits of rpd_params.flags */
#define RPD_PARAM_LAZY 1u     /* lazy layerwise projection (see rpd_params) */
#define RPD_PARAM_LAZY_ALL 2u /* with RPD_PARAM_LAZY: every masked position walks its layers */

/* per-position flag bits written to rpd_outputs.flags */
#define RPD_FLAG_CANDIDATE 1u  /* in the candidate set C_t (Eq. 5) */
#define RPD_FLAG_HIGH_CONF 2u  /* admitted because c_i >= theta_h */
#define RPD_FLAG_STABLE    4u  /* admitted through the stability test */
#define RPD_FLAG_COMMITTED 8u  /* in the commitment set A_t */
#define RPD_FLAG_FALLBACK  16u /* committed by the progress fallback */

/* bits of the optional device status word */
#define RPD_DEVICE_STATUS_MASKED_OVERFLOW 1 /* more masked positions than max_masked */

/*
 * The problem of one call (Section 3: the masked positions M_t of the canvas
 * and the hidden states of the final layers of one forward pass).
 *   K           number of final layers supplied, 1 <= K <= 64 (the paper
 *               projects layers l0..L, Appendix A.6; here the K supplied)
 *   B, L        sequences and canvas positions per sequence (B >= 1, L >= 1,
 *               B*L <= 2^24)
 *   d, V        hidden size and vocabulary size (1 <= d <= 2^20, 1 <= V < 2^31);
 *               bf16 requires d % 8 == 0
 *   dtype       RPD_DTYPE_BF16 or RPD_DTYPE_F32
 *   hidden      device [K][B][L][d]; hidden states already passed through the
 *               model's final normalisation; rows of unmasked positions are
 *               never read (they may hold anything, NaN included)
 *   w_u         device [V][d]; the unembedding (output head), d contiguous;
 *               16-byte aligned
 *   mask        device [B][L] uint8; nonzero = masked (in M_t)
 *   norm_weight optional device [d], same type as hidden: the gain g of the
 *               model's final normalization (RMS normalization). NULL: every
 *               supplied state is already normalized and is projected as is.
 *               Otherwise the states of layers 0 .. K-2 (and of layer K-1
 *               too if norm_final != 0) are first replaced by
 *               g * x / sqrt(mean(x^2) + norm_eps), evaluated in float64 and
 *               rounded (to nearest, ties to even) to the input type, as the
 *               model's normalization hands the output head (Appendix A.2
 *               "Intermediate-layer readout", A.6 "Layerwise projection":
 *               the final layer uses the native, already normalized state).
 *               16-byte aligned for bf16.
 *   norm_eps    >= 0, finite; the normalization's epsilon (unused without g)
 *   norm_final  0: layer K-1 is the model's native normalized state (the
 *               paper); 1: normalize it like the others
 *   max_masked  an upper bound on the number of masked positions summed over
 *               the batch, or -1. With -1 the call waits once for the exact
 *               count (and so for the work on the stream before it): it polls
 *               pinned memory that the kernel with the count writes, for up to
 *               2 ms, keeping its CPU busy, then synchronises the stream (and
 *               at once if it cannot use that memory). RPD_OK does not imply
 *               that the stream was synchronised or that earlier work on it
 *               succeeded. If the bound is exceeded, only the first
 *               max_masked masked positions (batch-major, canvas order) are
 *               scored, the results for the rest are undefined, and
 *               RPD_DEVICE_STATUS_MASKED_OVERFLOW is raised in the optional
 *               status word.
 */
typedef struct rpd_problem {
  int32_t K, B, L, d, V;
  int32_t dtype;
  const void* hidden;
  const void* w_u;
  const uint8_t* mask;
  int32_t max_masked;
  const void* norm_weight;
  float norm_eps;
  int32_t norm_final;
} rpd_problem;

/*
 * Hyperparameters (Table 4, Appendix A.6; LLaDA: theta_s 3.5, w 15; Dream:
 * theta_s 2.5, w 20; both theta_h 0.9, theta_c 0.6, K_max 6, beta 4 nats,
 * W 32). Requirements: 0 <= theta_c <= theta_h, w >= 0, k_max >= 1,
 * beta >= 0 (may be +inf), window >= 1, flags only RPD_PARAM_LAZY and
 * RPD_PARAM_LAZY_ALL (the latter only with the former), block >= 0; no NaN.
 *
 * block selects the commitment rule. 0: full RPD (Section 3.2), the
 * cumulative-entropy budget beta over the whole canvas with the fallback
 * over the first `window` masked positions. > 0: RPD-block (Section 3.2
 * "Variants", Appendix A.6 "RPD-block"; the paper uses 32): the canvas of
 * each sequence is cut into runs of `block` positions starting at 0, the
 * active block is the first run holding a masked position, every candidate
 * (Eq. 5) inside it is committed with no budget (beta and window are then
 * unused), and without one its most confident masked position is. The
 * reported upstream entropy is then the entropy over earlier masked
 * positions outside the commitment set.
 *
 * RPD_PARAM_LAZY in flags: lazy layerwise projection (Appendix A.6
 * "Layerwise projection": a position's intermediate layers are projected
 * from the final one down, no further than its agreement suffix needs). The
 * final layer of every masked position is projected first; then the
 * positions that walk project layer K-2, K-3, ..., each stopping after its
 * first disagreeing layer. With RPD_PARAM_LAZY_ALL as well, every masked
 * position with a finite final confidence walks (the procedure as the paper
 * states it), and persistence, drop and stability equal the eager
 * projection's everywhere. Without it only the positions with
 * theta_c <= c < theta_h walk: the only ones whose candidacy the stability
 * test decides (Eq. 5), a further saving of this library beyond the
 * paper's procedure that leaves every decision unchanged; outside that band
 * persistence, drop and stability are then not evaluated (persistence -1,
 * drop and stability NaN). Either way tokens, candidacy and commitment are
 * those of the eager projection, and the per-layer outputs of layers never
 * projected hold -1 / NaN. One projection pass takes several of a position's
 * next layers while its rows are few (each pass streams W_U again, and up to a
 * few hundred rows that is what it costs), and at least 1, 2, 4, .. of them; a
 * small call projects every layer in one pass, where that costs little more
 * than the least that walking can. The layers below a position's first
 * disagreement are then read and projected too, and reported as never
 * projected. Whether positions stop at once or agree on down to the last layer
 * is not known beforehand: a call whose positions all stop at once can take
 * longer than it would with one layer a pass, one whose positions agree takes
 * less (d = 4096, V = 126464, K = 4, 125 positions that all walk: 430 us, with one
 * layer a pass 372 to 710). Lazy projection pays where the projection is
 * compute-bound (many masked positions). While max_masked is at most 256, every
 * pass reads its count on the device and is launched once per size class the
 * row count may fall in (<= 64, <= 128, <= 192, <= 256, up to the bound; in fp32
 * 32, 64, 96, 128), all but one exiting at once. Above, the host waits for the
 * count of the previous pass, as for max_masked = -1, and plans the pass for
 * it. So with max_masked <= 256 the call never waits.
 *
 * logit_scale multiplies every logit before the softmax statistics (an
 * inverse temperature). The paper reads probabilities before any
 * temperature (Appendix A.2), i.e. 1; 0 is read as 1; otherwise it must be
 * finite and > 0. rpd_gate_commit ignores it.
 */
typedef struct rpd_params {
  float theta_h;   /* high-confidence threshold (bypasses stability), Eq. 5 */
  float theta_c;   /* minimum confidence for stability admission, Eq. 5 */
  float theta_s;   /* stability threshold, Eq. 5 */
  float w;         /* weight of the confidence-drop penalty, Eq. 4 */
  int32_t k_max;   /* cap on persistence, Eq. 4 */
  float beta;      /* cumulative entropy budget in nats, Section 3.2 */
  int32_t window;  /* fallback window W, Section 3.2 */
  uint32_t flags;  /* RPD_PARAM_* bits */
  int32_t block;   /* 0: full RPD; > 0: RPD-block with blocks of this many positions */
  float logit_scale; /* inverse temperature of the scoring softmax; 0 or 1: none */
} rpd_params;

/*
 * Outputs, all device memory, shape [B][L] unless noted. Unmasked positions
 * receive: commit 0, token -1, persistence 0, flags 0 and 0.0f elsewhere.
 *   commit            1 if the position is in A_t (Section 3.2)
 *   token             y_i, the final-layer argmax, for every masked
 *                     position, committed or not. Ties go to the lowest
 *                     index: logits equal in exact arithmetic are found
 *                     exactly while |logit_scale| * sum_k |W_U[y,k] x_k|
 *                     <= 256 (|max logit| + 1) at d = 4096 (the bound
 *                     scales with 1/(d+1)); a positive gap below the fp32
 *                     accumulation error 4 (d+1) 2^-24 sum_k |W_U[y,k] x_k|
 *                     may go either way
 *   entropy           H(p_i^(K-1)) in nats (Eq. 1)
 *   confidence        c_i = p_i^(K-1)(y_i)
 *   persistence       K_i (Eq. 2), counted within the K supplied layers
 *   drop              r_i (Eq. 3)
 *   stability         S_i = min(K_i, k_max) - w r_i (Eq. 4)
 *   flags             RPD_FLAG_* bits
 *   upstream_entropy  E_i: entropy summed over earlier masked positions of
 *                     the sequence that are not in A_t (Section 3.2),
 *                     evaluated before the fallback
 *   n_commit          [B] number of committed positions per sequence
 * Optional (NULL to skip):
 *   layer_argmax, layer_conf, layer_entropy   [K][B][L] per-layer argmax,
 *                     top probability and entropy at masked positions
 *                     (unmasked entries are left untouched)
 *   status            one int32 of RPD_DEVICE_STATUS_* bits, overwritten
 */
typedef struct rpd_outputs {
  uint8_t* commit;
  int32_t* token;
  float* entropy;
  float* confidence;
  int32_t* persistence;
  float* drop;
  float* stability;
  uint8_t* flags;
  float* upstream_entropy;
  int32_t* n_commit;
  int32_t* layer_argmax;
  float* layer_conf;
  float* layer_entropy;
  int32_t* status;
} rpd_outputs;

/* Device workspace bytes that rpd_score_commit needs for problem `p`
 * (pointers in `p` are not read; norm_weight is only tested for NULL).
 * Returns 0 if the shape is invalid. */
size_t rpd_workspace_size(const rpd_problem* p);

/*
 * The whole commit step (Sections 2.2, 3.1, 3.2). `workspace` is device
 * memory of at least rpd_workspace_size(p) bytes, 256-byte aligned, used only
 * during the call's stream work; its prior contents do not matter.
 */
rpd_status rpd_score_commit(const rpd_problem* p, const rpd_params* q, const rpd_outputs* o,
                            void* workspace, size_t workspace_bytes, void* stream);

/*
 * rpd_score_commit, recording caller-created HIP events (hipEvent_t, cast to
 * void*) on `stream` at its stage boundaries, for callers that time the
 * stages: events[0] before the masked-position compaction, [1] before the
 * projection (logit lens + fused softmax statistics; with a norm_weight, the
 * final normalization of the rows comes first, after [1]), [2] after it, [3]
 * after the cross-tile reduction and stability scoring, [4] after the
 * commitment scan. Only the first n_events (0..5) are used;
 * NULL entries are skipped (with RPD_PARAM_LAZY, [1] precedes the first
 * pass and [2] follows the last). Everything else is exactly
 * rpd_score_commit.
 */
rpd_status rpd_score_commit_timed(const rpd_problem* p, const rpd_params* q, const rpd_outputs* o,
                                  void* workspace, size_t workspace_bytes, void* stream,
                                  void* const* events, int32_t n_events);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * rpd_score_commit without a workspace argument. The workspace is a
 * library-owned static device array of RPD_NOALLOC_SCRATCH_BYTES on each
 * GPU the library runs on, held until the process ends; the call allocates
 * nothing (no hipMalloc, no allocating library routine). Problems whose
 * rpd_workspace_size exceeds RPD_NOALLOC_SCRATCH_BYTES are rejected with
 * RPD_ERR_WORKSPACE_TOO_SMALL before anything is enqueued (at the LLaDA-8B
 * vocabulary, up to about 8,400 projected rows: K * max_masked). Every call
 * on one GPU shares that GPU's array: calls that overlap on one GPU (other
 * streams, other threads) race and must be serialised by the caller. The
 * array's prior contents never matter (every kernel writes what it reads).
 * The first call on a device, with that device current, looks the array's
 * address up (RPD_ERR_HIP if that fails). Otherwise exactly
 * rpd_score_commit, including its validation and error reporting.
 */
#define RPD_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
rpd_status rpd_score_commit_noalloc(const rpd_problem* p, const rpd_params* q, const rpd_outputs* o,
                                    void* stream);

/*
 * Scoring and commitment from per-layer statistics that the caller already
 * has (Eq. 2-5 and Section 3.2), for callers whose logits come from
 * elsewhere. layer_argmax / layer_conf / layer_entropy are device [K][B][L]
 * in the layout rpd_score_commit writes them (only masked positions are
 * read; only the final layer's entropy is used). Inside the agreement suffix
 * the probability of the final token equals that layer's top probability,
 * which is how Eq. 3 is evaluated. Writes the required outputs of `o`; the
 * optional per-layer pointers and status of `o` are ignored. Needs no
 * workspace.
 */
rpd_status rpd_gate_commit(int32_t K, int32_t B, int32_t L, const uint8_t* mask,
                           const int32_t* layer_argmax, const float* layer_conf,
                           const float* layer_entropy, const rpd_params* q,
                           const rpd_outputs* o, void* stream);

/* projection kernel variants (values of rpd_projection_variant) */
enum {
  RPD_PROJ_BF16_S32 = 0,  /* bf16, at most 32 projected rows: W_U streamed once from HBM */
  RPD_PROJ_BF16_S64 = 1,  /* bf16, 33..64 rows, same kernel family */
  /* 2: no longer planned (a 65..128-row streaming form, replaced by 7) */
  RPD_PROJ_F32 = 3,       /* fp32 inputs, any row count */
  RPD_PROJ_BF16_BIG = 4,  /* bf16, more than 128 rows: MFMA tiles of 256 x 256 */
  /* 5: no longer planned (a 129..192-row streaming form, replaced by 6) */
  RPD_PROJ_BF16_BIG192 = 6, /* bf16, more than 128 rows where 256 x 192 tiles pad the rows less (129..192 rows
                               always; above, whenever ceil(R/192)*192 < ceil(R/256)*256) */
  RPD_PROJ_BF16_BIG128 = 7  /* bf16, 65..128 rows: one MFMA tile of 256 x 128 per vocabulary tile */
};

/*
 * The projection kernel variant (RPD_PROJ_*) that rpd_score_commit launches
 * for problem `p` (pointers in `p` are not read), where the projected rows
 * are K * max_masked; with max_masked < 0 this assumes every position is
 * masked (the call itself plans for the count it reads back). Returns -1 if
 * the shape or dtype is invalid. For instrumentation and tests.
 */
int32_t rpd_projection_variant(const rpd_problem* p);

/*
 * The end of an iteration (Section 3.2: the positions of A_t are filled with
 * their predictions y_i; every other position keeps its mask): for every
 * masked position with commit != 0, canvas = token and mask = 0.
 *   mask     [B][L] uint8, updated in place
 *   canvas   [B][L] int32, written only at the positions committed here
 *   commit, token  [B][L] uint8 / int32 as rpd_score_commit writes them
 *   progress optional int32 [1 + progress_len], zeroed by the caller before
 *            the first call: progress[0] counts the calls made with it and
 *            progress[1 + t] receives the number of positions still masked
 *            after call t (for t < progress_len), so a loop of iterations
 *            learns when the canvas is full without a read-back per
 *            iteration. With it the update runs in one workgroup (meant for
 *            canvases of up to some tens of thousands of positions); without
 *            it, over the whole GPU.
 *   step     optional int32 [B][L] (needs progress): at each position
 *            committed here, the call index progress[0] had on entry.
 * All pointers are device memory owned by the caller. NULL mask, canvas,
 * commit or token, or step without progress, -> RPD_ERR_NULL_POINTER; B or L
 * < 1 or B*L > 2^24 -> RPD_ERR_BAD_SHAPE; progress_len < 0 ->
 * RPD_ERR_BAD_PARAM. Enqueued on `stream`; it allocates nothing and never
 * synchronises, so a loop body of rpd_score_commit (max_masked >= 0, and at
 * most 256 with lazy projection) followed by this call can be captured in a
 * HIP graph.
 */
rpd_status rpd_apply_commit(int32_t B, int32_t L, uint8_t* mask, int32_t* canvas, const uint8_t* commit,
                            const int32_t* token, int32_t* progress, int32_t progress_len, int32_t* step,
                            void* stream);

/* ------------------------------------------------------------------------
 * Operators around the commit step: an output head with 4-bit weights, the
 * verification of drafted tokens, and the distillation of a drafter. The
 * conventions above hold for them too. Random numbers are inputs. Element
 * types are RPD_DTYPE_BF16, RPD_DTYPE_F16 and RPD_DTYPE_F32 as each entry
 * says; strides are in elements, the last dimension is contiguous, and rows
 * need no alignment beyond their element's. NaN and infinities follow IEEE
 * arithmetic and stay in the row (sequence) that holds them. Finite logits may
 * be of any size, at any scale: a mask of the type's lowest value is probability
 * 0, and a row of nothing else is flat (two logits whose difference exceeds
 * float32's range count as infinitely far apart).
 */

/*
 * An output head with 4-bit weights and group scales:
 *   W[v][k] = scales[v][k / group] * (code[v][k] - zeros[v][k / group])
 *   V, d        1 <= V < 2^28, 8 <= d <= 2^20, d % 8 == 0, V * d <= 2^36
 *   group       32, 64 or 128 columns that share a scale; the last group of a
 *               row may be shorter
 *   dtype       RPD_DTYPE_BF16 or RPD_DTYPE_F16: type of the scales and of
 *               the rows that are projected
 *   has_zeros   0: every zero point is 8; 1: zero points 0..15 are given
 * The codes are laid out once, by rpd_quant_pack, for the matrix cores.
 */
typedef struct rpd_quant_head {
  int32_t V, d, group, dtype, has_zeros;
} rpd_quant_head;

/* Bytes of the packed head (about V * d / 2 plus 2 or 3 per group); 0 if `h`
 * is out of range. */
size_t rpd_quant_packed_size(const rpd_quant_head* h);

/*
 * Lays a head out into `packed` (device, rpd_quant_packed_size bytes, 256-byte
 * aligned), which rpd_quant_project then reads in place of the inputs.
 *   codes   device [V][d/2] uint8; byte j of a row holds column 2j in its low
 *           and column 2j+1 in its high nibble
 *   scales  device [V][ceil(d / group)] of type dtype
 *   zeros   device [V][ceil(d / group)] uint8 (low nibble), NULL without has_zeros
 */
rpd_status rpd_quant_pack(const rpd_quant_head* h, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                          void* packed, size_t packed_bytes, void* stream);

/* Workspace bytes that rpd_quant_project needs for M rows (0 for the logits of
 * up to 16 rows; 0 too if h or M is out of range). */
size_t rpd_quant_workspace_size(const rpd_quant_head* h, int32_t M, int32_t statistics);

/*
 * M rows through the head: logits y = W x, or the softmax statistics of
 * logit_scale * y as rpd_gate_commit takes them (the logits then never reach
 * memory). Exactly one of `logits` and the three statistics is given. Codes
 * are exact operands and sums are float32; x is exact up to 2^-39 of the
 * row's largest finite magnitude. Equal rows of the head give equal logits;
 * of equal logits the lowest index is the argmax.
 *   M          0 <= M <= 2^20 (0: nothing is done)
 *   x          device [M][d] of type dtype, rows x_stride >= d apart
 *   logits     device [M][V], rows logits_stride >= V apart, of type
 *              logits_dtype: dtype or RPD_DTYPE_F32; or NULL
 *   argmax, confidence, entropy   device [M] int32 / float / float (top
 *              probability, nats); all given or all NULL. A row of NaN has
 *              argmax -1 and the others NaN
 *   logit_scale  finite and > 0, or 0 for 1; the statistics only
 *   workspace  rpd_quant_workspace_size bytes, 256-byte aligned (may be NULL
 *              where that is 0); its prior contents do not matter
 * The codes are streamed once for up to 32 rows (16 above d = 4096); the
 * workgroups of further rows read them at the same time, through the caches.
 */
rpd_status rpd_quant_project(const rpd_quant_head* h, const void* packed, int32_t M, const void* x, int64_t x_stride,
                             void* logits, int64_t logits_stride, int32_t logits_dtype, int32_t* argmax,
                             float* confidence, float* entropy, float logit_scale, void* workspace,
                             size_t workspace_bytes, void* stream);

#define RPD_VERIFY_GREEDY 1u /* accept a drafted token iff it is the target's argmax */

/*
 * Verification of drafted tokens (speculative decoding; a draft may come from
 * parallel commitments). With p_t = softmax(target_scale * target[b][t]) and
 * q_t = softmax(draft_scale * draft[b][t]), token x_t = token[b][t] of the
 * len[b] drafted ones is accepted with probability
 *   accept[b][t] = min(1, p_t(x_t) / q_t(x_t)),
 * that is while u[b][t] < accept[b][t]; the first that is not ends it. After n
 * accepted tokens one more is drawn: from max(0, p_n - q_n) where x_n was
 * turned down (from p_n if that is empty), from p_n where the draft ended:
 * the lowest v whose running sum exceeds r[b] times the whole. Without draft
 * logits (a draft that names one token with certainty) q_t is 1 at x_t.
 *   B, T, V    B >= 1, T >= 0 drafted tokens at most, 1 <= V <= 2^28,
 *              B * (T + 1) <= 2^20; together with V bounded by what one launch
 *              holds (logits of 100 GB are far below that)
 *   dtype      of the logits: RPD_DTYPE_BF16, _F16 or _F32
 *   target     device [B][T+1][V]; row t is the target's after the first t
 *              drafted tokens. Rows behind the draft (t > len) are not read
 *   draft      device [B][T][V] or NULL; rows t >= len are not read
 *   token      device [B][T]; one outside 0..V-1 is never accepted
 *   len        device [B], read as within 0..T, or NULL: T everywhere
 *   u, r       device [B][T] and [B] float32 in [0, 1)
 *   target_scale, draft_scale   inverse temperatures, finite and > 0, or 0 for 1
 *   flags      RPD_VERIFY_GREEDY: x_t is accepted iff it is the target's
 *              argmax (lowest index of equals, NaN never), and the further
 *              token is an argmax; draft, u, r and the scales are not used
 *   out_token  device [B][T+1] int32: the accepted tokens, the further one, -1
 *              behind it. The further token is -1 too where p_n has no
 *              distribution (NaN, +inf or nothing but -inf in the row)
 *   n_accept   device [B] int32
 *   accept     device [B][T] float32 (greedy: 1 or 0); 0 for t >= len; NaN
 *              where p_t or q_t has no distribution or both are 0 at x_t
 * Acceptance probabilities carry sums of float32 accuracy, or of float64 where
 * the rows are few; the drawn token's sums are float64. Outputs must not
 * overlap the inputs.
 */
typedef struct rpd_verify {
  int32_t B, T, V, dtype;
  const void* target;
  int64_t target_batch_stride, target_row_stride;
  const void* draft;
  int64_t draft_batch_stride, draft_row_stride;
  const int32_t* token;
  const int32_t* len;
  const float* u;
  const float* r;
  float target_scale, draft_scale;
  uint32_t flags;
  int32_t* out_token;
  int32_t* n_accept;
  float* accept;
} rpd_verify;

/* Workspace bytes of rpd_verify_draft (pointers only tested for NULL); 0 if
 * the shape is out of range. */
size_t rpd_verify_workspace_size(const rpd_verify* p);
rpd_status rpd_verify_draft(const rpd_verify* p, void* workspace, size_t workspace_bytes, void* stream);

#define RPD_DISTILL_MAX_K 256 /* longest list of a teacher's tokens */
#define RPD_DISTILL_STATE 8   /* floats kept per row between the loss and the gradient */

/*
 * Distillation from a teacher's top logits. For row n of the student's
 * logits, q = softmax(logit_scale * logits[n]); the teacher's list gives
 * p_j for its tokens: the softmax of logit_scale * teacher[n] over the list,
 * or, with teacher_lse, e^(logit_scale * teacher[n][j] - teacher_lse[n]), the
 * rest p_T = max(0, 1 - sum p_j) then being one entry for all tokens outside
 * the list (student's mass q_T); p_T is 0 where the list holds every token.
 *   loss[n] = weight[n] * (sum_j p_j ln(p_j / q_j) + p_T ln(p_T / q_T))
 *   grad[n] = weight[n] * grad_loss[n] * d loss_n / d logits[n]
 * Rows are independent (the masked positions of a canvas, say).
 *   N, V, k    0 <= N < 2^24 (0: nothing is done), 1 <= V <= 2^20,
 *              1 <= k <= RPD_DISTILL_MAX_K; together bounded by what one launch
 *              holds (logits of 100 GB are far below that)
 *   dtype      of logits and grad: RPD_DTYPE_BF16, _F16 or _F32
 *   logits     device [N][V], rows logits_stride >= V apart
 *   id         device [N][k]; an entry outside 0..V-1 is no part of the list
 *              (shorter lists are padded with -1); a token listed twice has
 *              the sum of its entries
 *   teacher    device [N][k] of type teacher_dtype (any of the three); -inf is
 *              probability 0
 *   teacher_lse  device [N] float32 or NULL: log-sum-exp of logit_scale times
 *              all of the teacher's logits
 *   weight     device [N] float32 or NULL (1): a row of weight 0 is not read,
 *              its loss and gradient are 0 (unmasked positions)
 *   grad_loss  device [N] float32 or NULL (1): the upstream gradient
 *   loss       device [N] float32
 *   state      device [N][RPD_DISTILL_STATE] float32: what the gradient needs
 *              of the loss
 *   grad       device [N][V], rows grad_stride >= V apart; not the logits'
 *              memory (rows of the logits' stride may lie between theirs)
 * A list without entries (or of probability 0 without teacher_lse) has loss
 * and gradient 0. A list token of student probability 0 makes the loss inf, and
 * so does any p_T > 0, be it the rounding of teacher_lse, where the student
 * excludes every token outside the list (give no teacher_lse there).
 */
typedef struct rpd_distill {
  int32_t N, V, k, dtype, teacher_dtype;
  const void* logits;
  int64_t logits_stride;
  const int32_t* id;
  const void* teacher;
  const float* teacher_lse;
  const float* weight;
  const float* grad_loss;
  float logit_scale;
  float* loss;
  float* state;
  void* grad;
  int64_t grad_stride;
} rpd_distill;

/* Workspace bytes of the entries below; 0 if N, V or k is out of range or N is 0. */
size_t rpd_distill_workspace_size(const rpd_distill* p);
/* loss and state; and, where `grad` is given, the gradient in the same pass */
rpd_status rpd_distill_loss(const rpd_distill* p, void* workspace, size_t workspace_bytes, void* stream);
/* the gradient, from the state that rpd_distill_loss left for the same inputs
 * (`loss` is not used; needs no workspace) */
rpd_status rpd_distill_grad(const rpd_distill* p, void* stream);

/* ------------------------------------------------------------------------
 * Drafting with an 8-bit output head: quantization to blocks of 8-bit floating
 * point, the head in that form, and sampling from its logits. The conventions
 * above hold for them too.
 */

/*
 * Blocks of 8-bit floating point (e4m3: 4 significant bits, largest 448, no
 * infinities): a scale for each 128 columns of a row (block_rows 1), or for
 * each 128 x 128 of a matrix (block_rows 128); blocks at an end may be smaller.
 *   scale = the smallest power of two in 2^-126 .. 2^120 with which the block's
 *           largest finite magnitude is at most 448 (1 where that is 0)
 *   code  = e4m3(x / scale), to nearest, ties to even; NaN of what is not finite
 *   rows, d    0 <= rows <= 2^28 (0: nothing is done), 1 <= d <= 2^28; together
 *              bounded by what one launch holds
 *   dtype      of x: RPD_DTYPE_BF16, _F16 or _F32
 *   x          device [rows][d], rows x_stride >= d apart
 *   codes      device [rows][d] bytes, rows codes_stride >= d apart
 *   scales     device [rows or ceil(rows / 128)][ceil(d / 128)] float32
 * x, codes and scales must not overlap.
 */
rpd_status rpd_fp8_quantize(int32_t rows, int32_t d, int32_t dtype, const void* x, int64_t x_stride, int32_t block_rows,
                            uint8_t* codes, int64_t codes_stride, float* scales, void* stream);

/*
 * An output head in e4m3 with a scale for each block of 128 x 128 (of any
 * float32 value):
 *   W[v][k] = scales[v / 128][k / 128] * code[v][k]
 *   V, d       1 <= V, d <= 2^20, V * d <= 2^35
 *   codes      device [V][d] bytes, contiguous
 *   scales     device [ceil(V / 128)][ceil(d / 128)] float32
 *   transpose  0: packs W; 1: packs its transpose, a head of d rows and V
 *              columns (for the gradient of the rows: dx = dy W)
 *   packed     device, 256-byte aligned, rpd_fp8_packed_size bytes (of (d, V)
 *              with transpose), not over codes or scales
 * The codes are laid out once, for the matrix cores.
 */
size_t rpd_fp8_packed_size(int32_t V, int32_t d); /* 0 if out of range */
rpd_status rpd_fp8_pack(int32_t V, int32_t d, const uint8_t* codes, const float* scales, int32_t transpose, void* packed,
                        size_t packed_bytes, void* stream);

/* Workspace bytes of rpd_fp8_project for M rows (0 for the logits of up to 16
 * rows of a large head; 0 too if out of range). */
size_t rpd_fp8_workspace_size(int32_t V, int32_t d, int32_t M, int32_t statistics);

/*
 * M rows through a packed head of V rows and d columns. The rows are quantized
 * first, as rpd_fp8_quantize does with block_rows 1; with x^ what their codes
 * and scales stand for, logits y = W x^, or the softmax statistics of
 * logit_scale * y as rpd_gate_commit takes them (of a head of 131072 rows and
 * more, or of many x, the logits then never reach memory). Codes and x^ are
 * exact operands (magnitudes below 2^-126 may count as 0, and what rounds to
 * 2^128 is infinite), sums are float32. Equal rows of the head give equal
 * logits; of equal logits the lowest index is the argmax.
 *   M          0 <= M <= 2^20 (0: nothing is done), M * V <= 2^38, M * d <= 2^36
 *   x          device [M][d] of type x_dtype (bf16, fp16 or fp32), rows x_stride >= d apart
 *   logits     device [M][V] of type logits_dtype (any of the three), rows
 *              logits_stride >= V apart, not over x; or NULL
 *   argmax, confidence, entropy, logit_scale   as rpd_quant_project's
 *   workspace  rpd_fp8_workspace_size bytes, 256-byte aligned (may be NULL where
 *              that is 0); its prior contents do not matter
 */
rpd_status rpd_fp8_project(int32_t V, int32_t d, const void* packed, int32_t M, const void* x, int64_t x_stride,
                           int32_t x_dtype, void* logits, int64_t logits_stride, int32_t logits_dtype, int32_t* argmax,
                           float* confidence, float* entropy, float logit_scale, void* workspace, size_t workspace_bytes,
                           void* stream);

/*
 * Sampling from rows of logits, from given random numbers. The tokens of a row
 * are taken in order of their logits, the largest first, equal ones by index;
 * with e_j = e^(scale (z_j - z_0)) of the j-th, those are kept that pass every
 * filter:
 *   top_k   j < top_k (0: off)
 *   top_p   e_0 + .. + e_(j-1) < top_p * (the sum over what top_k leaves), or
 *           j = 0 (1 and more: off)
 *   min_p   e_j >= min_p (0: off)
 * The token is the first in that order with e_0 + .. + e_j > r * (the sum over
 * the kept). A logit of -inf is never kept. A row with NaN or +inf, or of
 * nothing but -inf, has no distribution: token -1, probability NaN, none kept.
 *   N, V       0 <= N < 2^22 (0: nothing is done), 1 <= V <= 2^20
 *   dtype      of the logits: RPD_DTYPE_BF16, _F16 or _F32
 *   logits     device [N][V], rows logits_stride >= V apart
 *   r          device [N] float32 in [0, 1)
 *   logit_scale, top_k, top_p, min_p   for all rows: an inverse temperature,
 *              > 0 and at most 2^100, or 0 for 1; >= 0; > 0; in 0 .. 1
 *   scales, top_ks, top_ps, min_ps   device [N] float32 (top_ks int32), one for
 *              each row, in place of the number, or NULL. Values out of range:
 *              a scale of 0 is 1, one below 0 or above 2^100 leaves the row no
 *              distribution; top_k below 0 is off; top_p of 0 and less keeps
 *              one token, NaN is off; min_p below 0 or NaN is off, above 1 is 1
 *   token      device [N] int32
 *   prob       device [N] float32 or NULL: the token's probability among the kept
 *   kept       device [N] int32 or NULL: how many were kept
 *   filtered   device [N][V] of the logits' type or NULL, rows filtered_stride
 *              >= V apart: the logits of the kept tokens, -inf elsewhere (as
 *              rpd_verify_draft takes them); must not overlap the logits
 * Sums are of 64 bits; equal inputs give equal outputs.
 */
typedef struct rpd_sample {
  int32_t N, V, dtype;
  const void* logits;
  int64_t logits_stride;
  const float* r;
  float logit_scale;
  int32_t top_k;
  float top_p, min_p;
  const float* scales;
  const int32_t* top_ks;
  const float* top_ps;
  const float* min_ps;
  int32_t* token;
  float* prob;
  int32_t* kept;
  void* filtered;
  int64_t filtered_stride;
} rpd_sample;

/* Workspace bytes of rpd_sample_tokens: 0, it needs none of any shape
 * (`workspace` may be NULL and is not used). */
size_t rpd_sample_workspace_size(const rpd_sample* p);
rpd_status rpd_sample_tokens(const rpd_sample* p, void* workspace, size_t workspace_bytes, void* stream);

/* Static text for a status code. */
const char* rpd_status_string(rpd_status s);

/* Detail of the calling thread's most recent non-OK status ("" if none). */
const char* rpd_last_error(void);

/* RPD_ABI_VERSION of the library. */
int32_t rpd_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* RPD_H */
