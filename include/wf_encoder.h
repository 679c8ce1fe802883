/*
 * wf_encoder.h -- C ABI of the ragged, hush-terminated speech-encoder library (sm_100a).
 *
 * The library implements the encoding stage of a streaming speech pipeline in which each
 * audio buffer x is followed by a short fixed "hush" segment h instead of being padded to
 * 30 s (paper Sec. 4.1.2, "New paradigm: hush word": x (+) h), so that the encoder --
 * the 1,500-token, tens-of-layers cost named in Sec. 1.1 and Sec. 2.3 -- runs over real
 * tokens only.  Buffers of different lengths are batched without padding (the
 * variable-length batching problem raised in Sec. 3.3): every activation is a packed
 * [sum of rows, channels] matrix plus prefix sums.
 *
 * Conventions
 *   - "dev" pointers are CUDA device pointers on the device that was current when the
 *     encoder was created; "host" pointers are ordinary host memory.
 *   - All work is enqueued on the `stream` argument (a cudaStream_t passed as void*;
 *     NULL = the legacy default stream).  Calls return without synchronising unless stated.
 *     Host arrays are read or written before the call returns.
 *   - The caller owns every buffer it passes.  The library owns its converted weights,
 *     tables and workspace, sized at create time and released by wf_encoder_destroy.
 *   - Errors are return codes; nothing aborts.  After a non-zero return the outputs are
 *     undefined.  wf_last_error gives a human-readable message for the last failure on a
 *     handle.  A handle is not thread-safe; distinct handles are independent.
 *   - Calls on one handle share its workspace: enqueue them on one stream, or order the streams
 *     yourself so that two calls never run on the GPU at the same time.
 *   - Row counts: a buffer of L samples has T = floor(L/160) frames (L >= 401 required);
 *     with the hush segment of H frames it has T' = T + H rows and n = ceil(T'/2) tokens.
 */
#ifndef WF_ENCODER_H
#define WF_ENCODER_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct wf_encoder wf_encoder;

typedef enum {
  WF_OK = 0,
  WF_ERR_INVALID_ARG = 1,
  WF_ERR_TOO_SHORT = 2,      /* a buffer has fewer than 401 samples                        */
  WF_ERR_TOO_LONG = 3,       /* a sequence would have more than n_ctx tokens               */
  WF_ERR_CAPACITY = 4,       /* batch, samples or tokens exceed what create() sized        */
  WF_ERR_CUDA = 5,           /* a CUDA runtime/driver call failed                          */
  WF_ERR_DEVICE_TIMEOUT = 6, /* a bounded wait inside a kernel gave up                     */
  WF_ERR_UNSUPPORTED_ARCH = 7,
  WF_ERR_UNIMPLEMENTED = 8
} wf_status;

typedef enum { WF_F32 = 0, WF_BF16 = 1 } wf_dtype;

/* Model and capacity description.  d_model / n_head must be 64; d_model and d_mlp multiples
 * of 128 (d_model <= 1280); n_mel a multiple of 8, at most 128.  dtype selects the arithmetic
 * of the encoder body: WF_F32 = float32 SIMT kernels, WF_BF16 = bfloat16 tensor-core kernels
 * with float32 accumulation, a residual stream held to 16 significant bits (two bfloat16
 * planes), each LayerNorm's gain folded into the weight that follows it (the product is
 * rounded to bfloat16), bfloat16 output.  The front end is float32 in both. */
typedef struct {
  int n_mel, d_model, n_layer, n_head, d_mlp;
  int n_ctx;          /* most tokens one sequence may have (positions are a closed form)   */
  int hush_frames;    /* H; 0 = no hush segment (e.g. a 30 s padded run)                    */
  int dtype;          /* wf_dtype                                                           */
  int max_batch;      /* most sequences per call                                            */
  long max_tokens;    /* most tokens per call (sum over sequences)                          */
  long max_samples;   /* most audio samples per call (sum over sequences), below 2^31       */
} wf_config;

/* Weights: float32, device memory, read (and converted) once inside wf_encoder_create.
 * Linear weights are [out, in] row-major, conv kernels [out, in, 3].  The per-layer members
 * are HOST arrays of n_layer DEVICE pointers.  The key projection has no bias. */
typedef struct {
  const float *mel_fb;                 /* [n_mel, 201] non-negative filterbank               */
  const float *conv1_w, *conv1_b;      /* [d, n_mel, 3], [d]                                 */
  const float *conv2_w, *conv2_b;      /* [d, d, 3], [d]                                     */
  const float *const *ln1_g, *const *ln1_b;
  const float *const *wq, *const *bq, *const *wk, *const *wv, *const *bv;
  const float *const *wo, *const *bo;
  const float *const *ln2_g, *const *ln2_b;
  const float *const *w1, *const *b1;  /* [d_mlp, d], [d_mlp]                                */
  const float *const *w2, *const *b2;  /* [d, d_mlp], [d]                                    */
  const float *lnp_g, *lnp_b;          /* final LayerNorm                                    */
} wf_weights;

/* Builds an encoder on the current device: converts weights to the layouts the kernels
 * read, builds the windowed-DFT and sinusoid tables on the device, allocates workspace for
 * the stated capacities.  Synchronises `stream` before returning.  Fails with
 * WF_ERR_UNSUPPORTED_ARCH on a device that is not compute capability 10.x.
 * (Operation: the encoder of Sec. 1.1 / Sec. 2.3; weights are caller-provided.)
 * Four tuning switches of the WF_BF16 path are read from the environment here and kept in the
 * handle (a later create with another environment does not change this one):
 *   WF_PDL=0               launch kernels plainly instead of with programmatic stream
 *                          serialization (on by default: a kernel's set-up overlaps the tail of
 *                          the kernel before it);
 *   WF_GEMM_SMALL_TILES=0  never use 128 x 128 single-CTA tiles for small GEMMs;
 *   WF_GEMM_TILE=1|2|3     force 256 x 256 CTA-pair tiles, 128 x 128 or 128 x 256 single-CTA tiles for the
 *                          block GEMMs instead of letting the launcher choose by the problem's size;
 *   WF_GEMM_SPLIT_K=n      split the K range of a GEMM with few tiles over a cluster of CTAs when K
 *                          has at least n blocks of 64 (default 64; 0 = never).
 * None of them changes what is computed beyond float32 rounding order (which is fixed for a
 * given setting).  Results are bit-reproducible from call to call: no kernel of
 * the encoder combines partial results in an order that varies. */
wf_status wf_encoder_create(const wf_config *cfg, const wf_weights *w, void *stream,
                            wf_encoder **out);

/* Log-mel front end alone (Sec. 4.1.2, "target level": 16 kHz audio -> 100 rows per second):
 * reflect-padded 400-point periodic-Hann DFT every 160 samples, power, mel projection,
 * log10 with floor 1e-10, clamp to (per-buffer maximum - 8), (x + 4) / 4.
 *   audio       dev  float32, the B buffers back to back (sum of lengths samples)
 *   lengths     host B sample counts
 *   mel_out     dev  float32 [sum T_i, n_mel], rows of buffer i start at sum_{j<i} T_j
 *   frames_out  host B frame counts T_i (may be NULL) */
wf_status wf_logmel(wf_encoder *enc, const float *audio, const long *lengths, int B,
                    float *mel_out, long *frames_out, void *stream);

/* The whole path: front end, hush rows appended to each buffer's log-mel rows (x (+) h of
 * Sec. 4.1.2 at the log-mel level), conv stem, sinusoid positions restarting at 0 for every
 * sequence, n_layer pre-LN blocks whose attention sees one sequence's tokens only, final
 * LayerNorm.
 *   hush_mel        dev  float32 [hush_frames, n_mel] in normalised log-mel units;
 *                        may be NULL iff hush_frames == 0
 *   hidden_out      dev  [sum n_i, d_model]; float32 for WF_F32, bfloat16 for WF_BF16
 *   cu_seqlens_out  host B+1 token prefix sums (may be NULL) */
wf_status wf_encode(wf_encoder *enc, const float *audio, const long *lengths, int B,
                    const float *hush_mel, void *hidden_out, int *cu_seqlens_out, void *stream);

/* The paper's own variant of the method (Sec. 4.1.2 "Hush word target level", Sec. 5): the hush
 * word is a raw-audio segment (8000 samples = 0.5 s) that follows the buffer BEFORE the front
 * end, x (+) h, so frames at the junction straddle both and the per-buffer maximum sees the
 * hush frames too.  The samples are never copied: the front end reads index i >= L_i of buffer i
 * from hush_audio[i - L_i].  Needs an encoder created with hush_frames == 0.
 *   hush_audio    dev  float32 [hush_samples], shared by all buffers; hush_samples <= 16000
 *   row counts         T_i = floor((L_i + hush_samples) / 160), n_i = ceil(T_i / 2)
 * Everything else as wf_encode. */
wf_status wf_encode_raw_hush(wf_encoder *enc, const float *audio, const long *lengths, int B,
                             const float *hush_audio, int hush_samples, void *hidden_out,
                             int *cu_seqlens_out, void *stream);

/* Same as wf_encode but starting from normalised log-mel rows (e.g. from wf_logmel, or a
 * raw-audio-level hush word already concatenated by the caller with hush_frames == 0).
 *   mel     dev  float32 [sum T_i, n_mel] packed;   frames  host B row counts T_i >= 1 */
wf_status wf_encode_mel(wf_encoder *enc, const float *mel, const long *frames, int B,
                        const float *hush_mel, void *hidden_out, int *cu_seqlens_out,
                        void *stream);

/* wf_encode with HOST audio and HOST output: copies the samples to a library-owned device
 * buffer, encodes, copies the hidden states back, and synchronises `stream`.
 * `audio_host` and `hidden_out_host` should be pinned for the copies to run at full rate. */
wf_status wf_encode_host(wf_encoder *enc, const float *audio_host, const long *lengths, int B,
                         const float *hush_mel, void *hidden_out_host, int *cu_seqlens_out,
                         void *stream);

/* The same without the wait, for a caller that encodes buffer after buffer (every round of the
 * streaming pipeline re-encodes the stream's buffer, Sec. 4.3.2): the call returns once its work
 * is enqueued, and the library's two sets of staging buffers let the host-to-device copy of one
 * call and the device-to-host copy of the previous one run (on two streams of the library's own)
 * under the kernels in between.  hidden_out_host holds the result, and audio_host may be reused,
 * once wf_encode_host_wait(ticket) has returned; pass pinned memory, and do not reuse an output
 * buffer before its ticket has been waited for.  At most two calls are in flight: a third call
 * first waits for the oldest.  cu_seqlens_out is written before the call returns. */
wf_status wf_encode_host_async(wf_encoder *enc, const float *audio_host, const long *lengths, int B,
                               const float *hush_mel, void *hidden_out_host, int *cu_seqlens_out,
                               void *stream, long *ticket_out);
wf_status wf_encode_host_wait(wf_encoder *enc, long ticket);

/* The host-side planner of wf_encode / wf_encode_mel alone: no device, no encoder handle, no CUDA
 * call.  Row arithmetic of the method (Sec. 4.1.2: 100 log-mel rows per second, the hush segment
 * appended; Sec. 2.1: two rows per encoder token) and the ragged work lists, with the same
 * validation and status codes as the encoding calls.
 *   lengths             host  B sample counts, or frame counts if lengths_are_frames != 0
 *   tail_samples              raw-audio hush samples that follow every buffer (wf_encode_raw_hush), else 0
 *   num_sms                   SM count the attention work list is planned for (0: never use single-tile items)
 *   cu_seqlens_out      host  B+1 token prefix sums (may be NULL)
 *   totals_out          host  6 values: log-mel frames, rows of the padded-row layout, tokens,
 *                             front-end tiles, attention work-list entries, attention items (may be NULL)
 *   work_out, work_cap  host  the attention work list as the kernels read it (may be NULL): WF_F32 pairs
 *                             (sequence, first query row) per 16 rows; WF_BF16 triples (sequence, first query
 *                             row | kind << 30, first item) followed by one entry index per item */
wf_status wf_plan(const wf_config *cfg, const long *lengths, int B, int lengths_are_frames,
                  long tail_samples, int num_sms, int *cu_seqlens_out, long *totals_out,
                  int *work_out, int work_cap);

/* Synchronises `stream` and reports WF_ERR_DEVICE_TIMEOUT if any kernel's bounded wait gave
 * up since the last check, WF_ERR_CUDA if the stream is in error, else WF_OK. */
wf_status wf_check(wf_encoder *enc, void *stream);

/* Exercises the failure path behind WF_ERR_DEVICE_TIMEOUT without any fault: enqueues a one-warp
 * kernel that waits, through the same bounded wait as the GEMM and attention kernels but with
 * `poll_limit` polls (1 .. 2^20), on a barrier that is never signalled.  The wait runs out, the
 * kernel records it and ends normally; the next wf_check on this handle returns
 * WF_ERR_DEVICE_TIMEOUT (and clears the record), and the handle stays fully usable.
 * (Every wait of the paper's encoding stage as built here, Sec. 3.2 "Operations", is of this kind.) */
wf_status wf_selftest_wait_timeout(wf_encoder *enc, unsigned poll_limit, void *stream);

wf_status wf_encoder_destroy(wf_encoder *enc);
const char *wf_last_error(const wf_encoder *enc);

/* Per-kernel-class timing.  When enabled, every launch inside wf_encode* is bracketed by
 * CUDA events on the caller's stream.  wf_profile_read synchronises, then writes for class c
 * (0 front end, 1 layout/maps, 2 conv stem GEMMs, 3 LayerNorm kernels (WF_BF16: the final one
 * only), 4 block GEMMs, 5 attention)
 * the number of launches and their summed milliseconds since the last read, and resets. */
#define WF_N_KERNEL_CLASSES 6
wf_status wf_profile_enable(wf_encoder *enc, int on);
wf_status wf_profile_read(wf_encoder *enc, long *launches, double *millis);

/* Component entry points (used by the parity tests and for profiling one kernel alone).
 *
 * wf_gemm_bf16: C = epilogue(A W^T + bias) with the tcgen05 kernel the encoder blocks use
 * (the four GEMMs of a transformer block, Sec. 1.1).  Needs a WF_BF16 encoder.
 *   A dev bf16 [M, K] row-major, W dev bf16 [N, K] row-major, bias dev float32 [N];
 *   mode 0: C bf16 [M, N] = acc + bias;  1: C bf16 = gelu(acc + bias).
 *   K and N must be multiples of 8. */
wf_status wf_gemm_bf16(wf_encoder *enc, const void *A, const void *W, const float *bias, void *C,
                       long M, int N, int K, int mode, void *stream);

/* The three pieces with which the WF_BF16 path runs a pre-LN block (x += Wo attn(LN1 x) + bo;
 * x += W2 gelu(W1 LN2 x + b1) + b2, the blocks of the encoder of Sec. 1.1 / Sec. 2.3) without a
 * LayerNorm kernel: the residual stream x is stored as two bf16 planes, x = x_hi + x_lo with
 * x_hi = bf16(x) and x_lo = bf16(x - x_hi); x_hi doubles as the A operand of the GEMM behind a
 * LayerNorm, whose gain and shift are folded into that GEMM's weight and bias.
 *
 * wf_gemm_resid_bf16: (x_hi, x_lo) <- split(x_hi + x_lo + A W^T + bias), in place, each element
 *   by one thread (bit-reproducible).  Also writes, for every row and every 128 columns, the sum
 *   and the sum of squares of the new x:
 *   A dev bf16 [M, K], W dev bf16 [N, K], bias dev float32 [N], x_hi / x_lo dev bf16 [M, N],
 *   stats dev float32 [N / 128][M][2];  N a multiple of 128, K of 8.
 * wf_ln_fold: W dev float32 [N, K], ln_g / ln_b dev float32 [K], bias dev float32 [N] or NULL ->
 *   Wg dev bf16 [N, K] = bf16(W diag(ln_g)), colsum dev float32 [N] = row sums of Wg,
 *   cbias dev float32 [N] = bias + W ln_b.
 * wf_gemm_ln_bf16: C bf16 [M, N] = LayerNorm(x; ln_g, ln_b) W^T + bias (gelu of it if `gelu`),
 *   computed as rstd (x_hi Wg^T - mean colsum) + cbias with mean and rstd (biased variance,
 *   eps 1e-5) from `stats` [K / 128][M][2] as wf_gemm_resid_bf16 leaves them for an x of K columns.
 *   K a multiple of 128, N of 8. */
wf_status wf_gemm_resid_bf16(wf_encoder *enc, const void *A, const void *W, const float *bias,
                             void *x_hi, void *x_lo, float *stats, long M, int N, int K, void *stream);
wf_status wf_ln_fold(wf_encoder *enc, const float *W, const float *ln_g, const float *ln_b,
                     const float *bias, void *Wg, float *colsum, float *cbias, int N, int K,
                     void *stream);
wf_status wf_gemm_ln_bf16(wf_encoder *enc, const void *x_hi, const float *stats, const void *Wg,
                          const float *colsum, const float *cbias, void *C, long M, int N, int K,
                          int gelu, void *stream);

/* wf_attention: non-causal attention over packed tokens, one softmax per (sequence, head)
 * over that sequence's keys only (no padded token is computed).  qkv dev [M, 3 d_model]
 * (q | k | v, head h at columns 64 h), out dev [M, d_model]; element type follows the
 * encoder's dtype.  cu_seqlens host B+1. */
wf_status wf_attention(wf_encoder *enc, const void *qkv, const int *cu_seqlens, int B, void *out,
                       void *stream);

/* Resident stream windows (Sec. 3.2: every round a stream's audio buffer is extended at its end
 * by the newly arrived audio and now and then cut at its front once a transcript segment is
 * confirmed; Sec. 4.3.2: the buffer is re-encoded every round).  The library keeps each stream's
 * window (samples and un-normalised log-mel rows) on the device, so that a round frames only the
 * audio that is new: wf_streams_push recomputes just the frames whose 400 samples changed (the
 * new ones, the two at the old end whose reflected tail became real audio and, after a cut, the
 * first two), and wf_encode_streams runs the max / clamp / scale over the cached rows, appends the
 * hush segment and encodes.  Results are identical, bit for bit, to wf_encode on the same windows.
 *
 * wf_streams_create: windows for n_streams streams of up to max_window_samples samples each
 *   (rounded up to a multiple of 160); all windows start empty.  Device memory is allocated
 *   here and released by wf_streams_destroy (which synchronises the device first).
 * wf_streams_push: for each listed stream (ids host, B distinct ids), drop trim[i] samples at the
 *   front (a multiple of 160, at most the window; trim may be NULL), then append n_new[i]
 *   samples taken back to back from new_audio (dev float32).  The window must end up with at
 *   least 401 samples (WF_ERR_TOO_SHORT) and at most its capacity (WF_ERR_CAPACITY); on an
 *   error nothing is changed.
 * wf_streams_length: samples currently in a stream's window (host bookkeeping, no sync).
 * wf_encode_streams: as wf_encode, on the current windows of the listed streams, in the order
 *   listed. */
typedef struct wf_streams wf_streams;
wf_status wf_streams_create(wf_encoder *enc, int n_streams, long max_window_samples, wf_streams **out);
wf_status wf_streams_destroy(wf_streams *st);
wf_status wf_streams_length(const wf_streams *st, int stream_id, long *samples);
wf_status wf_streams_push(wf_streams *st, const int *ids, int B, const float *new_audio,
                          const long *n_new, const long *trim, void *stream);
wf_status wf_encode_streams(wf_streams *st, const int *ids, int B, const float *hush_mel,
                            void *hidden_out, int *cu_seqlens_out, void *stream);

/* wf_cross_kv: the cross-attention key and value projections of the encoder's output for every
 * decoder layer in one GEMM, kv = hidden W_kv^T + b_kv: the first thing prompt prefill (Sec. 3.2
 * "Operations", Sec. 4.3.2) needs from the encoding stage, and the same for every later decoding
 * round on this buffer.  Runs on the encoder's path (tcgen05 for WF_BF16, float32 SIMT else).
 *   hidden  dev  [M, d_model]                   path dtype (what wf_encode wrote)
 *   W_kv    dev  [n_dec_layers * 2 d_model, d_model] path dtype, row-major: rows
 *                [2 l d, 2 l d + d) are layer l's key weight, the next d rows its value weight
 *   b_kv    dev  float32 [n_dec_layers * 2 d_model] (the architecture's key projection has no
 *                bias: those slices are zero)
 *   kv      dev  [M, n_dec_layers * 2 d_model]  path dtype; layer l's keys are columns
 *                [2 l d, 2 l d + d) of every row, its values the next d columns
 * On the bf16 path all pointers must be 16-byte aligned. */
wf_status wf_cross_kv(wf_encoder *enc, const void *hidden, const void *W_kv, const float *b_kv,
                      long M, int n_dec_layers, void *kv, void *stream);

/* wf_dtw: dynamic time warping of B token-by-frame cost matrices (token timestamping from the
 * decoder's cross-attention, Sec. 3.2 "Workload mapping" and Sec. 4.3.2, which name DTW and give
 * no further detail: this is the classic recurrence D[i,j] = C[i,j] + min(D[i-1,j-1], D[i-1,j],
 * D[i,j-1]) with the path traced back from the last cell; float32; ties prefer the diagonal,
 * then the token step, then the frame step).
 *   cost         dev  float32, problem b is a row-major [n_tokens[b], n_frames[b]] matrix, the
 *                     problems back to back
 *   n_tokens, n_frames  host  B sizes (tokens <= 16384; fewer than 2^31 cells in total)
 *   trace_ws     dev  scratch, one byte per cost cell (caller-owned)
 *   token_start  dev  int32, sum of n_tokens entries: first frame of every token on the path
 *   total_cost   dev  float32 [B]: D at the last cell */
wf_status wf_dtw(wf_encoder *enc, const float *cost, const int *n_tokens, const int *n_frames, int B,
                 unsigned char *trace_ws, int *token_start, float *total_cost, void *stream);

/* Beam-pruning state machine (Sec. 4.2.2, "New design in beam pruning"): host-side integer logic
 * that tells a beam-search decoder which beam size to use in its next round, given the top-1
 * token of the current round and the previous round's transcript as a reference.  Decoding
 * starts with beam 1; the first comparable top-1 token is searched through the reference
 * (alignment; the aligned token counts as matched); afterwards a comparable token must equal the
 * next reference token; tokens flagged special (punctuation, timestamps, other special ids) are
 * never compared and leave the state unchanged; a failed search, a mismatch or an exhausted
 * reference restores `full_beam` until the session ends.
 *   reference   host  n_reference token ids (copied);  is_special  host  vocab_size flags (copied)
 *   wf_beam_pruner_step returns the beam size for the NEXT round, or -1 on a bad argument. */
typedef struct wf_beam_pruner wf_beam_pruner;
wf_status wf_beam_pruner_create(const int *reference, int n_reference, const unsigned char *is_special,
                                int vocab_size, int full_beam, wf_beam_pruner **out);
int wf_beam_pruner_step(wf_beam_pruner *p, int top1_token);
/* reference_index: next position to compare with (-1 before alignment); any pointer may be NULL */
wf_status wf_beam_pruner_state(const wf_beam_pruner *p, long *reference_index, int *fallen_back,
                               long *rounds, long *rounds_at_one);
wf_status wf_beam_pruner_destroy(wf_beam_pruner *p);

/* wf_attention_f32_static: wf_attention for float32 activations without an encoder handle and
 * without any allocation (the paper has no counterpart; this exists for integration only).
 * It is meant for callers that cannot call cudaMalloc: code running inside a process whose
 * device memory is owned and fully handed out by another allocator, or a plug-in that is
 * given pointers and must not grow its host's footprint.  Such callers cannot create an
 * encoder, because create() allocates workspace.  Here the per-call index arrays (token prefix
 * sums and query-tile list) live in a fixed 35 KB array inside the library image, held by
 * every GPU that loads the library until the process exits.
 *   qkv dev float32 [M, 3 d_model] (q | k | v, head h at columns 64 h), out dev float32
 *   [M, d_model], cu_seqlens host B+1 strictly increasing from 0; d_model a multiple of 64.
 * Limits: B <= 256 and M <= 65,536, else WF_ERR_CAPACITY.  No cudaMalloc, cudaFree or other
 * allocating call is made.  The first call on a device looks up the array's device address
 * (once per device, with that device current); make that first call outside any stream
 * capture.  A call on a stream that is being captured is rejected (WF_ERR_INVALID_ARG): the
 * index arrays are copied from the call's own stack frame.  That copy makes the host wait for
 * earlier work on the stream, so unlike the other entry points this one does not return early.
 * All calls on a device share the array and each overwrites what it reads, so calls are safe
 * back to back on one stream, but calls that may overlap on the GPU (different streams without
 * ordering between them) race on it.  Not thread-safe: call it from one host thread at a time. */
wf_status wf_attention_f32_static(const float *qkv, const int *cu_seqlens, int B, int d_model,
                                  float *out, void *stream);

/* ---- Operators of the decoding stage (Sec. 3.2 "Operations": prompt prefill, then beam-search
 * decoding over the encoder's output; Sec. 4.3.2).  The decoder's own GEMMs are the caller's; these
 * are the pieces in between: a paged key/value cache that is quantised as it is written, attention
 * of beams or of a tree of drafted tokens over it, beam selection and the reordering of states.
 *
 * A wf_decoder handle is host memory only: it holds the configuration and the last error message,
 * no device memory and no weights, and is created without a GPU.  Every buffer and workspace is the
 * caller's, so calls on several streams (or captured into several CUDA graphs) are independent as
 * long as their buffers are.  No call synchronises, allocates or copies from host memory: all of
 * them can be captured.  Calls work on the device that is current, which owns the buffers.  Sizes that decide the
 * launch are host arguments; lengths, tables and parents are device arrays, read when the kernel
 * runs.  What a kernel finds wrong in them (a page outside the cache, a position outside the page
 * table, prefix sums that do not increase, a parent outside the beams) it passes over without
 * touching memory, and records in `status` (dev int, may be NULL; bits are or-ed into it, the
 * caller zeroes it):
 *   1  a page index outside [0, n_pages): the position is treated as absent
 *   2  prefix sums, a start or a length that do not fit the rows or the page table.  Where prefix sums decrease, which
 *      of the sequences concerned has a row is not defined
 *   4  a parent beam outside [0, n_beam): the row stays as it is; a parent or path of drafted rows that does not fit
 *   8  a bounded wait inside a kernel gave up: the outputs of the rows concerned are NaN
 *   16 a sequence's rows were put off: no room for them, or no free pages (wf_page_plan)
 *   32 a token outside the vocabulary or a temperature that is negative or not finite (wf_draft_verify)
 * A handle's calls come from one host thread at a time; distinct handles are independent. */
typedef struct wf_decoder wf_decoder;

/* Element type of a cache: WF_CACHE_PATH stores the path's own type (float32 or bfloat16);
 * the other two store one byte per element and one bfloat16 scale s per vector of d_head elements
 * (a key or a value of one position and head).  With a = max |x_i| over the vector:
 *   WF_CACHE_E4M3   s = the least power of two with a / s <= 448;  code = x / s (exact) rounded to
 *                   the nearest e4m3 value, ties to even
 *   WF_CACHE_INT8   s = a / 127 (rounded to float32) rounded up to bfloat16;  code = the whole number
 *                   nearest to x / s, ties to even, the quotient not rounded before
 * s is at least 2^-126, and 1 if a = 0.  A vector that holds a NaN or an infinity gets s = NaN and
 * zero codes, and reads back as NaN.  A stored element stands for code * s.  Codes are finite: the two
 * e4m3 codes of NaN (0x7f, 0xff), which no write makes, are not part of the format, and what stands
 * for them where a caller stores them is not defined (NaN or 480 s); a NaN scale is a vector of NaN. */
typedef enum { WF_CACHE_PATH = 0, WF_CACHE_E4M3 = 1, WF_CACHE_INT8 = 2 } wf_cache_format;

/* n_kv_head divides n_head (query head h reads key/value head h / (n_head / n_kv_head)); d_head is
 * 64 or 128; dtype (wf_dtype) is the type of queries, keys, values and outputs; page_size is a power
 * of two from 16 to 256.  At most 1024 heads. */
typedef struct {
  int n_head, n_kv_head, d_head;
  int dtype;
  int cache_format;
  int page_size;
} wf_decoder_config;

wf_status wf_decoder_create(const wf_decoder_config *cfg, wf_decoder **out);
wf_status wf_decoder_destroy(wf_decoder *dec);
const char *wf_decoder_last_error(const wf_decoder *dec);

/* One layer's cache, caller-owned device memory, 16-byte aligned:
 *   k, v              [n_pages][n_kv_head][page_size][d_head] elements or codes
 *   k_scale, v_scale  bfloat16 [n_pages][n_kv_head][page_size]; NULL for WF_CACHE_PATH
 * n_pages * n_kv_head * page_size < 2^32 - 1. */
typedef struct {
  void *k, *v;
  void *k_scale, *v_scale;
  int n_pages;
} wf_cache;

/* New rows (tokens) of a batch of sequences, packed as everywhere in this library: sequence s has
 * rows cu_rows[s] .. cu_rows[s + 1] of the row arrays, and its row i sits at cache position
 * start[s] + i.  Position p is entry p % page_size of page page_table[s * table_stride + p / page_size].
 * Rows in front of cu_rows[0] (a call for some of a batch's sequences) and at or behind cu_rows[n_seq] (padding of a batch with
 * a fixed size) are neither read nor written.
 *   n_seq, n_rows        host  sequences; rows that the row arrays have
 *   cu_rows, start       dev   int [n_seq + 1], int [n_seq]
 *   page_table           dev   int [n_seq][table_stride] */
typedef struct {
  int n_seq, n_rows;
  const int *cu_rows, *start;
  const int *page_table;
  int table_stride;
} wf_rows;

/* wf_cache_write: quantises (or copies) the rows' keys and values into the cache.
 *   k, v   dev  path dtype [n_rows][n_kv_head][d_head], heads contiguous, consecutive rows k_stride /
 *               v_stride elements apart: for instance one layer's columns of what wf_cross_kv wrote
 * wf_cache_read: the rows' values back, each rounded once to the path dtype, in the same layout.
 * Pointers are 16-byte aligned and row strides whole multiples of 16 bytes.  n_rows <= 2^27, n_rows * n_kv_head < 2^32 - 1.  No
 * two rows of a write stand for the same place of the cache (sequences may share pages that the call does not write). */
wf_status wf_cache_write(wf_decoder *dec, const wf_cache *cache, const wf_rows *rows, const void *k,
                         long k_stride, const void *v, long v_stride, int *status, void *stream);
wf_status wf_cache_read(wf_decoder *dec, const wf_cache *cache, const wf_rows *rows, void *k, long k_stride,
                        void *v, long v_stride, int *status, void *stream);

/* Which positions of its sequence a query row sees besides the start[s] committed ones. */
typedef enum {
  WF_TAIL_NONE = 0,    /* none: the rows are not in the cache.  Beams over one buffer's cross-attention cache */
  WF_TAIL_CAUSAL = 1,  /* row i sees the batch rows 0 .. i of its sequence: a prompt, a chain of drafts, a single token */
  WF_TAIL_MASK = 2     /* row i sees batch row t if bit t of its mask is set: a tree of drafted tokens */
} wf_tail;

/* wf_tree_attention: attention of the rows' queries over their sequences' cache.  Row i of sequence s
 * sees the positions [0, start[s]), and with a tail those of the batch's own rows, start[s] + t (written with
 * wf_cache_write before):
 *   out_ih = sum_j p_ihj v_jg,  p_ih = softmax over the visible j of (scale <q_ih, k_jg>),  g = h n_kv_head / n_head
 *   lse_ih = log sum_j exp(scale <q_ih, k_jg>)
 * A row that sees nothing gets out = 0 and lse = -infinity.  What a row does not see has no influence
 * on it, whatever it holds (NaN included).  Scores, softmax and sums are float32, keys and values are the stored ones
 * (code * s).  WF_BF16: the products run on the tensor cores; a probability is rounded once to
 * bfloat16, in the quantised caches after multiplication with its value's scale.  Products with codes and
 * sums before the last division stay within float32 for queries below 2^100 and stored values times
 * positions below 2^119 in magnitude.
 *   q          dev   path dtype [n_rows][n_head][d_head], rows q_stride elements apart
 *   tail       host  wf_tail;  mask  dev  uint32 [n_rows][mask_words], bit t % 32 of word t / 32 (WF_TAIL_MASK only)
 *   max_rows   host  no sequence has more rows in this call (mask_words * 32 >= max_rows)
 *   max_len    host  no sequence has more positions, its own rows included; at most table_stride * page_size and 2^30.
 *                    Longer ones are cut there and reported.
 *   out        dev   path dtype [n_rows][n_head][d_head], rows out_stride elements apart
 *   lse        dev   float32 [n_rows][n_head], or NULL
 *   workspace  dev   16-byte aligned, at least the bytes that wf_tree_attention_workspace gives for the same sizes (may be
 *                    0: then NULL).  Nothing in it has to be set and nothing is kept in it between calls.  The bytes do not grow
 *                    with every size (fewer sequences are split more): ask for the sizes of each call.
 * Pointers are 16-byte aligned and row strides whole multiples of 16 bytes.  Results do not depend on the
 * order in which blocks run.  n_seq <= 65535. */
wf_status wf_tree_attention_workspace(wf_decoder *dec, int n_seq, int n_rows, int max_rows, int max_len, size_t *bytes);
wf_status wf_tree_attention(wf_decoder *dec, const wf_cache *cache, const wf_rows *rows, const void *q, long q_stride,
                            float scale, int tail, const unsigned *mask, int mask_words, int max_rows, int max_len,
                            void *out, long out_stride, float *lse, void *workspace, size_t workspace_bytes,
                            int *status, void *stream);

/* Exercises the failure path behind status bit 8 without any fault: while `on` is not 0, every bounded wait of the
 * handle's following wf_tree_attention calls gives up at once (where the call runs on 128-row tiles, the only ones that wait),
 * and every one of its wf_gemm_e4m3 calls.  on = -1 - w: in wf_gemm_e4m3 only the waits of every block's warp w (0 .. 21) give up at
 * once, the others after 4096 looks, so that some warps go on while others have given up.
 * Such a call ends normally, its rows are NaN, and the handle stays usable; 0 restores the ordinary limit. */
wf_status wf_selftest_attention_timeout(wf_decoder *dec, int on);

/* wf_beam_select: one round of beam search.  Of all continuations of the live beams of a sequence the
 * `keep` best: c_wv = score_w + x_wv - log sum_u exp(x_wu), in descending order, ties to the lower w, then the
 * lower v.  The logarithm of the sum and c are float64 (the exponentials and their first partial sums float32), so
 * that beams are told apart where they nearly tie.
 *   logits     dev   float32 or bfloat16 (logits_dtype, a wf_dtype) [B * n_beam][vocab], rows `ld` elements apart
 *   scores     dev   float32 [B][n_beam] sums of log probabilities so far; -infinity: an unused beam
 *   beams      dev   int [B]: beams live in this round (what wf_beam_pruner_step said), or NULL: all.  Values outside
 *                    [0, n_beam] are cut to it and reported in `status` (bit 2)
 *   finished   dev   uint8 [B][n_beam] or NULL: a beam with a non-zero flag has ended; it offers one continuation, end_token
 *                    at its own score, and its logits are not read
 *   end_token  host  the token that ends a text, or -1: none
 *   suppress   dev   uint32 [(vocab + 31) / 32] or NULL: tokens whose bit is set count as -infinity, before the softmax
 *   out_*      dev   [B][keep]: float32 scores, int parents and tokens, uint8 flags (1: ended by this token or before; may be
 *                    NULL).  With fewer continuations the rest is -infinity, -1, -1, 0
 * A beam whose logits hold a NaN or +infinity, or nothing but -infinity, offers no continuation.
 * n_beam <= 16, keep <= 32, vocab <= 2^28, n_beam * vocab < 2^31. */
wf_status wf_beam_select(wf_decoder *dec, const void *logits, int logits_dtype, long ld, int B, int n_beam, int vocab,
                         const float *scores, const int *beams, const unsigned char *finished, int end_token,
                         const unsigned *suppress, int keep, float *out_scores, int *out_parents, int *out_tokens,
                         unsigned char *out_finished, int *status, void *stream);

/* wf_beam_reorder: after a selection every beam takes over the states of the beam it grew from:
 * new[b][w] = old[b][parents[b][w]], in place; a negative parent leaves the row as it is.  One pass
 * that moves only rows whose parent is another beam.
 *   parents  dev   int [B][n_beam], n_beam <= 16
 *   states   host  contiguous per-beam states (token histories, scores, unpaged caches): row b * n_beam + w
 *                  of state i starts at ptr + (b * n_beam + w) * stride_bytes and its first row_bytes move
 *   caches   host  paged caches (every layer's) that share one page table.  The beams of a sequence have
 *                  one length: its pages that are full are shared, only their table entries move; the
 *                  page being filled is each beam's own, and the positions that it holds so far are
 *                  copied from the parent's.  (With n_beam pages set aside for every page index of a sequence no
 *                  allocation is needed: a page is written only while it is its beam's last one.)
 *   page_table, lengths  dev  int [B * n_beam][table_stride] (in place), int [B] positions held; NULL without caches
 * No row of one state, cache or the table may overlap another one's; a state, cache or table that is given twice, and states
 * of one stride whose rows overlap, are refused.  With n_beam = 1 nothing can move, and nothing is looked at. */
typedef struct {
  void *ptr;
  long row_bytes, stride_bytes;
} wf_beam_state;
wf_status wf_beam_reorder(wf_decoder *dec, const int *parents, int B, int n_beam, const wf_beam_state *states,
                          int n_states, const wf_cache *caches, int n_caches, int *page_table, int table_stride,
                          const int *lengths, int *status, void *stream);

/* wf_page_plan: rows and pages of one round for a batch whose sequences come and go, planned on the device.  Free pages are
 * a ring: state = {head, count}, entries pages[(head + i) % n_pages] for i < count.  Sequence s holds lengths[s] positions in
 * the first held[s] pages of its row of the page table, lengths[s] <= held[s] * page_size.  In this order, sequences by number:
 *   - a sequence whose `ended` flag is set (its place goes to another one) gives its pages back behind the free ones and
 *     begins at length 0; those pages are handed out by later calls, not by this one;
 *   - a sequence asks for new_rows[s] rows, and for the pages that they lack beyond the held ones.  It gets them if the rows
 *     asked for so far, its own included, are at most n_rows, and it needs no page or the pages asked for so far are at
 *     most `count`.  Otherwise it gets no row and no page in this round (status bit 16); pages come from the ring's front.
 * Written: the ring, its state, the page table, held and (of ended sequences) lengths, in place; and
 *   cu_rows   dev  int [n_seq + 1]: prefix sums of the rows that were granted
 *   row_seq, row_pos  dev  int [n_rows]: a row's sequence and its position lengths[s] + i, -1 behind the last row;  may be NULL
 *   row_slot  dev  int64 [n_rows]: page * page_size + position % page_size, -1 behind the last row or without a page;  may be NULL
 * The rows then go through wf_cache_write and wf_tree_attention with `lengths` as start, and wf_draft_commit adds them to the
 * lengths.  A sequence whose numbers do not fit (a negative one, more positions than pages, rows beyond the page table) gets no
 * rows, and of a pool whose state does not fit nothing is taken: bit 2.  n_seq <= 8192. */
typedef struct {
  int *pages, *state;
  int n_pages;
} wf_page_pool;
wf_status wf_page_plan(wf_decoder *dec, const wf_page_pool *pool, int n_seq, const int *new_rows, const unsigned char *ended,
                       int *lengths, int *held, int *page_table, int table_stride, int n_rows, int *cu_rows, int *row_seq,
                       int *row_pos, long long *row_slot, int *status, void *stream);

/* wf_draft_verify: which drafted tokens of every sequence the target keeps, and the token behind them (speculative
 * sampling: what is kept is distributed as the target's own samples are).  Row 0 of a sequence is its last token, the
 * others are drafts, each the child of an earlier row: a chain, or a tree as wf_tree_attention takes it.  At a row w, from
 * row 0 on, p = softmax(logits_w / T) (T = 0: all of it on the largest logit, the lowest index of equals) and w's children are
 * tried in row order.  With x a child's token and u its random number,
 *   u q(x) < p(x):  the child is kept, and the same is done there;
 *   otherwise       p <- max(p - q, 0) / sum of it (unless that sum is 0), and the next child is tried;
 * where none is kept the token that follows is the first v with sum_{i<=v} p_i > u' sum_i p_i.  q is the distribution that w's
 * children were drawn from, or, without `draft`, all of it on x (drafts that were looked up or chosen, not drawn).  T = 0: a
 * child is kept if p(x) = 1.  What is decided, a draft or the token that follows, is decided by sums in float64, exponentials included.
 *   logits       dev   float32 or bfloat16 (logits_dtype) [n_rows][vocab], rows `ld` elements apart
 *   cu_rows      dev   int [n_seq + 1];  max_rows  host  no sequence has more rows in this call (longer ones are cut, bit 2)
 *   tokens       dev   int [n_rows] (of a first row: not looked at);  parents  dev  int [n_rows], row of the sequence below the
 *                      row's own, or NULL: chains.  A row with a parent or token that does not fit is never tried (bits 4, 32)
 *   draft        dev   float32 [n_rows][vocab], rows draft_ld elements apart: row w is the q of w's children; or NULL
 *   temperature  dev   float32 [n_seq], or NULL: 1.  One that does not fit: the sequence keeps nothing (bit 32)
 *   accept_u, sample_u  dev  float32 [n_rows], [n_seq]: random numbers from [0, 1), u of every row and u' of every sequence
 *   kept         dev   int [n_seq]: rows that stay, the first one included; as many as tokens that are new.  0 without rows
 *   out_tokens   dev   int [n_seq][max_rows]: the kept drafts' tokens, then the one that follows; -1 behind
 *   path         dev   int [n_seq][max_rows]: the rows that stay, 0 first; -1 behind
 * A row whose logits hold a NaN or +infinity, or nothing but -infinity, has no distribution: none of its children is kept, and
 * the token that follows is -1.  max_rows <= 1024, vocab <= 2^28. */
wf_status wf_draft_verify(wf_decoder *dec, const void *logits, int logits_dtype, long ld, int vocab, int n_seq, int n_rows,
                          int max_rows, const int *cu_rows, const int *tokens, const int *parents, const float *draft, long draft_ld,
                          const float *temperature, const float *accept_u, const float *sample_u, int *kept, int *out_tokens,
                          int *path, int *status, void *stream);

/* wf_draft_commit: the rows that a verification keeps become the sequences' positions.  In every cache, the vectors at
 * position start[s] + path[s][i] move to start[s] + i for i < kept[s], and lengths[s] = start[s] + kept[s].  With path = NULL
 * (chains, prompts) nothing moves.
 *   start, kept  dev   int [n_seq];  path  dev  int [n_seq][path_stride], increasing
 *   lengths      dev   int [n_seq]; may be start itself
 *   caches       host  every layer's cache; they share the page table (dev, int [n_seq][table_stride]).  The positions
 *                      concerned are the sequence's own: no page that holds one is shared with another sequence
 * A kept[s] that is negative or above path_stride counts as 0 (bit 2); a row that is not above the one before it stays where it
 * is (bit 4), as one beyond the table or in a page that does not exist (bits 2, 1; reported of rows that need not move as well).  Without
 * path or caches a length beyond the table, if there is one, is reported (bit 2).  A cache that is given twice is refused.
 * n_seq <= 65535, path_stride <= 1024. */
wf_status wf_draft_commit(wf_decoder *dec, int n_seq, const int *start, const int *kept, const int *path, int path_stride, int *lengths,
                          const wf_cache *caches, int n_caches, const int *page_table, int table_stride, int *status, void *stream);

/* Matrices in 8 bits for a decoder's products: [rows, k] as e4m3 codes with one scale for each 128 channels of a row (the
 * last block of a row may have fewer).  A scale is a power of two, kept as its exponent: byte b stands for 2^(b - 127), 255 for
 * NaN.  An element is code * scale.
 *   codes   dev  [rows][k], rows `ld` bytes apart, 16-byte aligned
 *   scales  dev  bytes [ceil(k / 512)][scale_ld][4], aligned to 4: block b of row r is byte b % 4 at [b / 4][r], so that a
 *                word holds four blocks of a row and consecutive rows lie side by side.  scale_ld >= rows */
typedef struct {
  void *codes;
  unsigned char *scales;
  long ld, scale_ld;
} wf_e4m3;

/* wf_quantise_e4m3: x [rows, k] (float32 or bfloat16, rows ldx elements apart) as codes and scales, activations as well as
 * weights.  With a = max |x| over a block: scale = the least power of two s >= 2^-126 with a / s <= 448 (1 if a = 0), code =
 * x / s (exact) rounded to the nearest e4m3 value, ties to even.  A block with a NaN or an infinity gets the scale NaN and
 * zero codes.  The bytes behind a row's last block, up to a whole word, are written (127).  k <= 2^22. */
wf_status wf_quantise_e4m3(wf_decoder *dec, const void *x, int x_dtype, long ldx, long rows, int k, const wf_e4m3 *out, void *stream);

/* wf_gemm_e4m3: C[m, n] = act(A W^T + bias), A [m, k], W [n, k]: the decoder's projections.  Products of codes and scales are
 * exact, sums are the tensor cores' float32; act is the erf-form GELU if `gelu` (for bfloat16 outputs within 8e-6 of it, relative, down to
 * sums of -5, within half a step of bfloat16 down to -8, and 0 below -16; NaN of -infinity), and C (out_dtype: float32 or bfloat16) is
 * rounded once.  bias: dev float32 [n] or NULL.  C's rows are ldc elements apart, any alignment of its type; nothing behind a row's n
 * elements is written.  A NaN scale or code makes the sums that it is part of NaN. */
wf_status wf_gemm_e4m3(wf_decoder *dec, const wf_e4m3 *a, const wf_e4m3 *w, const float *bias, void *out, int out_dtype, long ldc, long m,
                       int n, int k, int gelu, int *status, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* WF_ENCODER_H */
