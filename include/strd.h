/*
 * strd.h -- C ABI of the stateful token-reduced prefill library for MI355X (gfx950).
 *
 * One hybrid layer of "Stateful Token Reduction for Long-Video Hybrid VLMs" is
 * prefilled on a reduced token set: score the vision tokens against the text
 * query, keep the top K in temporal order, compact every per-token tensor, run the
 * layer mixer (Mamba-2 scan or causal GQA attention) on the K + M survivors.
 *
 * Common rules for every entry point
 *   - A sequence is N vision tokens followed by M text tokens (Sec. 3.1).  All
 *     tensors are token-major, contiguous, batch 1.
 *   - Pointers marked [dev] are device pointers owned by the caller; [host] are
 *     host pointers.  The library allocates, frees and retains no device memory, with
 *     one exception that is stated where it applies: strd_linear hands the products its
 *     own kernel is not built for to rocBLAS and keeps that library's handle (and whatever
 *     it allocates) for the life of the process.
 *   - `io` is the element type of the tensors declared `const void*` / `void*`
 *     (STRD_F32 or STRD_BF16); accumulation, exponentials, decay, state and scores
 *     are fp32 (strd_ssd_prefill says where a long bf16 sequence is an exception).
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*; NULL = the null
 *     stream) and the call returns without synchronising.
 *   - `ws` is caller-provided scratch [dev] of at least the size the matching
 *     *_workspace() query returns (may be NULL when that size is 0); its contents
 *     are undefined before and after the call.  Tensor buffers and `ws` must be 16-byte
 *     aligned (the matrix-core kernels move 16-byte vectors straight from the caller's
 *     pointers; a misaligned buffer on such a shape is STRD_EINVAL), fp32 vectors of
 *     per-head or per-token scalars (A, D, dt) need only their natural alignment.
 *   - Return value: STRD_OK or a negative strd_status.  On STRD_EINVAL,
 *     STRD_EUNSUPPORTED and STRD_EWORKSPACE nothing was launched and no output was
 *     written.  STRD_EHIP reports a failed launch (hipGetLastError).
 *   - Shapes the kernels are not built for give STRD_EUNSUPPORTED; there is no CPU
 *     or library fallback.
 *   - The two scores and the two mixers each have two device kernels: a matrix-core
 *     (MFMA) kernel for bf16 tensors in the tile shapes listed at strd_*_kernel_path
 *     below, and a general kernel in fp32 arithmetic that serves fp32 tensors (whose
 *     1e-4 tolerance bf16 matrix cores cannot meet) and every other bf16 shape.  Which one a
 *     call will run is never implicit: strd_*_kernel_path answers it from the shape alone.
 */
#ifndef STRD_H
#define STRD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { STRD_F32 = 0, STRD_BF16 = 1 } strd_dtype;

typedef enum {
    STRD_OK = 0,
    STRD_EINVAL = -1,       /* inconsistent sizes or NULL where data is required  */
    STRD_EUNSUPPORTED = -2, /* valid problem, no kernel built for this shape       */
    STRD_EWORKSPACE = -3,   /* ws == NULL or ws_bytes too small                    */
    STRD_EHIP = -4          /* the HIP runtime refused a launch                    */
} strd_status;

/* Human-readable name of a status code (static storage, never NULL). */
const char *strd_status_string(int status);

/* ABI version: major * 1000 + minor. */
int strd_version(void);

/* Measurement aid (used by the benchmark, not by the path; for callers that want to know what
 * the matrix cores of their chip sustain): `workgroups` x 4 waves each issue `iters` x 32
 * independent v_mfma_f32_32x32x16_bf16 products on register-resident operands and write one
 * float per thread to out [dev] [workgroups * 256] (a checksum, so that nothing is optimised
 * away).  `mode` bit 0: random bf16 operands in +-[1, 2) instead of 1.0 everywhere; bit 1: the
 * 16 x 16 x 32 form of the instruction, twice as many products of half the size.  One launch is
 * workgroups * 4 * iters * 32 * 32768 flop in either form; time it with events on `stream`.
 * STRD_EINVAL for out == NULL, workgroups < 1, iters < 1 or mode outside 0..3. */
int strd_mfma_rate_probe(float *out, int workgroups, int iters, int mode, void *stream);

/* Which device kernel a call with these sizes runs: STRD_PATH_MFMA (bf16 matrix cores),
 * STRD_PATH_SIMT (fp32 arithmetic: fp32 tensors, and bf16 shapes outside the bf16
 * matrix-core tiles) or STRD_PATH_NONE (the call would return STRD_EINVAL or
 * STRD_EUNSUPPORTED).  Matrix-core shapes, all bf16: score_attn and attn_prefill d in {64, 128};
 * score_mamba n in {64, 128}; ssd_prefill n in {64, 128} and P a multiple of 32 (and every
 * tensor below 4 GiB).  Host-only, touches no device. */
typedef enum { STRD_PATH_NONE = 0, STRD_PATH_MFMA = 1, STRD_PATH_SIMT = 2 } strd_kernel_path;
int strd_score_attn_kernel_path(int M, int N, int Hq, int Hkv, int d, strd_dtype io);
int strd_score_mamba_kernel_path(int M, int N, int H, int G, int n, strd_dtype io);
int strd_ssd_prefill_kernel_path(int T, int H, int P, int G, int n, strd_dtype io);
int strd_attn_prefill_kernel_path(int T, int Hq, int Hkv, int d, strd_dtype io);

/* ---------------------------------------------------------------------------
 * score_attn -- attention-layer importance (Sec. 3.1 "Attention Layers"):
 *     s_i = 1/(M*Hq) * sum_{m,h} softmax_i( scale * q_m^h . k_i^{kv(h)} )
 * The softmax runs over the N vision keys only, so sum_i s_i = 1.  Query head h
 * reads key head kv(h) = h / (Hq/Hkv).
 *   q_txt  [dev] [M, Hq, d]   text-row queries (already projected / rotated)
 *   k_vis  [dev] [N, Hkv, d]  vision-row keys
 *   scores [dev] [N] fp32     output
 * Requires M,N >= 1, Hq % Hkv == 0, scale > 0.  Deterministic (fixed reduction order).
 * ------------------------------------------------------------------------- */
size_t strd_score_attn_workspace(int M, int N, int Hq, int Hkv, int d, strd_dtype io);
int strd_score_attn(const void *q_txt, const void *k_vis, float *scores, int M, int N, int Hq,
                    int Hkv, int d, float scale, strd_dtype io, void *ws, size_t ws_bytes,
                    void *stream);

/* ---------------------------------------------------------------------------
 * score_mamba -- Decoupled Content Alignment (Eq. "ssm_importance"), the
 * decay-free Mamba-2 score.  Delta is per head while b, c are per group, so the
 * mean runs over every head:
 *     s_i = 1/(M*H) * sum_{m,h} dt_i^h * | b_i^{g(h)} . c_m^{g(h)} |,  g(h) = h/(H/G)
 * which equals the paper's group form with the group-mean of Delta in b-bar.
 *   B_vis  [dev] [N, G, n]   vision-row input projections b
 *   C_txt  [dev] [M, G, n]   text-row output projections c
 *   dt_vis [dev] [N, H] fp32 discretisation steps (> 0, already softplus'd)
 *   scores [dev] [N] fp32    output
 * Requires M,N >= 1, H % G == 0.  Deterministic.
 * ------------------------------------------------------------------------- */
size_t strd_score_mamba_workspace(int M, int N, int H, int G, int n, strd_dtype io);
int strd_score_mamba(const void *B_vis, const void *C_txt, const float *dt_vis, float *scores,
                     int M, int N, int H, int G, int n, strd_dtype io, void *ws, size_t ws_bytes,
                     void *stream);

/* ---------------------------------------------------------------------------
 * score_mamba_full -- the Full Mamba Dynamic score (|w_{t,j}| of Eq. "ssm_weight"),
 * which the decay-free score above is ablated against: every term carries the
 * decay of the recurrence from vision token i to text row m,
 *     s_i = 1/(M*H) * sum_{m,h} dt_i^h * | b_i^{g(h)} . c_m^{g(h)} | * prod_{u=i+1}^{N+m} exp(dt_u^h * A^h).
 * With A = 0 it equals score_mamba.
 *   B_vis  [dev] [N, G, n]      C_txt [dev] [M, G, n]
 *   dt_all [dev] [N+M, H] fp32  steps of every token, vision rows first (the decay runs through
 *                               the later vision tokens and the text rows up to m)
 *   A      [dev] [H] fp32 (< 0) scores [dev] [N] fp32 output
 * Requires M,N >= 1, H % G == 0; the workspace is always needed.  Deterministic.
 * ------------------------------------------------------------------------- */
size_t strd_score_mamba_full_workspace(int M, int N, int H, int G, int n, strd_dtype io);
int strd_score_mamba_full(const void *B_vis, const void *C_txt, const float *dt_all, const float *A,
                          float *scores, int M, int N, int H, int G, int n, strd_dtype io, void *ws,
                          size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * select_topk -- keep the K highest-scoring vision tokens, in temporal order
 * (Sec. 3.1 "Token Selection").  Ties at the K-th score go to the lowest index.
 *   scores [dev] [N] fp32, finite and >= 0 (both score kinds are); -0.0 counts as 0.  Other
 *          values do not break the call: negative scores and infinities order as numbers, NaNs
 *          by their bit patterns (positive-signed above +inf, negative-signed below -inf), and
 *          exactly K indices are written in every case
 *   idx    [dev] [K] int32 output, strictly ascending
 * Requires 1 <= K <= N.  Bit-exact and deterministic.
 *   ws     [dev] strd_select_topk_workspace(N, K) bytes (0 up to 32768 scores and above 2^20;
 *          about 570 KB of histograms, counters, candidates and tables between); contents need not be initialised and
 *          are not preserved; STRD_EWORKSPACE if it is missing or too small
 * ------------------------------------------------------------------------- */
size_t strd_select_topk_workspace(int N, int K);
int strd_select_topk(const float *scores, int N, int K, int32_t *idx, void *ws, size_t ws_bytes,
                     void *stream);

/* select_topk_noalloc -- strd_select_topk for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same result,
 * bit for bit; no workspace argument: the histograms, counters, candidates and tables of the selection
 * live in a 570 KB array inside the library's image, one copy per GPU, held until the process ends.  The
 * call allocates and frees nothing (no hipMalloc / hipFree, no allocating library routine).
 *   N at most strd_select_topk_noalloc_max_n() = 1 048 576 scores; more gives STRD_EUNSUPPORTED
 *   and nothing is launched.  Other arguments and errors as strd_select_topk.
 * All calls on one GPU share that GPU's array (every call clears what it needs on `stream`
 * before using it, so nothing is carried from one call to the next): calls that overlap on one
 * GPU -- different streams, or different threads -- race; serialise them.  The first call on each
 * GPU looks the array's device address up (hipGetSymbolAddress); make that first call outside
 * any stream capture. */
int strd_select_topk_noalloc_max_n(void);
int strd_select_topk_noalloc(const float *scores, int N, int K, int32_t *idx, void *stream);

/* ---------------------------------------------------------------------------
 * compact -- drop the unselected vision tokens of one per-token tensor
 * (Sec. 3.1: retained tokens continue; text tokens are never dropped):
 *     dst[r, :]   = src[idx[r], :]   r < K
 *     dst[K+m, :] = src[N+m, :]      m < M
 *     pos_out     = the same gather applied to pos_in (identity map if pos_in NULL)
 *   src     [dev] [N+M rows of row_bytes]      dst [dev] [K+M rows]; must not overlap src
 *   idx     [dev] [K] int32, ascending, each in [0, N) (not checked on the device)
 *   pos_in  [dev] [N+M] int32 or NULL          pos_out [dev] [K+M] int32 or NULL
 * row_bytes > 0 and a multiple of 4; rows need only their natural alignment when
 * row_bytes % 16 != 0.  src/dst may be NULL when only the position map is wanted.
 * Requires 0 <= K <= N, M >= 0.  Bit-exact copy.
 * ------------------------------------------------------------------------- */
int strd_compact(const void *src, const int32_t *idx, void *dst, int N, int M, int K,
                 int64_t row_bytes, const int32_t *pos_in, int32_t *pos_out, void *stream);

/* compact_batch -- the same gather for up to STRD_COMPACT_MAX tensors that share one index
 * list (a reducing layer compacts every mixer input and the hidden states), in one launch.
 *   items [host] [n_items] {src [dev], dst [dev], row_bytes}; read before the call returns
 * Every item obeys the rules of strd_compact; n_items may be 0 when only pos_out is wanted. */
#define STRD_COMPACT_MAX 8
typedef struct {
    const void *src;
    void *dst;
    int64_t row_bytes;
} strd_compact_item;
int strd_compact_batch(const strd_compact_item *items, int n_items, const int32_t *idx, int N, int M,
                       int K, const int32_t *pos_in, int32_t *pos_out, void *stream);

/* ---------------------------------------------------------------------------
 * Packed batches of sequences -- scoring, selection and compaction (Sec. 3.1,
 * "Layer-wise Token Importance" and the token selection after it) for several
 * sequences of different lengths in one set of launches.  Each sequence is
 * reduced on its own, exactly as by the single-sequence calls above; the
 * point is that short sequences, whose calls are bound by launch latency,
 * share their launches.
 *
 * Layout.  The per-token tensors of the sequences lie one after the other
 * along the token axis (no padding): sequence b is rows
 * [row0_b, row0_b + N_b + M_b), row0_b = sum over earlier sequences of
 * (N + M), its N_b vision rows first, then its M_b text rows.  `seqs` is a
 * HOST array of `nseq` descriptors, read before the call returns.
 *   scores  [dev] [nseq, ld] fp32: row b holds the N_b scores of sequence b
 *           (entries past N_b are not touched); ld >= every N_b, ld % 4 == 0.
 *   idx     [dev] [sum of K_b] int32: the kept vision tokens of sequence b,
 *           ascending and local to the sequence (0 .. N_b - 1), start at
 *           offset sum of earlier K.
 *   compacted tensors: sequence b is rows [o_b, o_b + K_b + M_b),
 *           o_b = sum over earlier sequences of (K + M).
 *   pos_out [dev] [sum of (K_b + M_b)] int32: row number inside its own
 *           sequence's N_b + M_b input rows (pos_in == NULL), or
 *           pos_in[row0_b + that row]; pos_in [dev] [sum of (N_b + M_b)].
 * Requires 1 <= nseq <= STRD_VARLEN_MAX, every N_b >= 1, M_b >= 1,
 * 1 <= K_b <= N_b (the scores ignore K_b; select and compact use it), and for
 * strd_select_topk_varlen every N_b <= strd_select_topk_varlen_max_n()
 * (32768: one workgroup per sequence), else STRD_EINVAL / STRD_EUNSUPPORTED.
 * The same alignment rules as the single-sequence calls apply to the packed
 * base pointers.  Tie-breaking, NaN handling and error behaviour are those of
 * the single-sequence calls (a scale that is not > 0: STRD_EINVAL).
 * ------------------------------------------------------------------------- */
#define STRD_VARLEN_MAX 64
typedef struct strd_seq {
    int32_t N; /* vision tokens */
    int32_t M; /* text tokens (they follow the vision tokens) */
    int32_t K; /* vision tokens to keep */
} strd_seq;
size_t strd_score_attn_varlen_workspace(const strd_seq *seqs, int nseq, int Hq, int Hkv, int d, strd_dtype io);
int strd_score_attn_varlen(const void *q_all /* [dev] [rows, Hq, d] */, const void *k_all /* [dev] [rows, Hkv, d] */,
                           float *scores, int ld, const strd_seq *seqs, int nseq, int Hq, int Hkv, int d,
                           float scale, strd_dtype io, void *ws, size_t ws_bytes, void *stream);
/* The same, and the ld - N_b floats behind the scores of sequence b become 0. */
int strd_score_attn_varlen_padded(const void *q_all, const void *k_all, float *scores, int ld, const strd_seq *seqs, int nseq,
                                  int Hq, int Hkv, int d, float scale, strd_dtype io, void *ws, size_t ws_bytes, void *stream);
size_t strd_score_mamba_varlen_workspace(const strd_seq *seqs, int nseq, int H, int G, int n, strd_dtype io);
int strd_score_mamba_varlen(const void *B_all /* [dev] [rows, G, n] */, const void *C_all /* [dev] [rows, G, n] */,
                            const float *dt_all /* [dev] [rows, H] */, float *scores, int ld,
                            const strd_seq *seqs, int nseq, int H, int G, int n, strd_dtype io, void *ws,
                            size_t ws_bytes, void *stream);
int strd_score_mamba_varlen_padded(const void *B_all, const void *C_all, const float *dt_all, float *scores, int ld,
                                   const strd_seq *seqs, int nseq, int H, int G, int n, strd_dtype io, void *ws, size_t ws_bytes,
                                   void *stream);
int strd_select_topk_varlen_max_n(void);
int strd_select_topk_varlen(const float *scores, int ld, const strd_seq *seqs, int nseq, int32_t *idx,
                            void *stream);
int strd_compact_varlen(const strd_compact_item *items, int n_items, const int32_t *idx, const strd_seq *seqs,
                        int nseq, const int32_t *pos_in, int32_t *pos_out, void *stream);

/* ---------------------------------------------------------------------------
 * ssd_prefill -- Mamba-2 mixer over T tokens (Eqs. "ssm_state_update",
 * "ssm_output"), per head h with group g(h):
 *     S_t = exp(dt_t * A) * S_{t-1} + x_t (dt_t * b_t)^T ,   y_t = S_t c_t (+ D x_t)
 * evaluated in its chunked (state-space-dual) form with the state carried on chip.
 *   x   [dev] [T, H, P]          dt [dev] [T, H] fp32 (> 0)     A [dev] [H] fp32 (<= 0)
 *   B,C [dev] [T, G, n]          D  [dev] [H] fp32 or NULL
 *   S_in  [dev] [H, P, n] fp32 or NULL (zero state)
 *   y     [dev] [T, H, P]        S_out [dev] [H, P, n] fp32 or NULL
 * The bf16 matrix-core kernels add D x_t inside the token product (D joins the bf16 weight of
 * token t on itself), i.e. that term carries a relative rounding error of up to 2^-8, like every
 * other term of the sum and like the bf16 output itself.
 * Long bf16 sequences are cut into segments: there the part of an output that the state carries is rounded to bf16
 * before it is added (not where four heads of a group and P = 64 go together, from 64 heads on), and the first outputs of
 * a segment are rounded a second time when what the earlier segments left is added to them (from the 65th token on
 * where four heads go together).
 * Values of x, dt or S_in that are not finite stay in the state and show in every later output of their channel (dt: of
 * their head) and in S_out -- in a sequence cut into segments of fewer heads up to the end of the segment and, behind it,
 * for as long as the decays since its start are not zero in fp32.
 * `chunk` is the chunk length of the caller's formulation (> 0).  It is validated and
 * otherwise unused: it does NOT select the tiling.  The kernels always cut time into steps of
 * 64 or 32 tokens and carry the state across them on chip, so results do not depend on
 * `chunk` at all.  S_out of one call fed as S_in of the next continues the same scan; the two may be one buffer (but
 * not overlap in part).  Such a call runs a kernel in which nobody else reads what a workgroup writes: for long bf16
 * sequences the walk over the whole sequence (1.4 to 2.3 times the time of the segments), for a few small chunks in
 * single precision three launches instead of one.
 *   ws  [dev] strd_ssd_prefill_workspace(T, ...) bytes.  bf16 matrix-core shapes: 0 for short
 *       sequences; for long ones the sequence is cut into segments that run side by side, and the local end state and total
 *       decay of every segment but the last pass through the workspace ((segments - 1) * H * P * n
 *       + segments * H floats; with four heads together also 64 * P floats per head and segment and one per head and
 *       token); too small or NULL when needed: STRD_EWORKSPACE.  A state updated in place needs none there.  Other shapes: the state
 *       before every 64-token chunk and the chunks' decays, (P * n + 1) * H floats per chunk, of as many
 *       chunks as fit 256 MB (one at least), and two states more when that is not all of them.  Here it
 *       may be smaller or NULL: the call then walks the sequence token by token, which takes 65 times as
 *       long at 544 tokens; a few tokens (up to 2 to 8, by size) and states of more than 2^28 entries
 *       are always walked so, and need 0 bytes.
 * Requires T >= 0, H % G == 0.
 * ------------------------------------------------------------------------- */
size_t strd_ssd_prefill_workspace(int T, int H, int P, int G, int n, int chunk, strd_dtype io);
int strd_ssd_prefill(const void *x, const float *dt, const float *A, const void *B, const void *C,
                     const float *D, const float *S_in, void *y, float *S_out, int T, int H, int P,
                     int G, int n, int chunk, strd_dtype io, void *ws, size_t ws_bytes,
                     void *stream);

/* ssd_prefill_gather -- ssd_prefill on the K + M surviving tokens WITHOUT a compacted copy of
 * the mixer inputs: token t of the scan is row idx[t] (t < K) or N + (t - K) of the
 * uncompacted x, dt, B, C (N + M rows each).  Equal, bit for bit, to compacting the four
 * tensors with strd_compact and calling strd_ssd_prefill, minus that HBM round trip.
 *   idx [dev] [K] int32, ascending, each in [0, N)     y [dev] [K+M, H, P] (dense)
 *   ws  [dev] strd_ssd_prefill_workspace(K + M, ...) bytes, as for the dense call on K + M tokens.
 * Only shapes the matrix-core kernels cover (bf16, n in {64, 128}, P % 32 == 0, K + M >= 1);
 * anything else gives STRD_EUNSUPPORTED (compact, then call strd_ssd_prefill). */
int strd_ssd_prefill_gather(const void *x, const float *dt, const float *A, const void *B, const void *C,
                            const float *D, const float *S_in, const int32_t *idx, void *y, float *S_out,
                            int N, int M, int K, int H, int P, int G, int n, int chunk, strd_dtype io,
                            void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * attn_prefill -- causal softmax attention with grouped-query heads over T tokens
 * (App. "Attention via Kernel Functions", first equation):
 *     o_t^h = sum_{j<=t} softmax_j( scale * q_t^h . k_j^{kv(h)} ) v_j^{kv(h)}
 * in the order the tokens have in the (compacted) sequence.
 *   q [dev] [T, Hq, d]    k, v [dev] [T, Hkv, d]    o [dev] [T, Hq, d]
 * The bf16 matrix-core kernels give NaN for a row whose scores reach 1e9 in size (strd_attn_prefill_varlen does not).
 * Requires T >= 0, Hq % Hkv == 0, scale > 0 (else STRD_EINVAL).
 * ------------------------------------------------------------------------- */
size_t strd_attn_prefill_workspace(int T, int Hq, int Hkv, int d, strd_dtype io);
int strd_attn_prefill(const void *q, const void *k, const void *v, void *o, int T, int Hq, int Hkv,
                      int d, float scale, strd_dtype io, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Block glue around the mixers: what a hybrid layer does between
 * its projections and the scan or attention, apart from matrix products.  The paper builds on
 * the Mamba-2 block and does not restate these operations; they follow that block's published
 * definition.  All: [dev] tensors of the io dtype (weights included) unless stated, fp32
 * arithmetic, one rounding on output, asynchronous on `stream`, T = 0 allowed.
 *
 * rmsnorm:        out[t,:] = x[t,:] / sqrt(mean(x[t,:]^2) + eps) * w            x, out [T, d], w [d]
 * gated_rmsnorm:  v = y * silu(z); out = v / sqrt(mean_group(v^2) + eps) * w    y, out [T, D]; z rows of
 *                 pitch ldz >= D elements; `groups` equal groups of D / groups channels each; w [D]
 * conv1d_silu:    causal depthwise convolution over tokens with zero history, then SiLU,
 *                   o[t,c] = silu(b[c] + sum_{k<W} w[c,k] * xbc[t-(W-1)+k, c]),
 *                 on the first Cx + 2*Cb columns of xbc (rows of pitch ld elements); columns
 *                 [0,Cx) go to x_out [T,Cx], the next Cb to B_out [T,Cb], the last Cb to C_out
 *                 [T,Cb]; w [Cx+2*Cb, W], b [Cx+2*Cb] or NULL.  Cx, Cb, ld multiples of 8 and
 *                 16-byte (bf16) / 32-byte (fp32) aligned bases, W <= 4, else STRD_EUNSUPPORTED.
 * softplus_dt:    dt[t,h] = log(1 + exp(raw[t, col0+h] + bias[h])), raw rows of pitch ld in the io
 *                 dtype, bias [H] fp32 or NULL, dt [T,H] fp32.
 * linear:         out[T,Nd] = x[T,Kd] . w[Kd,Nd] (+ residual[T,Nd], which may be `out` itself): the
 *                 projections of a block, fp32 accumulation, the residual added in fp32 before the one
 *                 rounding.  Large bf16 products (see linear_mfma; at least one 256 x 256 output tile per
 *                 CU, 16-byte aligned pointers) run on the library's own kernel; everything else (fp32,
 *                 other shapes, small products) is handed to rocBLAS.  That second path is the one place
 *                 where something is retained: its first use in a process creates a rocBLAS handle (which
 *                 allocates device workspace of its own) and keeps it until the process ends; calls are
 *                 serialised on it.  Callers that must not allocate use strd_linear_mfma.
 * linear_library: the same product by rocBLAS whatever the shape (what strd_linear falls back to; kept as an
 *                 entry point so that the two can be timed side by side).
 * linear_mfma:    the same product by the library's own kernel only (bf16 matrix cores): no handle, no
 *                 allocation, nothing kept between calls.  bf16, Kd a multiple of 64, Nd a multiple of 8,
 *                 x and w below 4 GiB each, all pointers 16-byte aligned (STRD_EINVAL if not); other shapes
 *                 return STRD_EUNSUPPORTED (strd_linear_mfma_supported answers that from the shape alone:
 *                 1 or 0).  `residual` may be `out`.  Any size is computed correctly; below one output tile
 *                 per CU most of the chip idles.
 * ------------------------------------------------------------------------- */
int strd_linear(const void *x, const void *w, const void *residual, void *out, int T, int Kd, int Nd,
                strd_dtype io, void *stream);
int strd_linear_mfma(const void *x, const void *w, const void *residual, void *out, int T, int Kd, int Nd,
                     strd_dtype io, void *stream);
int strd_linear_library(const void *x, const void *w, const void *residual, void *out, int T, int Kd, int Nd,
                        strd_dtype io, void *stream);
int strd_linear_mfma_supported(int T, int Kd, int Nd, strd_dtype io);
/* How that kernel cuts the 256 x 256 tiles of its last round over the chip: 0 not at all, 1 into halves of 128
 * tokens, 2 into quarters of 128 x 128.  Host-only. */
int strd_linear_mfma_cut(int T, int Nd);
int strd_rmsnorm(const void *x, const void *w, void *out, int T, int d, float eps, strd_dtype io, void *stream);
int strd_gated_rmsnorm(const void *y, const void *z, int ldz, const void *w, void *out, int T, int D,
                       int groups, float eps, strd_dtype io, void *stream);
int strd_conv1d_silu(const void *xbc, int ld, const void *w, const void *b, void *x_out, void *B_out,
                     void *C_out, int T, int Cx, int Cb, int W, strd_dtype io, void *stream);
int strd_softplus_dt(const void *raw, int ld, int col0, const float *bias, float *dt, int T, int H,
                     strd_dtype io, void *stream);

/* ---------------------------------------------------------------------------
 * Variants around the reduced prefill.
 *
 * avgpool -- the average-pooling reduction that the "Reduction Types" ablation (Sec. 4,
 * ablation table, right half) sets against query-based selection.  The paper does not state
 * the window shape; here the N vision rows are cut into K consecutive windows
 * [floor(j N / K), floor((j+1) N / K)), j < K, each replaced by its mean (fp32 accumulation in
 * row order, one rounding), and the M text rows follow unchanged.  src [dev] [N+M, D], dst [dev]
 * [K+M, D], both of dtype io and contiguous (src == dst == NULL: positions only); pos_out [dev]
 * [K+M] or NULL receives pos_in (NULL = identity) of the first row of each window, then of the
 * text rows.  1 <= K <= N (K = 0 only with N = 0).
 *
 * ssd_decode_step -- one token of the Mamba-2 recurrence (Eqs. ssm_state_update, ssm_output with
 * T = 1) from the state a prefill left in S_out:  S <- exp(dt_h A_h) S + dt_h x b^T (in place),
 * y = S c + D x.  x, y [dev] [H, P] and B, C [dev] [G, n] of dtype io; dt, A, D (or NULL) [dev]
 * fp32 [H]; S [dev] fp32 [H, P, n], read and written.
 *
 * attn_decode_step -- the newest token's causal attention over a cache of T key/value rows, its
 * own row included (the last row of the appendix's softmax-attention equation): q, o [dev]
 * [Hq, d]; k_cache, v_cache [dev] [T, Hkv, d] -- after a reduced prefill these are the K + M
 * surviving rows followed by the generated ones.  d in {64, 128}, Hq / Hkv in {1, 2, 4, 8},
 * 16-byte (bf16) / 32-byte (fp32) aligned bases, else STRD_EUNSUPPORTED; scale > 0.  Workspace
 * [dev]: strd_attn_decode_step_workspace bytes, 16-byte aligned (STRD_EWORKSPACE otherwise).
 *
 * All asynchronous on `stream`; no call allocates.
 * ------------------------------------------------------------------------- */
int strd_avgpool(const void *src, void *dst, int N, int M, int K, int D, strd_dtype io, const int32_t *pos_in,
                 int32_t *pos_out, void *stream);
int strd_ssd_decode_step(const void *x, const float *dt, const float *A, const void *B, const void *C,
                         const float *D, float *S, void *y, int H, int P, int G, int n, strd_dtype io,
                         void *stream);
size_t strd_attn_decode_step_workspace(int T, int Hq, int Hkv, int d, strd_dtype io);
int strd_attn_decode_step(const void *q, const void *k_cache, const void *v_cache, void *o, int T, int Hq,
                          int Hkv, int d, float scale, strd_dtype io, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Serving what a reduced prefill keeps: attention over packed sequences with changed scores, a cache in 4 bits, decode steps
 * that gather attention weights, and eviction by them.
 *
 * Scores.  With x = scale * q_t^h . k_j, in this order:
 *     cap > 0:    x = cap * tanh(x / cap)                      (cap = 0: no cap)
 *     slopes:     x = x - slopes[h] * |pos[t] - pos[j]|        (NULL: no bias)
 *   slopes [dev] [Hq] fp32, finite, a negative one times the largest distance above -1e30; pos [dev] int32, a position per row (after a compaction the rows' old
 *   positions: pos_out of strd_compact), taken as fp32 numbers (exact below 2^24); NULL: the row's number in its sequence.
 * cap must be finite and >= 0, else STRD_EINVAL.
 * Weighted values are summed in fp32 before the sum is divided by that of the weights: a value's size times the number of rows has to stay below 2^112 (5e33).
 *
 * attn_prefill_varlen -- strd_attn_prefill for a packed batch (strd_seq above; K is not looked at, N and M may be 0, and so may a
 * sequence's rows altogether): a row attends to rows of its own sequence only,
 *     to those up to itself; with prefix != 0 a vision row to every vision row of its sequence instead.
 *   q [dev] [rows, Hq, d], k, v [dev] [rows, Hkv, d] with row pitches ldq, ldk, ldv in elements (>= a row's own), so that they may
 *   be column ranges of one projection; o [dev] [rows, Hq, d], contiguous.  Rows behind the last sequence are neither read nor
 *   written.  What a row does not see does not reach it, values that are not finite included.  pos holds one number per row.
 *   bf16 with d in {64, 128}, 16-byte aligned tensors and pitches that are multiples of 8 go to the matrix cores
 *   (strd_attn_prefill_varlen_kernel_path), d <= 256 otherwise; no workspace.  Hq % Hkv == 0, scale > 0, 1 <= nseq <=
 *   STRD_VARLEN_MAX, at most 2^30 rows.
 *
 * The 4-bit cache.  A row of keys (or values) of one kv head is cut into groups of 32 channels.  A group is 32 codes n in 0..15,
 * channel 2 i in the low half of byte i, channel 2 i + 1 in the high half, and two bf16 numbers s, z; a code stands for
 * z + s (n - 8).  With lo, hi the smallest and the largest of the 32 and fp32 arithmetic: s = bf16((hi - lo) / 15), 0 if below
 * 2^-100; z = bf16(lo + 8 s); n = clamp(rint((x - z) / s) + 8, 0, 15), ties to even.  A value is off by s / 2 and the rounding of s and z
 * at most (|z| 2^-8 + s / 16), where s = 0 by the group's spread too, which is below 2^-96 there.  A group with a value that is not finite,
 * or whose s or z is not, reads back as NaN.
 *   k_codes, v_codes [dev] [rows, Hkv, d / 2] bytes    k_meta, v_meta [dev] [rows, Hkv, d / 32, 2] bf16 (s, z)
 * all 16-byte aligned (else STRD_EINVAL); d a multiple of 32 up to 256, Hkv up to 65535 (else STRD_EUNSUPPORTED).  They compact as
 * any other tensor.
 *   kv4_store: rows row0 .. row0 + R - 1 of the cache from k, v [dev] [R, Hkv, d] with row pitches ldk, ldv (elements); the
 *              other rows are left as they are.  R = 0 allowed.
 *   kv4_load:  k, v [dev] [R, Hkv, d] (contiguous, 32-byte aligned) from rows row0 ..; values rounded once to io.
 * rows (the cache's capacity) bounds row0 + R: STRD_EINVAL beyond it.
 *
 * attn_decode_step_kv4, attn_decode_step_weights -- strd_attn_decode_step with changed scores over the first T rows of a 4-bit or of a
 * plain cache (the newest token's own row is the last), and the attention weight that each row has gathered:
 *     w_out[j] = (w_in ? w_in[j] : 0) + 1/Hq * sum_h softmax_j(x^h)
 *   w_in, w_out [dev] [T] fp32; w_out may be w_in; w_out NULL: no weights (w_in must then be NULL).  The token's position is
 *   pos[T - 1].  d <= 256, any Hq % Hkv == 0; io is the type of q, o and of a plain cache.  Workspace [dev], 16-byte aligned:
 *   *_workspace bytes (STRD_EWORKSPACE otherwise); `weights`: whether w_out is wanted.  Deterministic.
 *
 * cache_evict -- keeps K of T rows: the first `first`, the last `last`, and of those between the K - first - last with the
 * largest weights (ties to the lowest row; NaN and negative weights as in strd_select_topk), in their old order.
 *   w [dev] [T] fp32, 16-byte aligned        idx [dev] [K] int32 output, ascending
 *   items [host] [n_items], n_items <= STRD_COMPACT_MAX - 1: tensors of T rows cut down to K rows, by the rules of strd_compact
 *   w_out [dev] [K] fp32 or NULL: the kept rows' weights     pos_out [dev] [K] int32 or NULL: pos_in of the kept rows (NULL: idx)
 *   None of the outputs may overlap an input.  first, last >= 0, first + last <= K, 1 <= K <= T <= 2^30, else STRD_EINVAL.
 *   Workspace [dev]: strd_cache_evict_workspace bytes.  Bit-exact and deterministic.
 *
 * All asynchronous on `stream`; no call allocates.
 * ------------------------------------------------------------------------- */
int strd_attn_prefill_varlen_kernel_path(int Hq, int Hkv, int d, strd_dtype io);
int strd_attn_prefill_varlen(const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, void *o,
                             const strd_seq *seqs, int nseq, int prefix, float cap, const float *slopes, const int32_t *pos, int Hq,
                             int Hkv, int d, float scale, strd_dtype io, void *stream);
typedef struct {
    void *k_codes, *k_meta, *v_codes, *v_meta;
} strd_kv4;
int strd_kv4_store(const void *k, int64_t ldk, const void *v, int64_t ldv, const strd_kv4 *cache, int rows, int row0, int R, int Hkv, int d,
                   strd_dtype io, void *stream);
int strd_kv4_load(const strd_kv4 *cache, int rows, int row0, int R, void *k, void *v, int Hkv, int d, strd_dtype io, void *stream);
size_t strd_attn_decode_step_kv4_workspace(int T, int Hq, int Hkv, int d, int weights, strd_dtype io);
int strd_attn_decode_step_kv4(const void *q, const strd_kv4 *cache, void *o, int T, int Hq, int Hkv, int d, float scale, float cap,
                              const float *slopes, const int32_t *pos, const float *w_in, float *w_out, strd_dtype io, void *ws,
                              size_t ws_bytes, void *stream);
size_t strd_attn_decode_step_weights_workspace(int T, int Hq, int Hkv, int d, int weights, strd_dtype io);
int strd_attn_decode_step_weights(const void *q, const void *k_cache, const void *v_cache, void *o, int T, int Hq, int Hkv, int d,
                                  float scale, float cap, const float *slopes, const int32_t *pos, const float *w_in, float *w_out,
                                  strd_dtype io, void *ws, size_t ws_bytes, void *stream);
size_t strd_cache_evict_workspace(int T, int K, int first, int last);
int strd_cache_evict(const float *w, int T, int K, int first, int last, const strd_compact_item *items, int n_items,
                     const int32_t *pos_in, int32_t *pos_out, int32_t *idx, float *w_out, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Going on behind a prompt: sequences in parts, many of them side by side, and several drafted tokens at a time.
 *
 * Pools.  What a Mamba-2 layer carries of a sequence from one call to the next -- the window of its convolution, the last W - 1 input rows,
 * and the state of its scan -- is a slot of a pool of nslots.  A pool is read through *_in and written through *_out; the two are one buffer
 * (updated in place) or share no memory (STRD_EINVAL for anything between; slots that no sequence has are left as they are).
 *   - Packed batches (strd_seq above; K is not looked at, N and M may be 0, and so may a sequence's rows altogether): `slots` [host] [nseq] or
 *     NULL (sequence b has slot b), in [0, nslots) and no two the same, else STRD_EINVAL; `fresh` [host] [nseq] or NULL (none): a sequence with
 *     fresh[b] != 0 begins, from zeros, whatever its slot holds.  *_in NULL: all begin.  *_out NULL: nothing is left behind.  Without either
 *     pool slots are not looked at.  A sequence without rows leaves what it came with.
 *   - Single tokens: `slots` [dev] [batch] or NULL (entry e has slot e).  An entry whose slot is outside [0, nslots), or is that of an earlier
 *     entry, is left out: its outputs are zeros, no slot is touched.  So a batch may be padded with -1, also between two replays of a graph.
 *
 * conv1d_silu_varlen -- strd_conv1d_silu for a packed batch: rows before a sequence's first are those of its window, oldest first.
 *   xbc [dev] rows of pitch ld >= Ct = Cx + 2 Cb elements; window_in, window_out [dev] [nslots, W - 1, Ct] of the io dtype; w, b, outputs as
 *   there.  1 <= W <= 4 (else STRD_EUNSUPPORTED); any Cx, Cb, ld and alignment (16 bytes of channels at a time where Cx, Cb, ld and all
 *   addresses are whole multiples of that, else one, and rows * Ct up to 2^34 then, else STRD_EUNSUPPORTED).
 * conv1d_silu_step -- the same for one token each of `batch` sequences, and the softplus of dt with it: row [dev] [batch] of pitch
 *   ld >= Ct + H, dt_out[e, h] = log(1 + exp(row[e, Ct + h] + dt_bias[h])) fp32 (H = 0: none; dt_bias [H] fp32 or NULL).  Both windows are
 *   needed if W > 1 (W = 1: nslots still bounds the slots).  batch <= 65535.
 *
 * ssd_prefill_varlen -- strd_ssd_prefill for a packed batch: x, dt, B, C, y with the rows of all sequences; S_in, S_out [dev]
 *   [nslots, H, P, n] fp32.  Workspace [dev], 16-byte aligned: strd_ssd_prefill_varlen_workspace bytes for the same descriptors
 *   (STRD_EWORKSPACE).  H % G == 0; n <= 1024, H * P * n <= 2^30 (else STRD_EUNSUPPORTED).  bf16 heads of P = 64 in groups of whole
 *   fours with n = 64 or 128 run on the bf16 matrix cores: x, B, C, y and both pools 16-byte aligned (else STRD_EINVAL), two roundings to
 *   bf16 in an output (a third of what earlier tokens left, where each of heads 4 i to 4 i + 3 decays by 2^-12 or more in every 32 tokens of a stretch),
 *   none in a state; sums of more than 2^79 in a state may leave fp32.  Small batches of them run in fp32, as does
 *   every other shape and type, those at any alignment.  Final states are fp32 sums either way.  Where sequences are cut follows from
 *   the whole batch, and with it the last bits of a result (later decays of a head show in those of its earlier outputs).  Values that are not finite
 *   stay in their own sequence.  There one of x or of a state shows in every later output of its channel, one of dt of its head, one of B of all heads of its
 *   group, and, as tokens are weighed in blocks, up to 63 tokens earlier; one of C shows in its group's outputs at its own token.
 * ssd_decode_steps -- strd_ssd_decode_step for one token each of `batch` sequences: x, y [dev] [batch, H, P], dt [batch, H],
 *   B, C [batch, G, n], states in the pool.  batch <= 65535, H * P <= 2^24, H * P * n <= 2^30 (else STRD_EUNSUPPORTED).
 *
 * rope -- rotary positions on queries and keys: with f = pos[t] * freq[i], i < rot / 2, pair i of the first `rot` channels of every head,
 *     (a, b) -> amplitude * (a cos f - b sin f, a sin f + b cos f);
 *   interleaved != 0: pair i is channels 2 i and 2 i + 1, else i and i + rot / 2; the other channels are copied.
 *   q, k, q_out, k_out [dev] rows of Hq (Hkv) heads of d channels, of pitches ldq .. ldko in elements (>= a row's own); an output may be its
 *   input, pitch included, or share no element with q, k or the other output (else STRD_EINVAL).  Hq or Hkv may be 0 (pointers then unused).
 *   pos [dev] [rows] int32, any sign (after a compaction the rows' old positions); freq [dev] [rot / 2] fp32; angles are reduced in 64 bits,
 *   so far positions lose nothing.  2 <= rot <= d, rot even, amplitude finite; d <= 1024, rows <= 2^25 (else STRD_EUNSUPPORTED).
 * rope_frequencies -- freq for rot channels: base^(-2 i / rot), and for contexts longer than the `original` positions a model was trained on,
 *   `factor` times, the slow ones divided: with r = original * freq / (2 pi) turns in the trained length, those of r <= low are divided by factor,
 *   those of r >= high stay, between the two linear in r (low = high = infinity: all are divided; factor = 1: none).  freq_out [host] [rot / 2].
 *   base > 0, factor >= 1, original > 0, 0 <= low <= high.
 *
 * attn_tree_step -- attention of m drafted tokens, the nodes of a tree, over a cache of T rows and over each other:
 *     o_i^h = sum_j softmax_j(x) v_j over all rows of the cache and the nodes j whose bit is set in mask[i]
 *   q, o [dev] [m, Hq, d]; k_cache, v_cache [dev] [T, Hkv, d]; k_new, v_new [dev] [m, Hkv, d]; mask [dev] [m] 64-bit, bit j: node j is
 *   visible (bits from m on are not looked at).  1 <= m <= 64, T >= 0 (0: no cache needed).  A node that sees nothing gets zeros; what a node does
 *   not see does not reach it, values that are not finite included.  Scores with cap and slopes as in attn_prefill_varlen above; pos [dev] [T + m]
 *   int32, the cache's rows first; NULL: a row's number, and for a node T + the number of other nodes that it sees (in a tree: its depth).
 *   d <= 256, Hkv <= 65535, m * Hq <= 2^21 (else STRD_EUNSUPPORTED), Hq % Hkv == 0, T <= 2^30.  Workspace [dev], 16-byte aligned:
 *   strd_attn_tree_step_workspace bytes (STRD_EWORKSPACE).  Deterministic.
 * tree_mask -- mask of a tree: parent[i] in [-1, i) is node i's parent (-1: it hangs on the cache's last row); node i sees itself and its
 *   ancestors.  Host-only.  STRD_EINVAL for any other parent or m outside 1..64.
 *
 * All but the two host helpers are asynchronous on `stream`; no call allocates.
 * ------------------------------------------------------------------------- */
int strd_conv1d_silu_varlen(const void *xbc, int64_t ld, const void *w, const void *b, const void *window_in, void *window_out, int nslots,
                            const int32_t *slots, const uint8_t *fresh, const strd_seq *seqs, int nseq, void *x_out, void *B_out, void *C_out,
                            int Cx, int Cb, int W, strd_dtype io, void *stream);
int strd_conv1d_silu_step(const void *row, int64_t ld, const void *w, const void *b, const float *dt_bias, const void *window_in,
                          void *window_out, int nslots, const int32_t *slots, void *x_out, void *B_out, void *C_out, float *dt_out, int batch,
                          int Cx, int Cb, int H, int W, strd_dtype io, void *stream);
size_t strd_ssd_prefill_varlen_workspace(const strd_seq *seqs, int nseq, int H, int P, int G, int n, strd_dtype io);
int strd_ssd_prefill_varlen(const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D, const float *S_in,
                            float *S_out, int nslots, const int32_t *slots, const uint8_t *fresh, const strd_seq *seqs, int nseq, void *y, int H,
                            int P, int G, int n, strd_dtype io, void *ws, size_t ws_bytes, void *stream);
int strd_ssd_decode_steps(const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D, const float *S_in,
                          float *S_out, int nslots, const int32_t *slots, void *y, int batch, int H, int P, int G, int n, strd_dtype io,
                          void *stream);
int strd_rope(const void *q, int64_t ldq, void *q_out, int64_t ldqo, int Hq, const void *k, int64_t ldk, void *k_out, int64_t ldko, int Hkv,
              const int32_t *pos, const float *freq, int rows, int d, int rot, int interleaved, float amplitude, strd_dtype io, void *stream);
int strd_rope_frequencies(int rot, double base, double factor, double original, double low, double high, float *freq_out);
size_t strd_attn_tree_step_workspace(int T, int m, int Hq, int Hkv, int d, strd_dtype io);
int strd_attn_tree_step(const void *q, const void *k_cache, const void *v_cache, const void *k_new, const void *v_new, const uint64_t *mask,
                        void *o, int T, int m, int Hq, int Hkv, int d, float scale, float cap, const float *slopes, const int32_t *pos,
                        strd_dtype io, void *ws, size_t ws_bytes, void *stream);
int strd_tree_mask(const int32_t *parent, int m, uint64_t *mask_out);

/* ---------------------------------------------------------------------------
 * schedule_budgets -- per-layer token budgets of a retention schedule (Sec. 3.2
 * and App. "Reduction Schedule Configurations").  alpha_l is relative to the
 * original count N0; budgets never grow with depth and never fall below
 * min(K_min, current count):
 *     K_l = min(K_{l-1}, max(floor(alpha_l * N0), min(K_min, K_{l-1}))),  K_{-1} = N0
 *   alpha [host] [L] doubles in [0, 1]      K_out [host] [L] int32
 * Host-only helper; touches no device.
 * ------------------------------------------------------------------------- */
int strd_schedule_budgets(const double *alpha, int L, int N0, int K_min, int32_t *K_out);

/* Sigmoid retention schedule (App. "Sigmoid Schedule"), layers l = 0..L-1:
 *     alpha_l = a_end + (a_start - a_end) * sigmoid(k * (x0 - l / L))
 *   alpha_out [host] [L] doubles */
int strd_schedule_sigmoid(int L, double a_start, double a_end, double k, double x0,
                          double *alpha_out);

/* Step-decay retention schedule (App. "Step Decay Schedule"): alpha_l = alpha[r] for the layers
 * lo[r]..hi[r] (inclusive, 0-indexed; later ranges win), 1.0 elsewhere.
 *   lo, hi [host] [nranges] ints   alpha [host] [nranges] doubles in [0,1]   alpha_out [host] [L] */
int strd_schedule_step_decay(const int *lo, const int *hi, const double *alpha, int nranges, int L,
                             double *alpha_out);

/* Layer types of the 62-layer hybrid the schedules of the paper are written for (App. "Reduction
 * Schedule Configurations"): attention at layers 7, 16, 25, 34, 43, 52; the other 56 layers
 * alternate Mamba-2, MLP starting with Mamba-2 (28 + 28; the paper gives the counts, not the order).
 *   type_out [host] [L] int32 of STRD_LAYER_*; a shorter or longer L follows the same rule. */
enum { STRD_LAYER_MAMBA = 0, STRD_LAYER_MLP = 1, STRD_LAYER_ATTN = 2, STRD_HYBRID_LAYERS = 62 };
int strd_hybrid_layout(int L, int32_t *type_out);

/* The named schedules of the same table, as retention ratios for the STRD_HYBRID_LAYERS layers:
 * "attn_only_1st_attn", "all_attn_25", "all_attn_35", "all_attn_50", "first_mamba",
 * "second_mamba" (ranges as printed), "sigmoid_25", "sigmoid_35", "sigmoid_50" (k = 20, x0 = 0.11 /
 * 0.24 / 0.41, 1.0 -> 0.125), "all_attn_1m", "all_attn_2m" (the table only says 0.32 -> 0.15 over
 * the 6 attention layers plus 1 or 2 Mamba layers before each: taken as a linear fall over the
 * reducing layers up to layer 33, held afterwards).  Unknown name: STRD_EINVAL.
 *   alpha_out [host] [STRD_HYBRID_LAYERS] doubles */
int strd_schedule_named(const char *name, double *alpha_out);

#ifdef __cplusplus
}
#endif
#endif /* STRD_H */
