/*
 * dn.h -- C ABI of the deferred-normalization library (libdn.so), gfx950.
 *
 * Method: "LLM Inference Acceleration via Efficient Operation Fusion"
 * (Salmani & Soloveychik, arXiv 2502.17728).  A LayerNorm or a Softmax that
 * feeds a matrix product is split into an element-wise part, which becomes
 * the product's operand, and a per-row collective part (the LayerNorm
 * mean/variance, the softmax denominator), which is reduced concurrently and
 * applied once after the product (Sec. II, Fig. 1; Eq. (5) and Eq. (8)).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Tensor pointers are DEVICE pointers (hipMalloc'd or equivalent), row-major
 *   and contiguous, 16-byte aligned.  The caller owns all memory; the library
 *   allocates nothing.  Two library-owned device arrays exist on each GPU the
 *   library runs on, held until the process ends: the 1 MiB mailbox in which
 *   the workgroups of one LayerNorm/RMSNorm product exchange their shares of
 *   the row moments (every entry stamped with its call's number, so no call
 *   ever uses another's; see ln_linear_deferred), and the partials array of
 *   attention_decode_deferred_noalloc.  No other state outlives a call.
 * - Every call validates its arguments on the host BEFORE any HIP call; an
 *   invalid call returns a status and enqueues nothing.  A valid call only
 *   enqueues kernels on `stream` (NULL = the default stream) and returns; it
 *   never synchronizes.  Buffers must stay alive until that work completes.
 *   Calls on different streams are independent (reentrant).
 * - Element types: DN_F32 (IEEE fp32) or DN_BF16 (bfloat16).  All accumulation
 *   is fp32; outputs are rounded once, to nearest even, to the input type.
 * - NaN/Inf inputs are not errors: they propagate as in the plain definition.
 * - Sizes are int64 element counts; K and N (and d) must be multiples of 8.
 * - Output ranges must not overlap input ranges (checked: DN_ERR_INVALID_ARG).
 */
#ifndef DN_H
#define DN_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DN_API __attribute__((visibility("default")))

typedef enum { DN_F32 = 0, DN_BF16 = 1 } dn_dtype;

typedef enum {
    DN_OK = 0,
    DN_ERR_INVALID_ARG = 1, /* NULL pointer, size < 1, bad eps, overlap, bad descriptor   */
    DN_ERR_UNSUPPORTED = 2, /* valid request outside what the kernels implement            */
    DN_ERR_MISALIGNED = 3,  /* a tensor pointer is not 16-byte aligned                     */
    DN_ERR_HIP = 4          /* the HIP runtime reported an error when launching            */
} dn_status;

/* Human-readable name of a status code (static string; never NULL). */
DN_API const char* dn_status_string(int status);

/* Library version, (major << 16) | minor. */
DN_API int dn_version(void);

/* ======================================================================= */
/* LayerNorm -> Linear, deferred (Sec. II-A, Eq. (1), (2), (4), (5))        */
/* ======================================================================= */

/*
 * Static weights prepared once (the paper computes the static factors of
 * Eq. (5) "at compile time", Sec. II-A; here once per weight set, off the
 * per-token path).  From W[K][N] (the paper's F, n x m), gamma[K], beta[K]
 * and an optional bias[N], ln_linear_prepare writes into `packed`:
 *   Wt'[N][K] = (Diag(gamma) W)^T  rounded once to `dtype` (K contiguous),
 *   c[N]      = sum_k W'[k][n]     over the ROUNDED W' (fp32),
 *   b[N]      = sum_k beta[k] W[k][n] + bias[n]     (fp32; beta F of Eq. (5)).
 * `packed` must be ln_linear_packed_bytes(K, N, dtype) bytes, 256-byte
 * aligned, device memory; `*w_out` is filled on the host and is what
 * ln_linear_deferred takes.  beta and bias may be NULL (treated as zero).
 * Layout of W'^T in `packed` (version 2): 16-row x 64-byte fragment chunks
 * (16 output features x 32 bf16 or 16 fp32 of K), in chunk order
 * [ceil(N/16)][ceil(K/kchunk)][64 lanes][16 B], zero padded; lane l of a
 * chunk holds feature 16*nb + (l & 15) at K offset kchunk*kc + (l >> 4)*(16 B).
 */
typedef struct {
    int64_t K, N;           /* normalized dim, output features                */
    int32_t dtype;          /* dn_dtype of W' and of x/out                    */
    int32_t layout_version; /* DN_LN_LAYOUT_VERSION when produced by prepare   */
    void* packed;           /* device buffer holding Wt', c, b                */
} ln_linear_weights;

#define DN_LN_LAYOUT_VERSION 2

/* Bytes of the packed buffer for (K, N, dtype); 0 if the request is invalid. */
DN_API size_t ln_linear_packed_bytes(int64_t K, int64_t N, int dtype);

DN_API dn_status ln_linear_prepare(const void* W, const void* gamma, const void* beta,
                            const void* bias, int64_t K, int64_t N, int dtype,
                            void* packed, size_t packed_bytes,
                            ln_linear_weights* w_out, hipStream_t stream);

/*
 * out[M][N] = LayerNorm(x[M][K]) . W + bias, computed the deferred way:
 * the MFMA product acc = x . W' runs on the un-normalized x while the row
 * statistics (sum x, sum x^2) are reduced in the same workgroup, and the
 * epilogue applies  out = rstd * (acc - mean * c) + b  once (Eq. (5) with the
 * centering (I - E/n) applied as  x(I - E/n)W' = xW' - mean 1 W').
 * mean and the biased variance follow Eq. (1); rstd = 1/sqrt(var + eps) as
 * in Eq. (2).  eps must be finite and >= 0.  x and out have w->dtype.
 * On the large-tile kernels (bf16, K % 64 == 0, more than 128 rows unless the
 * few-row kernel is clearly the faster) the
 * workgroups that share a 256-row block split the reduction of its moments
 * and exchange the sums through the library's mailbox; a workgroup that does
 * not find a peer's sums within 200 us (a peer not resident on a busy GPU)
 * reduces all its rows itself, so the result never depends on scheduling.
 * (DN_MOMENT_WAIT_TICKS in the environment overrides the wait, in 10 ns
 * ticks; 0 makes every workgroup reduce its rows itself.)  A launch recorded
 * under stream capture (a HIP graph) uses no mailbox: each workgroup reduces
 * the moments of its rows alongside its first tile, so every replay of the
 * graph normalizes with its own inputs' statistics.  A row holding
 * NaN or +-inf gives an all-NaN output row; with eps = 0 a row whose fp32
 * one-pass variance is exactly 0 (a constant row whose squares sum exactly)
 * gives NaN, as (x - mean) / 0 does.  |x| >= 2^64 (fp32 overflow of x^2) is
 * outside the supported range.
 */
DN_API dn_status ln_linear_deferred(const void* x, const ln_linear_weights* w, int64_t M,
                             float eps, void* out, hipStream_t stream);

/*
 * out[M][N] = RMSNorm(x[M][K]) . W + bias (Sec. II-A, RMSNorm in Llama
 * models, Eq. (6)), the deferred way: acc = x . W' on the MFMA with the row
 * sum of squares reduced concurrently, then  out = rstd * acc + b  with
 * rstd = 1/sqrt(sum_k x^2 / K + eps).  Eq. (6) subtracts no mean, so c is not
 * used.  Eq. (6) prints no eps: eps is an argument inside the root, finite
 * and >= 0, and eps = 0 is the printed form (an all-zero row then gives NaN).
 * w comes from ln_linear_prepare with the RMSNorm gamma; Eq. (6) has no
 * shift, so pass beta = NULL there (a non-NULL beta adds beta W to every
 * row, as it does for LayerNorm).  Same argument rules, layout, ownership
 * and status codes as ln_linear_deferred.
 */
DN_API dn_status rms_linear_deferred(const void* x, const ln_linear_weights* w, int64_t M,
                              float eps, void* out, hipStream_t stream);

/*
 * Post-LN placement (Sec. II-A: the residual branch taken right after the
 * normalization instead of before it).  There the normalized rows y are needed
 * twice -- as the input of the next linear layer and as the residual -- so the
 * call returns both: out[M][N] = y . W + bias the deferred way (exactly as
 * ln_linear_deferred / rms_linear_deferred, the product never waiting for the
 * statistics), and y[M][K] = (x - mean) rstd gamma + beta (RMS: x rstd gamma)
 * applied afterwards from the statistics the product's kernel reduced, which
 * it exports to stats[2 M] (fp32 (mean, rstd) pairs; RMS: mean = 0).  gamma
 * (and beta, nullable, LayerNorm only) are the [K] vectors that were folded
 * into w, in w->dtype.  stats and y: caller-owned device memory, 16-byte
 * aligned, overlapping no other argument.  Status codes as ln_linear_deferred;
 * DN_ERR_UNSUPPORTED also when y is too large for one launch.
 */
DN_API dn_status ln_linear_deferred_post(const void* x, const ln_linear_weights* w, int64_t M, float eps,
                                  const void* gamma, const void* beta, float* stats, void* y,
                                  void* out, hipStream_t stream);

DN_API dn_status rms_linear_deferred_post(const void* x, const ln_linear_weights* w, int64_t M, float eps,
                                   const void* gamma, float* stats, void* y, void* out,
                                   hipStream_t stream);

/* ----------------------------------------------------------------------- */
/* Ablations of the LayerNorm -> Linear fusion                              */
/* ----------------------------------------------------------------------- */

/*
 * Eq. (5) taken literally: the centering (I - E/n) of Eq. (3) folded into
 * the static weight, W'' = (I - E/n) Diag(gamma) W, i.e. gamma_k W[k][n]
 * minus its column mean (fp64, unrounded), rounded once to dtype; c is set
 * to 0 so ln_linear_deferred computes out = rstd * (x . W'') + b, the
 * epilogue of Eq. (5) with no mean term.  Same arguments, layout and status
 * codes as ln_linear_prepare; the result is used with ln_linear_deferred.
 * Equal to the mean * c epilogue in exact arithmetic; in floating point the
 * rounded W'' columns no longer sum to exactly 0, so rows with a large
 * |mean| / std lose about |mean| / std * 2^-9 of relative accuracy (bf16).
 */
DN_API dn_status ln_linear_prepare_centered(const void* W, const void* gamma, const void* beta,
                                     const void* bias, int64_t K, int64_t N, int dtype,
                                     void* packed, size_t packed_bytes,
                                     ln_linear_weights* w_out, hipStream_t stream);

/*
 * Serial (not concurrent) statistics: a pre-pass kernel computes each row's
 * mean and 1/sqrt(var + eps) (two passes over the row, Eq. (1)-(2)) into
 * stats[2 M] (fp32 pairs; caller-owned device memory, 16-byte aligned, not
 * overlapping x, out or the weights), then the product runs with the same
 * deferred epilogue, reading them instead of reducing the moments
 * concurrently.  It isolates what concurrency buys over a stats pre-pass.
 * K must also fit the row kernel (<= 16384 bf16 / 8192 fp32) else
 * DN_ERR_UNSUPPORTED.  Otherwise as ln_linear_deferred.
 */
DN_API dn_status ln_linear_serial(const void* x, const ln_linear_weights* w, int64_t M, float eps,
                           float* stats, void* out, hipStream_t stream);

/*
 * Fused without deferral (ablation of Eq. (5)): the same statistics pre-pass
 * as ln_linear_serial into stats[2 M], then one kernel that normalizes each x
 * fragment as it is loaded, xh = (x - mean) / sqrt(var + eps) rounded to the
 * GEMM dtype, and runs xh . W' + b (W' = Diag(gamma) W and b = beta W + bias
 * from ln_linear_prepare, so this is y F of Eq. (4) with y formed in
 * registers).  The normalization sits on the product's input path instead of
 * after it, which isolates what deferral buys over plain fusion.  bf16 only,
 * and only where the 256 x 256 kernel applies (M > 128, K % 64 == 0,
 * K and N < 2^22; it runs there even when ln_linear_deferred would take
 * 128 x 128 tiles); other shapes give DN_ERR_UNSUPPORTED.  Otherwise as
 * ln_linear_serial.
 */
DN_API dn_status ln_linear_norm_on_load(const void* x, const ln_linear_weights* w, int64_t M, float eps,
                                 float* stats, void* out, hipStream_t stream);

/* ======================================================================= */
/* RMSNorm -> gated MLP input (SwiGLU), deferred                            */
/* ======================================================================= */

/*
 * The Llama MLP input stage (Sec. II-A, subsubsection on RMSNorm in Llama
 * models, which fuses the up-projection and gating): y = RMSNorm(x) (Eq. (6)),
 * h = SiLU(y Wg) * (y Wu) element-wise, SiLU(z) = z / (1 + e^-z).
 * Deferred: both products run on the MFMA over the un-normalized x, each x
 * fragment feeding the gate and the up columns, with sum x^2 reduced
 * concurrently; the epilogue applies rstd to both products (before the SiLU,
 * which is not homogeneous, so the deferral ends there) and writes h once.
 *
 * swiglu_prepare folds gamma into both [K][N] weights and packs them into one
 * buffer of swiglu_packed_bytes(K, N, dtype) bytes (256-byte aligned device
 * memory): Wg' and Wu' in the fragment-chunk layout of ln_linear_prepare,
 * interleaved by 16-feature blocks (block 2j = gate features 16j.., block
 * 2j+1 = up features 16j..), with c and b (zero: no shift, no bias) in the
 * same interleaved order.  *w_out gets N (the output features) and
 * layout_version DN_SWIGLU_LAYOUT_VERSION; only rms_swiglu_deferred takes it.
 * rms_swiglu_deferred writes h[M][N] in w->dtype; eps as for
 * rms_linear_deferred.  Status codes and alignment rules as for the
 * LayerNorm -> Linear calls.
 */
#define DN_SWIGLU_LAYOUT_VERSION 0x102

DN_API size_t swiglu_packed_bytes(int64_t K, int64_t N, int dtype);

DN_API dn_status swiglu_prepare(const void* W_gate, const void* W_up, const void* gamma,
                         int64_t K, int64_t N, int dtype, void* packed, size_t packed_bytes,
                         ln_linear_weights* w_out, hipStream_t stream);

DN_API dn_status rms_swiglu_deferred(const void* x, const ln_linear_weights* w, int64_t M,
                              float eps, void* h, hipStream_t stream);

/* ======================================================================= */
/* Softmax -> P.V, deferred (Sec. II-B, Eq. (7), (8) and its footnote)      */
/* ======================================================================= */

/*
 * out[BH][Lq][d] = softmax(S[BH][Lq][Lk]) . V[BH][Lk][d] per head, computed
 * the deferred way: the MFMA consumes the un-normalized numerators
 * exp(s - m) (rounded to bf16), the row max m (footnote of Eq. (7)) is kept
 * online per key tile, the row sum l is accumulated concurrently, and the
 * epilogue divides once: out = acc / l (Eq. (8)).
 * causal = 1 keeps key j for query i iff j <= i (requires Lq == Lk); the
 * stored values at j > i are ignored (tiles wholly above the diagonal are
 * never read; inside diagonal tiles they are masked).  causal = 0 uses every
 * key.  A row whose kept scores are all -inf gives NaN.  dtype must be
 * DN_BF16; d must be 64 or 128; Lk a multiple of 8, Lq * Lk <= 2^31 and
 * Lk * d * 2 < 2^32 (else DN_ERR_UNSUPPORTED).
 */
DN_API dn_status softmax_pv_deferred(const void* S, const void* V, int64_t BH, int64_t Lq,
                              int64_t Lk, int64_t d, int causal, int dtype, void* out,
                              hipStream_t stream);

/*
 * The same deferred Softmax -> P.V with the scores formed in the kernel:
 * out[BH][Lq][d] = softmax(scale * Q K^T) . V per head, Q[BH][Lq][d],
 * K, V[BH][Lk][d] (Sec. II-B carried one operation earlier, so that S never
 * exists in memory: Eq. (8)'s numerators exp(s - m) come straight from the
 * Q.K^T product on the matrix core, the row max is kept online, the row sum
 * reduced alongside, and out = acc / l once).  causal = 1 keeps key j for
 * query i iff j <= i (Lq == Lk).  scale must be finite and > 0.  dtype must
 * be DN_BF16; d 64 or 128; Lq * d * 2 and Lk * d * 2 < 2^31 per head (else
 * DN_ERR_UNSUPPORTED).  A row whose scores are all -inf cannot occur (finite
 * inputs); NaN inputs propagate.
 */
DN_API dn_status attention_deferred(const void* Q, const void* K, const void* V, int64_t BH,
                             int64_t Lq, int64_t Lk, int64_t d, int causal, float scale,
                             int dtype, void* out, hipStream_t stream);

/*
 * attention_deferred with grouped-query attention (as in the Llama 3 models
 * the paper evaluates): K, V hold BH_kv heads [BH_kv][Lk][d], and Q, out
 * hold BH_kv * group query heads [BH_kv * group][Lq][d]; query head h reads
 * key/value head h / group (the group's query heads are consecutive).  Each
 * query head is computed exactly as by attention_deferred.  group >= 1;
 * other rules and status codes as attention_deferred.
 */
DN_API dn_status attention_gqa_deferred(const void* Q, const void* K, const void* V, int64_t BH_kv,
                                 int64_t group, int64_t Lq, int64_t Lk, int64_t d, int causal,
                                 float scale, int dtype, void* out, hipStream_t stream);

/*
 * Decode-shaped attention: Lq <= 16 query rows per head against all Lk keys
 * (the key/value cache holds exactly the visible keys, so no mask).  The keys
 * of all heads are dealt in order to at most one resident round of workgroups,
 * the same number of 128-key units to each but the last; where a head's keys went to several, each leaves its un-normalized partial sums
 * (acc, l and the reference max m, fp32) in `workspace`, and one merge kernel
 * combines them, m = max m_g, out = sum 2^(m_g - m) acc_g /
 * sum 2^(m_g - m) l_g -- the deferred division of Eq. (8) once more, across
 * key ranges.  workspace: caller-owned device memory of
 * attention_decode_workspace_bytes(BH, Lq, Lk, d) bytes, 16-byte aligned, not
 * overlapping the other arguments; its contents are scratch.  Q[BH][Lq][d],
 * K, V[BH][Lk][d], out[BH][Lq][d]; other rules as attention_deferred
 * (DN_ERR_UNSUPPORTED for Lq > 16).  Grouped-query attention (g query heads
 * sharing each key/value head, the g heads consecutive): pass Q and out as
 * [BH][g * Lq][d] -- the same memory as [BH * g][Lq][d] -- with Lq := g * Lq
 * (<= 16), so each key/value tile read from HBM serves all g heads at once.
 * Where every workgroup has whole heads one pass writes out directly (the
 * workspace is then not touched).  A workspace smaller than
 * attention_decode_workspace_bytes asks for is taken if it holds the partials
 * of every head cut into equally many ranges, one workgroup each (BH * n * Lq
 * * (d + 4) floats, n = about 256 / BH at d = 128, 512 / BH at d = 64); the
 * keys are then cut that way.  attention_decode_workspace_bytes
 * returns 0 for an invalid request.
 */
DN_API size_t attention_decode_workspace_bytes(int64_t BH, int64_t Lq, int64_t Lk, int64_t d);

DN_API dn_status attention_decode_deferred(const void* Q, const void* K, const void* V, int64_t BH,
                                    int64_t Lq, int64_t Lk, int64_t d, float scale, int dtype,
                                    void* workspace, size_t workspace_bytes, void* out,
                                    hipStream_t stream);

/*
 * For callers that cannot allocate (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): attention_decode_deferred
 * with no workspace argument.  The key-range partials go to a 12 MiB device
 * array that the library holds on each GPU it runs on until the process ends;
 * no call allocates or frees memory.  Heads that fill the chip by themselves
 * (256 at d = 128, 512 at d = 64), or at most 128 keys, leave no partials: one
 * workgroup then reads each head whole and the array is not touched.  Every
 * request attention_decode_deferred accepts fits it (the partials stay below
 * 4.25 MiB at d = 64 and 4.125 MiB at d = 128); a request that would not gives
 * DN_ERR_UNSUPPORTED.  The array keeps the last call's partials, which every
 * call overwrites before it reads them; calls that leave partials and overlap on one GPU (concurrent streams)
 * share it and race.  Arguments, layout, grouped-query use and status codes as
 * attention_decode_deferred; the output is bitwise the same as with a workspace
 * of attention_decode_workspace_bytes.
 */
DN_API dn_status attention_decode_deferred_noalloc(const void* Q, const void* K, const void* V, int64_t BH,
                                            int64_t Lq, int64_t Lk, int64_t d, float scale, int dtype,
                                            void* out, hipStream_t stream);

/* ======================================================================= */
/* Rotary positions                                                         */
/* ======================================================================= */

/*
 * Rotary positions turn pairs of dimensions of a query or key head by an angle
 * proportional to the token's position, y_p = x_p cos - x_q sin and
 * y_q = x_q cos + x_p sin, where (p, q) = (2i, 2i + 1) (interleaved) or
 * (i, i + rot/2) (halves), i < rot/2; dimensions from rot on stay as they are.
 *
 * rotary_table fills table[positions][rot/2][2] (fp32, caller-owned, 16-byte
 * aligned) with amplitude * cos and amplitude * sin of n * inv_freq[i] for
 * n < positions, evaluated in fp64 and rounded once; once per model, off the
 * per-token path.  inv_freq[rot/2] are fp64 device values, 8-byte aligned: plain
 * frequencies base^(-2i/rot), or any that were scaled for long contexts.
 * amplitude is finite (1 where the scaling asks for none).
 *
 * rotary_apply turns x[T][H][d] (DN_F32 or DN_BF16; x_stride elements between
 * tokens, heads contiguous) by table row positions[t] into out (out_stride
 * likewise).  inverse = 1 is the transpose: the gradient with respect to x from
 * the gradient with respect to out, and with amplitude 1 the turn back (else
 * amplitude^2 times it).  out may be x itself with equal strides; other overlaps
 * are refused.  rot is a multiple of 16 up to d, d a
 * multiple of 16, strides multiples of 16 bytes and at least H * d.  A position
 * outside the table gives NaN in the turned dimensions.  positions: int32, 4-byte
 * aligned.  Arithmetic is fp32, each result rounded once.
 */
DN_API dn_status rotary_table(const double* inv_freq, int64_t rot, int64_t positions, double amplitude, float* table,
                       hipStream_t stream);

DN_API dn_status rotary_apply(const void* x, int64_t x_stride, const int32_t* positions, const float* table,
                       int64_t table_rows, int64_t T, int64_t H, int64_t d, int64_t rot, int interleaved, int inverse,
                       int dtype, void* out, int64_t out_stride, hipStream_t stream);

/* ======================================================================= */
/* Paged key/value cache                                                    */
/* ======================================================================= */

/*
 * A cache is one caller-owned device buffer of `pages` pages of DN_KV_PAGE
 * tokens for `heads` key/value heads of d = 64 or 128 dimensions; which pages
 * hold which sequence is the caller's.  Slot s is token s % 64 of page s / 64.
 * Formats: DN_KV_BF16 holds bfloat16; DN_KV_FP8 holds OCP e4m3 codes with one
 * fp32 scale per token and head, x = code * scale, scale = max(max |x| / 448,
 * 2^-120), the code rounded to nearest even.  Either way a row (K or V of one
 * token and head) that holds a NaN or an infinity (in DN_KV_BF16 also a turned
 * key that would round to one) is held as all NaN: codes 0, scale NaN (the scale
 * is 1 elsewhere in DN_KV_BF16).
 * Layout (version 1) of `data`: [pages][heads][block], block = K codes, V codes,
 * 64 K scales, 64 V scales.  With E = 8 (bf16) or 16 (fp8) elements in 16 bytes,
 * token 4E u + E a + 8 j + 4 t + i, dimension 4E c + E g + r of K lies at byte
 * (((((E/8 u + j) 2 + t) d/(4E) + c) 4 + g) 16 + 4 a + i) 16 + r 16/E, and token
 * 4E u + E g + r, dimension 16 n + w of V at byte
 * (((u d/16 + n) 4 + g) 16 + w) 16 + r 16/E.
 * kv_cache_describe checks the sizes (pages * 64 < 2^31), the buffer's
 * kv_cache_bytes and its 256-byte alignment and fills *out on the host; it
 * touches no memory, and no entry point reads slots that were never written
 * except as masked keys, so the buffer needs no clearing.
 */
#define DN_KV_PAGE 64
#define DN_KV_LAYOUT_VERSION 1
typedef enum { DN_KV_BF16 = 1, DN_KV_FP8 = 2 } dn_kv_format;

typedef struct {
    int64_t pages, heads, d;
    int32_t format;         /* dn_kv_format                          */
    int32_t layout_version; /* DN_KV_LAYOUT_VERSION when described   */
    void* data;
} kv_cache;

/* Bytes of the buffer; 0 if the request is invalid. */
DN_API size_t kv_cache_bytes(int64_t pages, int64_t heads, int64_t d, int format);

DN_API dn_status kv_cache_describe(void* data, size_t bytes, int64_t pages, int64_t heads, int64_t d, int format,
                            kv_cache* out);

/*
 * Takes the rows of a QKV projection, qkv[T][q_heads + 2 heads][d] (DN_BF16;
 * `stride` elements between tokens, a multiple of 8): turns the query heads into
 * q_out[T][q_heads][d] and the key heads as rotary_apply does, and puts keys and
 * values into the cache at slots[t] (quantised from the turned fp32 values, one
 * rounding).  q_heads is a multiple of the cache's heads, or 0 (q_out then NULL):
 * rows of keys and values alone.  rot = 0 turns nothing (positions and table
 * unused).  A slot outside the cache (-1 by convention) is not written: padding.
 * A slot named twice in a call is left with either token, whole or mixed.
 */
DN_API dn_status kv_cache_append(const kv_cache* cache, const void* qkv, int64_t stride, const int32_t* slots,
                          const int32_t* positions, const float* table, int64_t table_rows, int64_t rot,
                          int interleaved, int64_t T, int64_t q_heads, int dtype, void* q_out, hipStream_t stream);

/* K, V [T][heads][d] (DN_BF16): the values held at slots[t], zeros for a slot outside the cache. */
DN_API dn_status kv_cache_read(const kv_cache* cache, const int32_t* slots, int64_t T, int dtype, void* K, void* V,
                        hipStream_t stream);

/*
 * Deferred attention of B ragged sequences over the cache.  Sequence b's new
 * tokens are rows q_start[b] .. q_start[b + 1] - 1 of Q[T][q_heads][d] (q_start
 * ascending from 0 to T; a sequence may have none); its kv_len[b] cached tokens,
 * the new ones last, lie in pages block_table[b][0], [1], .. (table_width entries
 * a row).  Query i of n sees keys 0 .. kv_len[b] - n + i: one new token is a decode
 * step, many are a prefill chunk, and both may meet in one call.  One tile size,
 * by the mean of the new tokens, serves the whole call: a long chunk beside single
 * tokens runs faster as two calls, each over its own sequences.  Query head h
 * reads key/value head h / (q_heads / heads).  out[T][q_heads][d]; Q has q_stride
 * elements between tokens (a multiple of 8), scale finite and > 0, dtype DN_BF16.
 * q_start, kv_len and block_table are int32 device arrays, read on the device, so a
 * recorded graph replays with their new contents.  Rows of Q and out past
 * q_start[B] are neither read nor written.  A query that sees no key gives
 * zeros; one whose scores are all -inf gives NaN.  Sums over values are fp32 and
 * divided last, with numerators up to 2^8: the largest value times the number of
 * keys is to stay below 2^119.  Entries outside the cache, the table or [0, T] are
 * kept inside (page 0, the table's width, T): memory stays safe, the rows
 * concerned are unspecified.
 * workspace: caller-owned, 256-byte aligned, attention_cache_workspace_bytes
 * (with prefix_len = 0), scratch of one call at a time: the kernels keep lists in
 * it that they follow.  Where one workgroup reads a tile's keys whole
 * one launch writes out; else partial sums go through the workspace as in
 * attention_decode_deferred.
 *
 * attention_shared_prefix_deferred: the same where all B sequences share
 * prefix_len >= 1 leading tokens in the pages prefix_table[0], [1], ..; block_table
 * and kv_len then count each sequence's own tokens, and every query also sees the
 * whole prefix.  The prefix is read once per key/value head for the queries of all
 * sequences together, and its partial sums are merged with those over the
 * sequences' own keys.
 * attention_cache_workspace_bytes returns 0 for an invalid request.
 */
DN_API size_t attention_cache_workspace_bytes(int64_t T, int64_t B, int64_t q_heads, int64_t heads, int64_t d,
                                       int64_t table_width, int64_t prefix_len);

DN_API dn_status attention_cache_deferred(const void* Q, int64_t q_stride, int64_t T, int64_t q_heads,
                                   const kv_cache* cache, const int32_t* block_table, int64_t table_width,
                                   const int32_t* q_start, const int32_t* kv_len, int64_t B, float scale, int dtype,
                                   void* workspace, size_t workspace_bytes, void* out, hipStream_t stream);

DN_API dn_status attention_shared_prefix_deferred(const void* Q, int64_t q_stride, int64_t T, int64_t q_heads,
                                           const kv_cache* cache, const int32_t* prefix_table, int64_t prefix_len,
                                           const int32_t* block_table, int64_t table_width, const int32_t* q_start,
                                           const int32_t* kv_len, int64_t B, float scale, int dtype, void* workspace,
                                           size_t workspace_bytes, void* out, hipStream_t stream);

/* ======================================================================= */
/* Unfused comparators: the conventional sub-graph of Fig. 1(a)             */
/* ======================================================================= */

/* y[M][K] = (x - mean)/sqrt(var + eps) * gamma + beta, Eq. (1)-(2).  beta may be NULL. */
DN_API dn_status layernorm(const void* x, const void* gamma, const void* beta, int64_t M,
                    int64_t K, float eps, int dtype, void* y, hipStream_t stream);

/* y[M][K] = x / sqrt(sum_k x^2 / K + eps) * gamma, Eq. (6) (eps as for
   rms_linear_deferred).  Same rules and status codes as layernorm. */
DN_API dn_status rmsnorm(const void* x, const void* gamma, int64_t M, int64_t K, float eps,
                  int dtype, void* y, hipStream_t stream);

/* h[i] = SiLU(g[i]) * u[i] for count elements (count a multiple of 8); the
   conventional last step of the gated MLP input.  h must not overlap g or u. */
DN_API dn_status silu_mul(const void* g, const void* u, int64_t count, int dtype, void* h,
                   hipStream_t stream);

/*
 * P[BH][Lq][Lk] = softmax of each row of S (Eq. (7) with the max subtraction).
 * causal = 0: every key.  causal = 1: keys j <= i, and P = 0 for j > i (dense,
 * the conventional output).  causal = 2: keys j <= i, and only the aligned
 * 8-element groups that contain some j <= i are written (entries j > i inside
 * such a group are 0; the rest of the upper triangle is left untouched); this
 * is the input gemm(a_causal = 1) expects.  causal != 0 requires Lq == Lk.
 * dtype must be DN_BF16; Lk <= 16384.
 */
DN_API dn_status softmax(const void* S, int64_t BH, int64_t Lq, int64_t Lk, int causal,
                  int dtype, void* P, hipStream_t stream);

/*
 * C[batch][M][N] = A[batch][M][K] . B (+ bias[N]), fp32 accumulation.
 * b_layout = 0: B is [batch][K][N] (row-major, N contiguous).
 * b_layout = 1: B is given transposed, [batch][N][K] (K contiguous).
 * b_layout = 2: B is the packed buffer ln_linear_prepare wrote for (K, N,
 *               dtype) -- with gamma = 1 it holds W itself; its c and b parts
 *               are ignored.  batch must be 1.  This is the weight layout and
 *               main loop ln_linear_deferred uses, so the two paths differ
 *               only by the fusion.
 * a_causal = 1: A is lower-triangular by contract (A[i][j] treated as 0 for
 *               j > i, never read beyond the diagonal tile); requires M == K,
 *               bf16 and b_layout 0 or 1.
 * bias may be NULL.
 */
DN_API dn_status gemm(const void* A, const void* B, const void* bias, int64_t batch, int64_t M,
               int64_t K, int64_t N, int b_layout, int a_causal, int dtype, void* C,
               hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* DN_H */
