/*
 * chameleon.h -- C ABI of the MI355X (gfx950) hot path of Chameleon's per-tensor,
 * format-adaptive post-training quantization (arXiv 2609.33496, "Chameleon: Dynamic Format
 * Adapter for Efficient Diffusion"): the quantized linear layer of a denoiser.
 *
 *   cham_select_weight_formats  offline per-output-channel weight-format search + packing
 *                               (Sec. 4.5, Eq. weight-argmax; palettes of Sec. 4.2)
 *   cham_act_stats_accumulate   calibration power sums and range per (layer, bucket)
 *                               (Sec. 4.4; App. A.7, Alg. 1 first loop)
 *   cham_build_act_lut          kurtosis + SNR routing + ScaleZP -> format/scale/zero LUT
 *                               (Sec. 4.3; App. A.7, Alg. 1 second loop)
 *   cham_quantize_act           activation quantization to the LUT's format, static
 *                               (UNet path, Alg. 2) or dynamic per-tensor (DiT path, Alg. 3)
 *   cham_mixed_linear           Y = dequant(X codes) . dequant(W codes)^T with per-channel
 *                               weight formats (Sec. 6: same-format sub-GEMMs / weights
 *                               dequantized in registers)
 *
 * Conventions shared by every call:
 *   - Every pointer inside a descriptor or passed as a buffer is DEVICE memory unless its
 *     comment says "host".  The caller owns every buffer; the library allocates nothing and
 *     keeps no mutable global state beyond a per-device cache of the CU count (filled once,
 *     atomically) and, for cham_quantize_act_noalloc only, an 8 KB device array per GPU
 *     with its address (see there).  Calls are thread-safe, except that calls of
 *     cham_quantize_act_noalloc that overlap on one GPU share that array.
 *   - `stream` is a hipStream_t (NULL = the default stream).  Every call only enqueues work
 *     on that stream and returns without synchronizing.
 *   - Argument errors are detected on the host and returned synchronously before anything is
 *     enqueued; launch errors are returned as CHAM_EHIP.  No exception crosses the ABI.
 *   - Layouts are row-major.  W is [N][K] (C_out x C_in, as nn.Linear stores it), X is [M][K],
 *     Y is [M][N].  MX blocks are 32 contiguous elements along K; NF4 blocks 64.
 *   - Workspace: calls that take (ws, ws_bytes) need at least cham_workspace_bytes(op, ...)
 *     bytes of device memory aligned to 256 bytes; its contents need not be initialized.
 */
#ifndef CHAMELEON_H_
#define CHAMELEON_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------------------
 * status codes
 * ------------------------------------------------------------------------------------- */
#define CHAM_OK 0
#define CHAM_EINVAL (-1)     /* NULL pointer, negative or zero size, bad layer/bucket index  */
#define CHAM_ESHAPE (-2)     /* K not a multiple of 32 (every call) or of 64 (NF4 enabled;
                                mixed_linear), or beyond a call's size limit               */
#define CHAM_EFORMAT (-3)    /* unknown format id, empty or out-of-range palette mask        */
#define CHAM_EHIP (-4)       /* a HIP launch or runtime call failed                          */
#define CHAM_EWORKSPACE (-5) /* ws NULL or smaller than cham_workspace_bytes()               */

/* Human-readable message for a status code (static storage, never NULL). */
const char* cham_status_string(int status);

/* Library version as (major << 16) | (minor << 8) | patch. */
int cham_version(void);

/* ---------------------------------------------------------------------------------------
 * number formats (Sec. 4.2)
 * ------------------------------------------------------------------------------------- */
/* Weight formats, in the paper's palette order F_w^(8) then F_w^(4).  palette_mask bit f
 * enables format f. */
#define CHAM_W_INT8_SYM 0
#define CHAM_W_INT8_ASYM 1
#define CHAM_W_MXINT8 2
#define CHAM_W_INT4_SYM 3
#define CHAM_W_INT4_ASYM 4
#define CHAM_W_NF4 5
#define CHAM_W_FP4 6
#define CHAM_W_MXINT4 7
#define CHAM_W_MXFP4 8
#define CHAM_W_NFMT 9
/* The few-step 4-bit search set {INT4-asym, NF4, FP4, MXINT4, MXFP4} and F_w^(8). */
#define CHAM_MASK_W4 0x1F0u
#define CHAM_MASK_W8 0x007u

/* Activation formats = the runtime LUT codes 0..4. */
#define CHAM_A_INT8_ASYM 0
#define CHAM_A_FP8_E4M3 1
#define CHAM_A_FP8_E5M2 2
#define CHAM_A_MXFP8_E4M3 3
#define CHAM_A_MXINT8 4
#define CHAM_A_NFMT 5

/* ---------------------------------------------------------------------------------------
 * 1. per-output-channel weight-format search (Sec. 4.5, Eq. weight-argmax)
 *
 * For each output channel n, W[n][:] is round-tripped through every enabled format and the
 * format with the smallest sum of squared reconstruction errors (= the largest SQNR; ties go
 * to the lowest id) is kept, with its codes and metadata.  Quantizers (App. A.11, App. A.12):
 *   INT-sym   s = amax/Q (Q = 127, 7), q = clamp(round(w/s), -Q, Q), w^ = q s
 *   INT-asym  App. A.7 ScaleZP on the channel's own [lo, hi]: s = (hi-lo)/L (L = 255, 15),
 *             z = round(-lo/s), not clamped (a one-sided row has z outside [0, L]);
 *             q = clamp(round(w/s) + z, 0, L), w^ = (q - z) s; a constant row (hi == lo)
 *             takes s = |lo| (1 if lo == 0), so z = -sign(lo) and w^ = w
 *   FP4 E2M1  per channel s = amax/6, e = E2M1(clamp(w/s, +-6)), w^ = e s
 *   NF4       per 64-block a = absmax, c = nearest NF4 level to w/a, w^ = v_c a
 *   MXINT8/4  per 32-block E = floor(log2 amax), k = clamp(round(w 2^(F-E)), +-Q),
 *             F = 6 / 2, Q = 127 / 7, w^ = k 2^(E-F)
 *   MXFP4     per 32-block E = floor(log2 amax) - 2 (OCP MX v1.0), e = E2M1(clamp(w/2^E, +-6))
 * "round" is half-to-even, w/s is computed as w * (1/s) in binary32, and every floating
 * scale is floored at FLT_MIN; E8M0 exponents are clamped to [-127, 127] (all-zero block
 * -> -127) and stored biased (E + 127).
 * ------------------------------------------------------------------------------------- */
typedef struct cham_wq {
    int64_t N, K;           /* W is [N][K]; K > 0, even; K % 64 == 0 if NF4 enabled,
                               K % 32 == 0 if any MX format enabled                          */
    uint32_t palette_mask;  /* bit f enables format f; nonzero, bits >= 9 must be clear        */
    int32_t code_bits;      /* 4 if every enabled format is 4-bit, else 8; filled in by
                               cham_select_weight_formats (the caller may leave it 0)        */
    uint8_t* fmt;           /* [N]      chosen format id per channel                          */
    uint8_t* codes;         /* [N][K/2] two 4-bit codes per byte, even k in the low nibble
                               (code_bits 4), or [N][K] one code per byte (code_bits 8).
                               Codes: INT-sym, MXINT two's complement; INT-asym unsigned q;
                               NF4 level index 0..15 (ascending); E2M1 sign|exp(2)|mantissa */
    float* scale;           /* [N]      s of INT-sym/INT-asym/FP4 channels, 0 otherwise       */
    float* zero;            /* [N]      z of INT-asym channels (an integral binary32, any
                               magnitude), 0 otherwise                                        */
    float* nf4_absmax;      /* [N][K/64] block absmax of NF4 channels, 0 otherwise;
                               may be NULL iff NF4 is not enabled                             */
    uint8_t* e8m0;          /* [N][K/32] biased block exponent of MX channels, 0 otherwise;
                               may be NULL iff no MX format is enabled                        */
    int32_t* perm;          /* [N]      channels stably sorted by chosen format; NULL = skip   */
    int32_t* group_off;     /* [10]     start of each format's group in perm, [9] = N;
                               NULL = skip                                                    */
    double* err;            /* [N][9]   per-format error sums (diagnostic, relative accuracy
                               1e-5; -1 for disabled formats); NULL = skip                    */
    void* packed;           /* cham_packed_bytes(N, K) bytes, 256-byte aligned: the weights in
                               the layout cham_mixed_linear consumes (per channel its format
                               parameters; the weights decoded to half precision in the order
                               of the matrix-core operand, 2 bytes each).  Written by the
                               search when non-NULL (K must then be a multiple of 64);
                               cham_mixed_linear reads it instead of deriving it from the
                               codes on every call.  It must come from the search that wrote
                               these codes, by the same library version.  NULL = skip.       */
} cham_wq;

/* Search the formats of W [N][K] (device, binary32, finite) and fill *wq's buffers.
 * Ownership: the caller owns W and every buffer in *wq.  Errors: CHAM_EINVAL (NULL W/wq/
 * required buffer, N < 1), CHAM_EFORMAT (mask), CHAM_ESHAPE (K not a multiple of 32, or of
 * 64 with NF4 enabled, a packed layout requested or K > 8192; K > 32768: a row is held in
 * the registers of one workgroup), CHAM_EHIP. */
int cham_select_weight_formats(const float* W, cham_wq* wq, void* stream);

/* Bytes of the packed GEMM layout of an N x K weight (see cham_wq.packed). */
size_t cham_packed_bytes(int64_t N, int64_t K);

/* The same search for nlayers independent weight matrices (Sec. 4.5 applies per layer):
 * W is a host array of nlayers device pointers, wq a host array of nlayers descriptors,
 * each with its own buffers.  Results are those of nlayers separate calls; layers that
 * share a kernel variant share launches (fewer, fuller launches for a model's layers).
 * Every layer is checked before anything is launched; the first error is returned.
 * Errors: as cham_select_weight_formats, CHAM_EINVAL also for NULL arrays or nlayers < 1. */
int cham_select_weight_formats_batch(const float* const* W, cham_wq* wq, int32_t nlayers, void* stream);

/* The packing step of the search on its own: writes wq[i].packed for n weights whose
 * fmt, codes, scale, zero, NF4 absmax and E8M0 a search (with packed = NULL) has already
 * filled, with code_bits as that search set it; perm, group_off and err are not touched.
 * The layout is the bits the search writes when it packs.  It lets a caller pack one group
 * of layers on another stream while the search of the next group runs.  wq: host array of
 * n descriptors.  Every descriptor is checked before anything is launched.  Errors:
 * CHAM_EINVAL (NULL arrays or buffers, n < 1, packed not 256-byte aligned, code_bits not
 * that of the palette), CHAM_EFORMAT (mask), CHAM_ESHAPE (K not a multiple of 64, or
 * K > 2^20), CHAM_EHIP. */
int cham_pack_weights_batch(const cham_wq* wq, int32_t n, void* stream);

/* ---------------------------------------------------------------------------------------
 * 1b. DiT joint (group size, format) weight search (Sec. 4.6 (i))
 *
 * For one linear layer W [N][K], every tuple (g, f) of the enabled group sizes g (groups of
 * g consecutive input channels along K; the last group holds K mod g when g does not divide
 * K) and enabled formats f is evaluated: each group is quantized with its own parameters as
 * the format's per-channel quantizer above defines them (INT-sym / INT-asym on the group's
 * range, FP4 amax/6, NF4 the group absmax), and the layer's input-aware error
 * sum_n sum_k energy[k] (w - w^)^2 (energy[k] = E[x_k^2], the activation energy of input
 * channel k) is formed in binary64.  The tuple with the smallest error (= the largest
 * input-aware SQNR) is chosen, ties to the lowest index t = group index * 9 + format; MX
 * formats use their own 32-blocks and are evaluated at g = 32 only.  The choice stays on
 * the device (choice[]), so no synchronization is needed before the GEMM.
 * ------------------------------------------------------------------------------------- */
#define CHAM_NGROUPS 5          /* group sizes 32, 64, 128, 192, 288 (bit i of group_mask)  */
#define CHAM_GMASK_ALL 0x1Fu
/* The DiT fork's 4-bit search set {INT4-asym, NF4, FP4}; at 8 bits F_w^(8). */
#define CHAM_MASK_DIT_W4 0x070u

typedef struct cham_gwq {
    int64_t N, K;           /* W is [N][K]; K % 32 == 0, K <= 8192                           */
    uint32_t palette_mask;  /* formats searched (bit f = format f)                            */
    uint32_t group_mask;    /* group sizes searched (bit i = the i-th size); nonzero          */
    int32_t code_bits;      /* 4 if every enabled format is 4-bit, else 8 (set by the search) */
    int32_t* choice;        /* [2] device: the chosen group size and format id                */
    uint8_t* fmt;           /* [N]      the chosen format id in every entry                   */
    uint8_t* codes;         /* [N][K/2] (4-bit) or [N][K] (8-bit), as in cham_wq              */
    float* gscale;          /* [N][K/32] per group j (at index j): INT scale, FP4 scale or NF4
                               absmax; 0 past the last group and for MX formats               */
    float* gzero;           /* [N][K/32] per group: INT-asym zero point (integral), else 0    */
    uint8_t* e8m0;          /* [N][K/32] MX block exponents (0 unless an MX format is chosen);
                               may be NULL iff no MX format is enabled                        */
    double* err;            /* [45]     layer error of tuple t (-1 if not evaluated); NULL = skip */
    void* packed;           /* cham_packed_bytes(N, K) bytes, 256-byte aligned: the GEMM
                               layout, written by the search when non-NULL (4-bit palettes and
                               K % 64 == 0 only); NULL = skip                                  */
} cham_gwq;

/* Search W [N][K] (device, binary32, finite, 16-byte aligned) with error weights energy[K]
 * (device, binary32, 16-byte aligned) and fill *gq.  ws: CHAM_OP_GSELECT bytes (the
 * per-channel errors).  Errors: CHAM_EINVAL (NULL or misaligned buffer, N < 1), CHAM_EFORMAT
 * (masks; only MX formats without g = 32), CHAM_ESHAPE (K, or packing with 8-bit codes),
 * CHAM_EWORKSPACE, CHAM_EHIP. */
int cham_select_group_formats(const float* W, const float* energy, cham_gwq* gq, void* ws, size_t ws_bytes,
                              void* stream);

/* Calibration pre-pass of the search's weights: colsq[k] += sum_m X[m][k]^2 over X [M][K]
 * (device binary32; colsq device binary64 [K]), summed in a fixed order (bitwise
 * reproducible); E[x_k^2] = colsq[k] / rows.  ws: CHAM_OP_COLSQ bytes.
 * Errors: CHAM_EINVAL, CHAM_EWORKSPACE, CHAM_EHIP. */
int cham_act_colsq_accumulate(const float* X, int64_t M, int64_t K, double* colsq, void* ws, size_t ws_bytes,
                              void* stream);

/* ---------------------------------------------------------------------------------------
 * 2. calibration statistics (Sec. 4.4; Alg. 1) and the LUT (Sec. 4.3; Alg. 1)
 * ------------------------------------------------------------------------------------- */
typedef struct cham_act_stats {
    int32_t L, B;  /* layers, timestep buckets                                            */
    double* nS;    /* [L*B][5] n, sum x, sum x^2, sum x^3, sum x^4 (binary64)               */
    float* lohi;   /* [L*B][2] running min, max (binary32)                                 */
} cham_act_stats;

/* Set every accumulator to n = S_k = 0, lo = +inf, hi = -inf. */
int cham_act_stats_reset(cham_act_stats* st, void* stream);

/* Add one activation tensor X (numel binary32 values, device, 16-byte aligned) of `layer` at a timestep of
 * `bucket` into the accumulator: n += numel, S_k += sum x^k, lo/hi = min/max.  The sums are
 * reduced in a fixed order (bitwise reproducible run to run).  ws: CHAM_OP_STATS bytes.
 * Errors: CHAM_EINVAL (NULL, numel < 1, layer/bucket out of range), CHAM_EWORKSPACE, CHAM_EHIP. */
int cham_act_stats_accumulate(const float* X, int64_t numel, int32_t layer, int32_t bucket,
                              cham_act_stats* st, void* ws, size_t ws_bytes, void* stream);

/* The same for n tensors X[i] (host array of device pointers) of (layer[i], bucket[i]),
 * e.g. every instrumented layer's input of one calibration forward pass: the result is
 * bitwise that of n calls in array order (tensors of the same (layer, bucket) are added in
 * that order), in fewer launches.  numel, layer, bucket: host arrays of n.  ws: the sum of
 * cham_workspace_bytes(CHAM_OP_STATS, numel[i], 0, 0) over i.  Every argument is checked
 * before anything is launched.  Errors: as cham_act_stats_accumulate. */
int cham_act_stats_accumulate_batch(const float* const* X, const int64_t* numel, const int32_t* layer,
                                    const int32_t* bucket, int32_t n, cham_act_stats* st, void* ws,
                                    size_t ws_bytes, void* stream);

#define CHAM_SCHED_SCALED_LINEAR 0
#define CHAM_SCHED_LINEAR 1
typedef struct cham_schedule {
    int32_t T;                   /* diffusion steps (betas indexed 0..T-1)                    */
    double beta0, beta1;         /* first and last beta                                        */
    int32_t kind;                /* CHAM_SCHED_SCALED_LINEAR: (sqrt(b0)+(sqrt(b1)-sqrt(b0))s/(T-1))^2
                                    CHAM_SCHED_LINEAR:        b0 + (b1-b0) s/(T-1)             */
    double kappa_lo, kappa_hi;   /* kurtosis gates (3, 5)                                      */
    double snr_lo, snr_hi;       /* SNR gates (0.2, 2.0)                                       */
    int32_t snr_gate_on;         /* 0 routes by kurtosis alone                                 */
} cham_schedule;

/* SDXL's scaled-linear schedule 0.00085 -> 0.012, T = 1000, gates (3, 5, 0.2, 2.0), on. */
void cham_schedule_default(cham_schedule* s);

typedef struct cham_lut {
    int32_t L, B, T;  /* layers, buckets, schedule length                                  */
    uint8_t* F;       /* [L*B] format code 0..4                                             */
    float* S;         /* [L*B] scale                                                        */
    float* Z;         /* [L*B] zero point (integral, binary32)                              */
} cham_lut;

/* For every (l, b): kappa = m4/m2^2 from the power sums; SNR at the bucket midpoint
 * t_b = floor(b T/B + T/(2B)) with alpha_bar_t = prod_{s<=t} (1 - beta_s) and
 * SNR = alpha_bar/(1 - alpha_bar) (Sec. 3.1, Eq. snr); Route (Sec. 4.3): shortcut -> 3,
 * kappa > hi or SNR < lo -> 2, kappa <= lo and SNR > hi -> 0, else 1; ScaleZP (App. A.7) on
 * the bucket's [lo, hi] (an empty bucket gets S = 1, Z = 0).  is_shortcut: device [L] or
 * NULL.  kappa: device [L*B] binary64 or NULL.  lut->L, B must equal st's (B <= 1024); lut->T
 * is set to sch->T.  The SNR product is evaluated as a tree of binary64 products.
 * Errors: CHAM_EINVAL, CHAM_EHIP. */
int cham_build_act_lut(const cham_act_stats* st, const cham_schedule* sch,
                       const uint8_t* is_shortcut, cham_lut* lut, double* kappa, void* stream);

/* Bucket of timestep t (Alg. 2): min(floor(t B / T), B - 1); -1 if t < 0 or T, B < 1. */
int32_t cham_bucket(int32_t t, int32_t T, int32_t B);

/* ---------------------------------------------------------------------------------------
 * 3. activation quantization (Alg. 2 static / Alg. 3 dynamic)
 * ------------------------------------------------------------------------------------- */
typedef struct cham_aq {
    int64_t M, K;      /* X is [M][K]                                                        */
    int32_t fmt;       /* activation format used (filled in by the quantize call)             */
    int32_t nsamples;  /* S >= 1 samples of M/S consecutive rows each (M % S == 0), e.g. the
                          two halves of a CFG-doubled batch; each has its own (s, z)          */
    uint8_t* codes;    /* [M][K] INT8-asym unsigned q, FP8 / MXFP8 codes, MXINT8 two's compl. */
    uint8_t* e8m0;     /* [M][K/32] biased block exponents, 255 = NaN (MX formats; may be NULL
                          otherwise)                                                          */
    float* scale;      /* [S] the scale s of each sample (1 for MX formats)                   */
    float* zero;       /* [S] the zero point z of each sample (0 unless INT8-asym)            */
} cham_aq;

/* Quantize X [M][K] (device, finite binary32, 16-byte aligned; out->codes 4-byte aligned)
 * to activation format `fmt`:
 *   INT8-asym  q = clamp(round(x/s) + z, 0, 255); dynamic (s, z) by ScaleZP on this X's own
 *              [lo, hi] (App. A.7: s = (hi-lo)/255, z = round(-lo/s), z not clamped)
 *   FP8        e = E4M3 / E5M2(clamp(x/s, +-448 / +-57344)), round to nearest even
 *   MXFP8      per 32-block E = floor(log2 amax) (the paper's exponent: values in (-2, 2)),
 *              e = E4M3(x / 2^E)
 *   MXINT8     per 32-block E = floor(log2 amax), k = clamp(round(x 2^(6-E)), +-127)
 * Static (dynamic = 0): s = *s_dev, z = *z_dev (device pointers, e.g. LUT entries), the same
 * for every sample.  Dynamic (dynamic = 1, Alg. 3's per-sample, per-forward micro-scaling):
 * each of the out->nsamples samples takes (s, z) = ScaleZP(fmt, min, max) of its own rows
 * (one sample = per-tensor); s_dev/z_dev are ignored.  The (s, z) used are written to
 * out->scale[S] / out->zero[S].  1 <= nsamples <= 1024.  ws: CHAM_OP_QUANT_ACT
 * bytes.  Errors: CHAM_EINVAL, CHAM_EFORMAT, CHAM_ESHAPE (K % 32 for MX), CHAM_EWORKSPACE,
 * CHAM_EHIP. */
int cham_quantize_act(const float* X, int32_t fmt, int32_t dynamic, const float* s_dev,
                      const float* z_dev, cham_aq* out, void* ws, size_t ws_bytes, void* stream);

/* cham_quantize_act without a workspace argument, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc).  Same arguments, results and errors as cham_quantize_act; it calls no
 * allocating routine.  The dynamic min/max partials live in an 8 KB array of device memory
 * that the library holds on each GPU it runs on until the process ends; it is large enough
 * for every size this call accepts (the launch caps its partials at 1024).  All calls on one
 * GPU share that array: calls that overlap on one GPU (different streams, other threads)
 * race and must be ordered by the caller.  Errors: as cham_quantize_act (without
 * CHAM_EWORKSPACE); CHAM_EHIP also if the array's address cannot be obtained. */
int cham_quantize_act_noalloc(const float* X, int32_t fmt, int32_t dynamic, const float* s_dev,
                              const float* z_dev, cham_aq* out, void* stream);

/* The per-step runtime lookup of Alg. 2 / Alg. 3: b = cham_bucket(t, lut->T, lut->B), the
 * format is F_host[layer*B + b] (a host mirror of lut->F, copied once after calibration, so
 * no device synchronization is needed per step), and the scale/zero are read on the device
 * from lut->S/Z[layer*B + b] (static) or computed from X (dynamic). */
int cham_quantize_act_lut(const float* X, const cham_lut* lut, const uint8_t* F_host,
                          int32_t layer, int32_t t, int32_t dynamic, cham_aq* out, void* ws,
                          size_t ws_bytes, void* stream);

/* Alg. 2's runtime quantization and Alg. 1's moment gathering in one pass over each input,
 * for a model that keeps calibrating while it runs: tensor X[i] (out[i].M x out[i].K
 * binary32, device, 16-byte aligned) of layer[i] at timestep t is quantized as
 * cham_quantize_act_lut(X[i], lut, F_host, layer[i], t, 0, &out[i], ...) would do it
 * (static scales: the LUT's S/Z of (layer[i], b), b = cham_bucket(t, lut->T, lut->B), as
 * the device holds them when the kernel runs), and its moments are added into st at
 * (layer[i], b) as cham_act_stats_accumulate_batch adds them.  Codes, E8M0 bytes, scales,
 * zero points and accumulators are the bits those two calls give, in that order, on the
 * same inputs.  A LUT built afterwards from st sees this call's moments; the codes of this
 * call do not depend on them.  out: host array of n descriptors (fmt is filled in from
 * F_host).  layer: host array of n.  st->L, B must equal lut's.  ws: the sum of
 * cham_workspace_bytes(CHAM_OP_STATS, out[i].M * out[i].K, 0, 0) over i.  Every argument is
 * checked before anything is launched.  Errors: CHAM_EINVAL, CHAM_EFORMAT, CHAM_ESHAPE
 * (K % 32), CHAM_EWORKSPACE, CHAM_EHIP. */
int cham_quantize_act_lut_accumulate_batch(const float* const* X, const int32_t* layer, int32_t n, int32_t t,
                                           const cham_lut* lut, const uint8_t* F_host, cham_aq* out,
                                           cham_act_stats* st, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------
 * 4. the mixed-format linear layer
 *
 * Y[m][n] = sum_k x^[m][k] w^[n][k], with x^ = DQ(xq) and w^ = DQ(wq) exactly as the
 * quantizers above define them, accumulated in binary32 on the matrix cores.  Accuracy:
 * |Y - Y_exact| <= 1e-3 * sum_k |x^ w^| per element.  Operands are decoded to half
 * precision: NF4 levels times their block absmax, and INT-asym weight levels q - z beyond
 * 2^11 in magnitude, carry one rounding (relative 2^-11; INT8-asym channels with |z| beyond
 * 2^22, whose values agree to 6e-5, up to 2^-10); INT8-asym activations are decoded
 * exactly, a zero point beyond +-1024 through a per-channel correction (the channel's sum of
 * dequantized weights, binary64, times (z - z') s in the epilogue).  Block-scaled operands
 * (NF4 and MX weights, MX activations) are held relative to the largest block of their
 * channel or row: blocks within 2^28 of it are exact (NF4: one rounding), blocks further
 * below fall into half precision's subnormal range and lose bits.  An activation block whose
 * exponent byte is 255 (NaN) makes its rows of Y NaN.  xq->K must equal wq->K and be a multiple of
 * 64; the kernels address operands with 32-bit offsets, so K <= 2^20, N < 2^21 and the
 * weights' decode layout (cham_packed_bytes) stays below 2^31 bytes (CHAM_ESHAPE otherwise);
 * xq->codes, wq->codes and Y must be 16-byte aligned.  Y [M][N] is written in the
 * original channel order.  When the output has too few tiles to fill the GPU, K is split
 * across workgroups whose partial outputs a second kernel adds in split order; no atomics
 * are used, so Y is bitwise reproducible run to run.  If wq->packed is set it supplies the
 * weights' decode layout; otherwise a pre-pass derives it from the codes and metadata into
 * the workspace.  ws: what cham_mixed_linear_workspace_query reports for these operands
 * (2 M K + 4 M bytes reserved and not written for MX activations, the weights' layout
 * when wq->packed is NULL, the k-split partial outputs when the plan splits; possibly 0,
 * then ws may be NULL), 256-byte aligned; CHAM_OP_LINEAR bytes always suffice.
 * Errors: CHAM_EINVAL, CHAM_EFORMAT, CHAM_ESHAPE, CHAM_EWORKSPACE, CHAM_EHIP.
 * ------------------------------------------------------------------------------------- */
int cham_mixed_linear(const cham_aq* xq, const cham_wq* wq, float* Y, void* ws, size_t ws_bytes,
                      void* stream);

/* Exact workspace bytes of cham_mixed_linear for these operands (host only: reads the
 * descriptors, launches nothing, dereferences no device pointer) into *bytes (host).
 * Errors: those of cham_mixed_linear's argument checks (CHAM_EINVAL, CHAM_EFORMAT,
 * CHAM_ESHAPE), and CHAM_EINVAL for a NULL bytes. */
int cham_mixed_linear_workspace_query(const cham_aq* xq, const cham_wq* wq, size_t* bytes);

/* The same linear layer with group-scaled weights from cham_select_group_formats (the DiT
 * path, Sec. 4.6 (i)): each 32-element half of a 64-wide k-step lies in one group (every
 * group size is a multiple of 32), whose scale and zero point build its decode table;
 * accuracy as above.  4-bit palettes only (gq->code_bits == 4; the 8-bit group-scaled
 * decode is not built: CHAM_EFORMAT).  ws: as cham_mixed_linear (exact bytes from
 * cham_mixed_linear_grouped_workspace_query; CHAM_OP_LINEAR bytes always suffice). */
int cham_mixed_linear_grouped(const cham_aq* xq, const cham_gwq* gq, float* Y, void* ws, size_t ws_bytes,
                              void* stream);

/* Exact workspace bytes of cham_mixed_linear_grouped (as cham_mixed_linear_workspace_query). */
int cham_mixed_linear_grouped_workspace_query(const cham_aq* xq, const cham_gwq* gq, size_t* bytes);

/* The UNet path's 3x3 convolution (stride 1, zero padding 1) on quantized activations, as
 * an implicit GEMM on the same kernels: the layers downstream of a shortcut concatenation
 * (up-block resnet conv1) whose inputs Sec. 4.6 routes to MXFP8 whatever the LUT's gates
 * say (cham_build_act_lut's is_shortcut).  xq: the activation codes of B images of H x W
 * pixels with C channels, channels last (xq->M = B H W rows, xq->K = C, C % 64 == 0; its
 * samples are 1 or B images).  wq: the weights as a linear layer [Co][9 C] with
 * k = (ky * 3 + kx) * C + c (searched like any linear weight).  Y [B H W][Co] (device,
 * binary32): Y[b,y,x][o] = sum over ky, kx, c of x^[b, y+ky-1, x+kx-1, c] w^[o, k],
 * out-of-image pixels zero.  The GEMM gathers the codes per output pixel and tap and decodes
 * them to half precision (MX formats relative to the largest block exponent of the pixels an
 * output tile gathers: exact for blocks within 2^28 of it; INT8-asym q - z rounded once when
 * beyond 2^11 or where the zero point is no integer); accuracy as cham_mixed_linear.
 * ws: cham_conv3x3_workspace_bytes.
 * Errors: CHAM_EINVAL (sizes, pointers, samples), CHAM_EFORMAT, CHAM_ESHAPE (C % 64, or
 * 2 B (H + 2) (W + 2) C beyond 2^31 - 4096), CHAM_EWORKSPACE, CHAM_EHIP. */
int cham_conv3x3_mixed(const cham_aq* xq, int32_t B, int32_t H, int32_t W, const cham_wq* wq, float* Y,
                       void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of cham_conv3x3_mixed for B images of H x W x C and Co output channels
 * (0 for sizes out of range). */
size_t cham_conv3x3_workspace_bytes(int64_t B, int64_t H, int64_t W, int64_t C, int64_t Co);

/* The launch plan cham_mixed_linear takes for M x N x K (diagnostics; host only, launches
 * nothing).  out (host, out_len >= 10 int32) receives {launches, always 1; k-splits; first row 0,
 * end row M, tile rows, tile channels; four zeros}.  code_bits (4 or 8) is checked and does not
 * change the plan.  The plan depends on the current device's CU count (256 when no device is
 * visible).  Errors: CHAM_EINVAL (NULL out, out_len < 10, sizes < 1, code_bits not 4 or 8). */
int cham_linear_plan(int64_t M, int64_t N, int64_t K, int32_t code_bits, int32_t* out, int32_t out_len);

/* ---------------------------------------------------------------------------------------
 * 5. operators around 8-bit linear layers
 *
 * What a transformer block runs between its matrix products when those read 8-bit codes: the
 * residual's addition with the root-mean-square norm, and the activation function between two
 * feed-forward products, each ending in codes and scales in one pass; and a product whose
 * scales follow blocks of 128.  The two passes write either the block format below, which
 * cham_block_linear reads, or one of the activation formats of section 3 with one scale per
 * token, which cham_mixed_linear reads.  Rows may be strided; element types are CHAM_T_*.
 * Row starts must be 16-byte aligned (base pointers and row strides), K % 32 == 0.  M = 0 is
 * an empty call: nothing launched, CHAM_OK (its row pointers may be NULL).
 * ------------------------------------------------------------------------------------- */
#define CHAM_T_F32 0
#define CHAM_T_F16 1
#define CHAM_T_BF16 2
#define CHAM_T_N 3
#define CHAM_T_EXACT 256  /* or-ed into y_type: a 16-bit Y of cham_block_linear from exact products */

/* The block format: E4M3 codes with one scale per row and 128 consecutive elements (the last
 * block of a row holds K mod 128 if 128 does not divide K):
 *   s = amax / 448, floored at FLT_MIN, or (pow2) the next power of two at or above that
 *   c = E4M3(clamp(y fl(1/s), +-448)), round to nearest even
 * A block that holds a NaN or an infinity has the scale NaN (byte 255), so everything computed
 * from it is NaN; its codes are unspecified. */
typedef struct cham_bq {
    int64_t M, K;      /* codes of [M][K]                                                    */
    int32_t pow2;      /* 0: binary32 scales; 1: powers of two, held as E8M0 bytes (E + 127)  */
    uint8_t* codes;    /* [M][K] E4M3, 16-byte aligned                                       */
    void* scale;       /* [ceil(K / 128)][M], block-major: the scales of one block of all rows
                          are consecutive (float, or uint8_t if pow2)                         */
} cham_bq;

/* Weights in the block format: one scale for each 128 x 128 block (ragged at both ends). */
typedef struct cham_bw {
    int64_t N, K;      /* codes of [N][K]                                                    */
    int32_t pow2;      /* as in cham_bq                                                       */
    uint8_t* codes;    /* [N][K] E4M3, 16-byte aligned                                       */
    void* scale;       /* [ceil(N / 128)][ceil(K / 128)] (float, or uint8_t if pow2)          */
} cham_bw;

/* h = x + r (binary32), y = h / sqrt(mean(h^2) + eps) * g: the norm sees the unrounded sum; h is
 * written rounded to its own type.  The squares, their sum and the root are binary64, so every
 * finite h has its norm; y carries three roundings to binary32 behind it. */
typedef struct cham_norm {
    int64_t M, K;      /* K <= 32768                                                         */
    const void* x;     /* [M][K], row stride ldx elements                                    */
    int64_t ldx;
    const void* r;     /* the residual [M][K], row stride ldr; NULL = none                   */
    int64_t ldr;
    void* h;           /* [M][K], row stride ldh, of r's type; may be r itself (same stride), no
                          other overlap with the inputs; NULL = not written                   */
    int64_t ldh;
    const void* g;     /* [K] weights, 16-byte aligned; NULL = ones                          */
    int32_t x_type;
    int32_t r_type;    /* type of r and h: x_type or CHAM_T_F32                              */
    int32_t g_type;
    float eps;         /* >= 0 (a row of zeros with eps = 0 is NaN)                          */
} cham_norm;

/* The norm of n, written in the block format (out->M, K equal n's).
 * Errors: CHAM_EINVAL (NULL, sizes, strides, alignment, eps), CHAM_EFORMAT (types),
 * CHAM_ESHAPE (K % 32, K > 32768, M >= 2^31, or a launch of 2^32 lanes: a row takes 64 up to
 * K = 2048, 256 up to 8192, then 1024), CHAM_EHIP. */
int cham_rms_norm_quantize_block(const cham_norm* n, cham_bq* out, void* stream);

/* The norm of n, written in activation format fmt of section 3 with dynamic scales of each
 * token: out->nsamples must be M (scale [M], zero [M]; e8m0 [M][K/32] for MX formats), codes
 * 8-byte aligned.  A row that holds a NaN or an infinity takes the scale NaN; in MX formats its
 * block of 32 takes the exponent byte 255, which is NaN, and MXFP8 codes that are NaN.  Errors: as
 * above, CHAM_EFORMAT also for fmt. */
int cham_rms_norm_quantize(const cham_norm* n, int32_t fmt, cham_aq* out, void* stream);

/* Activation functions, in binary32: relative error at most 1e-6 + 4e-7 a with a the size of the
 * exponent's argument (GELU: x^2, and 1.2e-6 more); values below 2^-119 may come out as 0. */
#define CHAM_ACT_NONE 0       /* x                                                            */
#define CHAM_ACT_SILU 1       /* x / (1 + exp(-x))                                            */
#define CHAM_ACT_GELU 2       /* x Phi(x), Phi the normal distribution function               */
#define CHAM_ACT_GELU_TANH 3  /* x / (1 + exp(-2 sqrt(2/pi) (x + 0.044715 x^3))): GELU's tanh
                                 form, 0.5 x (1 + tanh(...)), written without cancellation    */
#define CHAM_ACT_N 4

/* y = f(x) u (u = NULL: y = f(x)); x and u may be the two halves of one matrix.  With
 * CHAM_ACT_NONE and no u this is the quantizer alone. */
typedef struct cham_gate {
    int64_t M, K;      /* K <= 32768 for the per-token formats                               */
    const void* x;     /* [M][K], row stride ldx elements                                    */
    int64_t ldx;
    const void* u;     /* [M][K], row stride ldu; NULL = none                                */
    int64_t ldu;
    int32_t type;      /* of x and u                                                          */
    int32_t act;       /* CHAM_ACT_*                                                          */
} cham_gate;

/* The gate of a, written in the block format (out->M, K equal a's), or in an activation
 * format with one scale per token (as cham_rms_norm_quantize).  Errors: CHAM_EINVAL,
 * CHAM_EFORMAT (types, act, fmt), CHAM_ESHAPE (K % 32, K > 32768 with one scale per token, K >
 * 2^30 otherwise, M >= 2^31, or a launch of 2^32 lanes: one per 16 elements in the block and MX
 * formats, as in the norm in the others), CHAM_EHIP. */
int cham_gated_quantize_block(const cham_gate* a, cham_bq* out, void* stream);
int cham_gated_quantize(const cham_gate* a, int32_t fmt, cham_aq* out, void* stream);

/* Weights W [N][K] (row stride ldw elements) brought to the block format: out->N, K and pow2
 * are given.  N >= 1.  Errors: CHAM_EINVAL, CHAM_EFORMAT, CHAM_ESHAPE (K % 32, or 2^32 lanes at
 * 512 for each block of 128 x 128), CHAM_EHIP. */
int cham_block_quantize_weights(const void* W, int32_t type, int64_t ldw, cham_bw* out, void* stream);

/* Y[m][n] = sum over blocks b of xs[b][m] ws[n / 128][b] sum_{k in b} xc[m][k] wc[n][k],
 * accumulated in binary32 and rounded once to y_type.  Binary32 outputs, and 16-bit ones with
 * CHAM_T_EXACT or-ed into y_type, form every product exactly: the error before the rounding is at
 * most (128 + blocks) 2^-23 S, S = sum over b of xs ws sum |xc wc|.  Other 16-bit outputs use the
 * 8-bit matrix instructions at twice the rate: of 8 neighbouring k they drop what lies more than 13
 * bits below the largest product, at most 7 2^-13 S in all.  On heavy-tailed data that is 3e-5 to
 * 4e-5 of the result (root mean square, measured; a binary16 rounding is 2e-4), but where large
 * products cancel, what is left of the sum may be lost.  The product of an activation's and a
 * weight's scale is formed in binary32: where it overflows, Y is infinite or NaN, and below 2^-126 it
 * loses bits of Y.  x->pow2 must equal w->pow2.  Y [M][N], row stride ldy elements (any; any N).  The
 * order of the additions is fixed by the sizes and y_type (no atomics): Y is bitwise reproducible.
 * No workspace.  Errors: CHAM_EINVAL, CHAM_EFORMAT (y_type), CHAM_ESHAPE (K % 32, K > 2^20, M or N >
 * 2^31 - 257, or a launch of 2^32 lanes), CHAM_EHIP. */
int cham_block_linear(const cham_bq* x, const cham_bw* w, void* Y, int32_t y_type, int64_t ldy,
                      void* stream);

/* The launch plan cham_block_linear takes for M x N x K and y_type (diagnostics; host only): out
 * (host, out_len >= 3) receives {tile rows, tile channels, wavefront groups that split k inside a
 * workgroup}; tiles of 16 x 16 are the few-row kernel's.  Depends on the current device's CU
 * count (256 when no device is visible).  Errors: CHAM_EINVAL, CHAM_EFORMAT, CHAM_ESHAPE. */
int cham_block_linear_plan(int64_t M, int64_t N, int64_t K, int32_t y_type, int32_t* out, int32_t out_len);

/* ---------------------------------------------------------------------------------------
 * 6. attention
 *
 * What a transformer block runs between the product that makes queries, keys and values and the
 * one that reads attention's output: the norm of each head with the rotation by the token's
 * position, a paged cache of keys and values that is written and read back, and attention over
 * whole prompts or over the cache.  Sequences lie packed, one after another, in matrices
 * [T][H][D] of tokens, heads and D elements.  D % 8 == 0, 8 <= D <= 128.
 * Query head h reads key head h / (Hq / Hk); Hq % Hk == 0.
 * ------------------------------------------------------------------------------------- */
#define CHAM_T_E4M3 3  /* a cache's codes; no other operand's type */

/* Rows of heads [T][H][D]: element d of head h of token t at p[t * token + h * head + d].  p, token
 * and head are multiples of 16 bytes; rows may overlap in no way where they are written. */
typedef struct cham_heads {
    void* p;
    int64_t token, head;   /* strides in elements                                             */
    int32_t H;
    int32_t type;          /* CHAM_T_F32, CHAM_T_F16, CHAM_T_BF16                             */
} cham_heads;

#define CHAM_ROT_HALF 0    /* element i turns with element i + R/2                            */
#define CHAM_ROT_PAIRS 1   /* element 2i turns with element 2i + 1                            */

/* y = x / sqrt(mean_D(x^2) + eps) * g (norm), then the pairs (a, b), i = 0 .. R/2 - 1, of the first
 * R elements turn by the angle t = pos freq[i]: (a cos t - b sin t, b cos t + a sin t) * amp.
 * The squares, their sum and the root are binary64 for binary32 elements and where a row's mean square lies
 * outside 2^-60 .. 2^100, else binary32 (y within 2^-20): every finite row has its norm.  Angles are binary64
 * up to their reduction by pi/2, so far positions keep their angle (absolute error below 2^-53 |t| + 2^-24, and a
 * pair its length at any t); elements behind R are not touched but by the norm;
 * the rest is binary32, rounded once to the output's type. */
typedef struct cham_rotate {
    int64_t T;             /* tokens                                                          */
    int32_t D;
    int32_t R;             /* even, 0 (no rotation) .. D                                      */
    int32_t layout;        /* CHAM_ROT_*                                                      */
    int32_t norm;          /* 0 or 1                                                          */
    float eps;             /* >= 0; only read with norm                                       */
    float amp;             /* factor of the turned pairs; 1 = a rotation                      */
    const void* qg;        /* weights [D] of the norm, 16-byte aligned; NULL = ones           */
    const void* kg;
    int32_t qg_type, kg_type;
    const int32_t* pos;    /* [T] positions; NULL if R = 0                                    */
    const double* freq;    /* [R / 2] angle for each position; NULL if R = 0                  */
} cham_rotate;

/* Norm and rotation of queries and keys: qo = y(q), ko = y(k), of the inputs' types (one type for
 * all four), any strides; an output may be its input itself, with equal strides, and overlaps
 * nothing else.  Hq or Hk may be 0 (that pair is not touched).
 * Errors: CHAM_EINVAL (NULL, sizes, strides, alignment, eps, amp), CHAM_EFORMAT (types, layout),
 * CHAM_ESHAPE (D, H > 2^16, T >= 2^31 - 2^16, or a launch of 2^32 lanes: 256 for up to 8 tokens), CHAM_EHIP. */
int cham_norm_rotate(const cham_rotate* r, const cham_heads* q, const cham_heads* qo, const cham_heads* k,
                     const cham_heads* ko, void* stream);

/* A cache of keys and values in pages: [pages][H][page][D], so the tokens of a page lie together
 * for each head.  Token t of a sequence whose pages are table[0], table[1], ... lies in page
 * table[t / page], place t % page; slot = page index * page + place.
 * E4M3: codes with one scale for each token and head, s = amax / 448 floored at FLT_MIN,
 * c = E4M3(y fl(1/s)); a row that holds a NaN or an infinity has the scale NaN. */
typedef struct cham_cache {
    int64_t pages;         /* pages * page < 2^31                                             */
    int32_t H, D;          /* E4M3: D % 16 == 0                                               */
    int32_t page;          /* tokens of a page: a power of two, 16 .. 32768                   */
    int32_t type;          /* CHAM_T_F16, CHAM_T_BF16 or CHAM_T_E4M3                          */
    void* k;               /* 16-byte aligned, as v                                           */
    void* v;
    float* ks;             /* E4M3: [pages][H][page]; else NULL                               */
    float* vs;
} cham_cache;

/* Norm and rotation (r) of keys and queries in one pass with the keys and the values, which take
 * neither, written into the cache: token t goes to slot slots[t]; a slot outside 0 .. pages * page - 1
 * (-1, by custom) takes none.  Two tokens of one slot leave it undefined.  q and qo may be NULL.
 * One type for q, qo, k and v.  Errors: as cham_norm_rotate. */
int cham_cache_write(const cham_cache* c, const int32_t* slots, const cham_rotate* r, const cham_heads* k,
                     const cham_heads* v, const cham_heads* q, const cham_heads* qo, void* stream);

/* Sequences of a cache brought back into packed rows: row cu[b] + t holds token t of sequence b, its
 * page table[b][t / page].  table [B][width], cu [B + 1] (device, ascending from cu[0] >= 0; rows
 * from cu[B] on, and before cu[0], are left as they are); ko and vo have T rows of c's heads, of one type, the values code
 * times scale rounded to it.  A token without a page (outside 0 .. pages - 1, or t / page >= width)
 * comes back as zeros.  Errors: as cham_norm_rotate. */
int cham_cache_read(const cham_cache* c, const int32_t* table, int64_t width, const int32_t* cu, int64_t B, int64_t T,
                    const cham_heads* ko, const cham_heads* vo, void* stream);

/* o_i = sum_j p_ij v_j, p_i the softmax over the keys j that query i sees of scale <q_i, k_j>.
 * causal: query i of a sequence's nq sees its first nk - nq + i + 1 of nk keys (the last query sees all
 * of them); else all.  A query that sees none gets zeros; keys that are not seen have no influence,
 * whatever they hold; nor have other rows of q.  Products in 16 bits (q, k, v as they are; p rounded to their type;
 * over E4M3 values p times the value's scale rounded to binary16), sums, maxima and statistics in binary32, one
 * rounding at the end.  In binary16 terms below 2^-27 of a row's largest may be left out, and those below 2^-16 of it
 * have fewer than 11 bits.  Results are bitwise reproducible. */
typedef struct cham_attn {
    int64_t B;             /* sequences, < 2^24                                               */
    int64_t T;             /* rows of q and o                                                 */
    int32_t D;
    int32_t causal;        /* 0 or 1 (cham_cache_attention: always causal, not read)          */
    float scale;           /* > 0, finite                                                     */
    int32_t pad;
    const int32_t* cu_q;   /* [B + 1] first rows, ascending from 0 to at most T: rows behind the
                              last sequence are left as they are.  NULL: B sequences of T / B   */
    cham_heads q, o;       /* CHAM_T_F16 or CHAM_T_BF16, one type; o overlaps no input (o.p ==
                              q.p is refused)                                                 */
} cham_attn;

#define CHAM_ATTN_NO_WS 256
#define CHAM_ATTN_NO_WS_ONE 1024

/* Attention over packed keys and values k, v [Tk][Hk][D] of q's type: cu_k as cu_q, NULL: B
 * sequences of Tk / B rows.  ws: cham_attention_workspace_bytes(a, Hk) bytes, written before they are
 * read; calls that may overlap (two streams, two graphs) need workspaces of their own.  With at most
 * CHAM_ATTN_NO_WS keys (Tk, or width * page) no call needs one, and ws may be NULL; nor does a
 * cham_cache_attention of one query a sequence (cu_q NULL, T = B) with at most CHAM_ATTN_NO_WS_ONE.
 * Errors: CHAM_EINVAL (NULL, sizes, strides, alignment, T % B or Tk % B without cu_q or cu_k, scale,
 * o over q), CHAM_EFORMAT (types), CHAM_ESHAPE (D, H > 2^16, B >= 2^24, T Hq / Hk or Tk of 2^31 - 2^16 and
 * more, a token stride of k or v of 2^24 elements and more, or a launch of 2^32 lanes), CHAM_EWORKSPACE,
 * CHAM_EHIP. */
int cham_attention(const cham_attn* a, const cham_heads* k, const cham_heads* v, int64_t Tk, const int32_t* cu_k,
                   void* ws, size_t ws_bytes, void* stream);

/* Attention of each sequence's newest tokens over its tokens in a cache: lens[b] (device) counts
 * sequence b's tokens, the queries' own among them, which have been written before; table [B][width] as
 * in cham_cache_read.  Always causal.  A token without a page is seen by no query; lens beyond
 * width * page (or 2^31 - 2^16) count as that.  c's type is q's, or E4M3.  ws and errors as cham_attention. */
int cham_cache_attention(const cham_attn* a, const cham_cache* c, const int32_t* table, int64_t width,
                         const int32_t* lens, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of both for Hk key heads (0 for sizes out of range).  They depend on the current
 * device's CU count. */
size_t cham_attention_workspace_bytes(const cham_attn* a, int32_t Hk);

/* ---------------------------------------------------------------------------------------
 * workspace sizes
 * ------------------------------------------------------------------------------------- */
#define CHAM_OP_SELECT 0
#define CHAM_OP_STATS 1
#define CHAM_OP_QUANT_ACT 2
#define CHAM_OP_LINEAR 3
#define CHAM_OP_GSELECT 4   /* cham_select_group_formats: N output channels              */
#define CHAM_OP_COLSQ 5     /* cham_act_colsq_accumulate: K input channels               */
/* Bytes of workspace op needs at these sizes (M rows of X -- numel for CHAM_OP_STATS --,
 * N output channels, K inner size).  0 means no workspace. */
size_t cham_workspace_bytes(int32_t op, int64_t M, int64_t N, int64_t K);

#ifdef __cplusplus
}
#endif
#endif /* CHAMELEON_H_ */
