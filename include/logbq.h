/*
 * logbq.h -- C ABI of liblogbq, LogbQuant weight-only inference (4-bit and 8-bit codes) on AMD
 * MI355X (gfx950).
 *
 * LogbQuant (Bohn et al., arXiv 2607.01127) quantizes each weight matrix with its own
 * logarithmic codebook of base b and shift s (Sec. 3.1): a weight x maps to the integer
 * q = sign(x) * round(log_b|x| + s) with |q| <= q_max = 2^(n-1) - 1 (Eq. 1), and q decodes to
 * sign(q) * b^(|q| - s), or 0 for q = 0 (Eq. 2). b and s come from the effective weight range
 * [w_min, w_max] (Eq. 3, Eq. 4); w_min discards a fraction eps of the signal energy (Eq. 5).
 * Inference dequantizes through a lookup table instead of evaluating b^x (Sec. 3.3).
 *
 * Conventions shared by every call
 *   - Every call validates all of its arguments before it touches the GPU, and returns a
 *     logbq_status. No device memory is allocated inside a call. Device calls are enqueued on
 *     the given stream and return at once, so they can be captured in a HIP graph; the one
 *     exception is logbq_fit_device, which waits for each of its passes because the host
 *     chooses the next pass's bin. Faults of an enqueued kernel surface at the caller's next
 *     synchronisation.
 *   - `stream` is a hipStream_t passed as void*; NULL is the default stream.
 *   - The caller owns every buffer. "device" pointers are HIP device memory of the current
 *     device; "host" pointers are ordinary host memory.
 *   - Weights are row-major [N][K] (N out features, K in features, as a PyTorch Linear).
 *   - 4-bit codes: row-major [N][K/2] bytes; element (n, k) is the nibble at byte
 *     n*K/2 + k/2, the low nibble when k is even. A nibble is sign<<3 | magnitude: bit 3 set
 *     means negative, magnitude 0..7 is |q|. Code 8 ("-0") is never written and decodes to +0.
 *   - 8-bit codes: row-major [N][K] bytes, one code per weight: sign<<7 | magnitude (0..127).
 *     Code 128 ("-0") is never written and decodes to +0.
 *   - Shapes: K must be a multiple of 32 (every packed row is then 16-byte aligned);
 *     device pointers must be 16-byte aligned. N = 0 or M = 0 is a valid empty call.
 */
#ifndef LOGBQ_H
#define LOGBQ_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LOGBQ_ABI_VERSION 2

typedef enum logbq_status {
  LOGBQ_OK = 0,
  LOGBQ_ERR_INVALID_ARG = 1,   /* null pointer, negative size, eps outside (0,1), ... */
  LOGBQ_ERR_NONFINITE = 2,     /* fit: a weight is NaN or Inf                           */
  LOGBQ_ERR_DEGENERATE = 3,    /* fit: all weights zero, or w_min == w_max (b = 1)      */
  LOGBQ_ERR_UNSUPPORTED = 4,   /* bits not 4 or 8, K % 32 != 0, misaligned, too large    */
  LOGBQ_ERR_HIP = 5,           /* a HIP call failed (no device, launch failure, ...)    */
  LOGBQ_ERR_HOST_RESOURCE = 6  /* host scratch memory could not be allocated              */
} logbq_status;

/* Per-tensor codebook parameters (Sec. 3.1, Sec. 3.2). Plain data; copy freely.
 * ABI version 2 widened codebook and thresholds for 8-bit codes (version 1 had 16 and 8). */
typedef struct logbq_params {
  int32_t bits;            /* codebook bit width n: 4 or 8                                 */
  int32_t qmax;            /* q_max = 2^(n-1) - 1                                          */
  double eps;              /* pruned energy fraction of Eq. 5                               */
  double wmin;             /* w_min of Eq. 5                                                */
  double wmax;             /* w_max = max |w| (Sec. 3.2)                                    */
  double base;             /* b of Eq. 3                                                    */
  int32_t shift;           /* s of Eq. 4 (an integer)                                       */
  int32_t reserved;
  int64_t wmin_index;      /* position of w_min in |w| sorted ascending                     */
  float codebook[256];     /* Dequant (Eq. 2) of every n-bit code, float32; entries from
                              2^n on are 0                                                  */
  float thresholds[128];   /* [k] = smallest float32 whose magnitude index exceeds k,
                              k = 0..qmax-1; entries from qmax on are +inf                  */
} logbq_params;

/* Per-tensor parameters of the comparison baseline: asymmetric linear quantization,
 * Quant(s, z, x) = round(x / s) - z (Sec. 2), at tensor granularity (Sec. 4). Plain data.
 * s = (max w - min w) / (2^n - 1) and z = round(min w / s), ties rounded up; code q in
 * 0 .. 2^n - 1 stands for s (q + z). Only n = 4 is provided. */
typedef struct logbq_uniform {
  int32_t bits;            /* 4                                                            */
  int32_t zero;            /* z                                                            */
  double wmin;             /* min w (signed)                                               */
  double wmax;             /* max w (signed)                                               */
  double scale;            /* s                                                            */
  float codebook[16];      /* s (q + z) rounded to float32: the codebook logbq_linear and
                              logbq_dequantize take for these codes                        */
  float thresholds[15];    /* [j - 1] = smallest float32 x whose code is at least j (+inf
                              if none), j = 1 .. 15                                          */
  float reserved;
} logbq_uniform;

/* ABI version of the loaded library (LOGBQ_ABI_VERSION it was built with). */
int32_t logbq_abi_version(void);

/* Static English name of a status code; never NULL. */
const char* logbq_status_str(int32_t status);

/*
 * logbq_fit -- per-tensor codebook parameters (Sec. 3.1 Eq. 3-4, Sec. 3.2 Eq. 5). Host only.
 *   w_host : host, numel float32 weights, read only.
 *   bits   : codebook width n, 4 or 8.
 *   eps    : pruned energy fraction, 0 < eps < 1 (the paper uses 4e-3 at 4 bits, 1e-6 at 8).
 *   out    : host, filled on success; untouched on error.
 * w_max = max|w|. w_min is the smallest |w_i| at which the ascending float64 prefix sum of
 * w^2, divided by the total, reaches eps (sequential summation in ascending |w| order).
 * b = (w_max / w_min)^(1/q_max); s = q_max - J with J the largest integer such that
 * b^J <= w_max. codebook[k] = float32(b^(k-s)), codebook[h+k] = -codebook[k] (h = 2^(n-1),
 * k = 1..q_max), codebook[0] = codebook[h] = +0. thresholds[k] is exact: the smallest float32
 * t with t >= b^(k + 1/2 - s).
 * Errors: INVALID_ARG (null, numel < 2, eps outside (0,1)), UNSUPPORTED (bits not 4 or 8),
 * NONFINITE (NaN/Inf weight), DEGENERATE (w_max == 0, or w_min == w_max), HOST_RESOURCE (the
 * host scratch could not be allocated).
 * Reentrant; allocates host scratch of 8*numel bytes internally for the sort, which runs on up
 * to 16 threads (LOGBQ_HOST_THREADS = 1..16 in the environment sets the count; the result does
 * not depend on it; if no thread can be started the sort runs on the calling thread).
 */
int32_t logbq_fit(const float* w_host, int64_t numel, int32_t bits, double eps,
                  logbq_params* out);

/* Bytes of device workspace logbq_fit_device needs. */
#define LOGBQ_FIT_WORKSPACE_BYTES 110600

/*
 * logbq_fit_device -- the per-tensor fit on device-resident weights (Sec. 3.1 Eq. 3-4,
 * Sec. 3.2 Eq. 5), with the energy sums of Eq. 5 taken exactly.
 *   w_dev        : device, numel float32 weights, 16-byte aligned, read only.
 *   numel        : 2 <= numel < 2^40.
 *   bits, eps    : as logbq_fit.
 *   workspace_dev: device, LOGBQ_FIT_WORKSPACE_BYTES bytes, 8-byte aligned, owned by the
 *                  caller; overwritten.
 *   out          : host, filled on success; untouched on error.
 *   stream       : hipStream_t the passes run on.
 * w_max = max|w|. w_min = |w| at the smallest position i of |w| sorted ascending (ties in any
 * order) with sum_{j <= i} w_j^2 >= eps * sum_j w_j^2, both sums exact (squares of float32
 * values are exact rationals); wmin_index = i. b, s, codebook and thresholds then follow
 * exactly as in logbq_fit. logbq_fit sums in float64, in sequence; the two agree unless the
 * exact ratio lies within float64 rounding of eps.
 * Three radix-selection passes over the weights (bits 30..20, 19..11, 10..0 of the float32
 * pattern of |w|) accumulate per-bin counts and exact integer energy sums on the device; the
 * host picks each pass's bin with exact integer arithmetic. Blocks the calling thread until
 * the stream has run the passes (not capturable in a HIP graph).
 * Errors: INVALID_ARG (null, numel < 2, eps outside (0,1)), UNSUPPORTED (bits not 4 or 8,
 * numel too large, misaligned), NONFINITE (NaN/Inf weight), DEGENERATE (w_max == 0 or
 * w_min == w_max), HIP (a HIP call failed), HOST_RESOURCE (host copies of the bins could not
 * be allocated).
 */
int32_t logbq_fit_device(const float* w_dev, int64_t numel, int32_t bits, double eps,
                         void* workspace_dev, logbq_params* out, void* stream);

/*
 * logbq_fit_exact -- logbq_fit_device's fit on host weights: the same three radix-selection
 * passes, run on the host, and the same exact selection, so the parameters equal
 * logbq_fit_device's bit for bit (Sec. 3.2 Eq. 5 with exact sums, Sec. 3.1 Eq. 3-4).
 *   w_host, numel, bits, eps, out: as logbq_fit (2 <= numel < 2^40).
 * Errors: as logbq_fit (HOST_RESOURCE included). Reentrant; allocates at most 48 KiB of host
 * scratch.
 */
int32_t logbq_fit_exact(const float* w_host, int64_t numel, int32_t bits, double eps,
                        logbq_params* out);

/*
 * logbq_encode -- Quant (Eq. 1) of a weight matrix into 4-bit or 8-bit codes (Sec. 3.3 packing).
 *   w_dev        : device, [n][k] float32 weights.
 *   n, k         : shape; k % 32 == 0.
 *   p            : host, parameters from logbq_fit (bits 4 or 8).
 *   codes_dev    : device, written: [n][k/2] bytes for 4 bits, [n][k] for 8 bits.
 *   codebook_out : host, 2^bits floats, receives p->codebook[0 .. 2^bits) (may be NULL).
 *   stream       : hipStream_t or NULL.
 * The magnitude index of x is the number of thresholds t with |x| >= t, which equals
 * clamp(round-half-up(log_b|x| + s), 0, q_max); the sign bit (bit n-1) is set for negative x
 * with a nonzero magnitude. NaN and +-0 encode to 0, +-Inf to the largest magnitude with its
 * sign.
 * Errors: INVALID_ARG (null, negative size, qmax not 2^(bits-1) - 1, thresholds[0..qmax)
 * not positive and ascending), UNSUPPORTED (bits, k % 32, alignment), HIP (launch failure).
 */
int32_t logbq_encode(const float* w_dev, int64_t n, int64_t k, const logbq_params* p,
                     uint8_t* codes_dev, float* codebook_out, void* stream);

/*
 * logbq_linear -- y = x . W_hat^T on packed codes: weight-only inference with the codebook
 * lookup fused into the product (Sec. 3.3).
 *   x_dev     : device, [m][k] IEEE float16 activations (bit patterns as uint16).
 *   m, k      : batch rows and in features; k % 32 == 0, m <= 4194240 (65535 * 64).
 *   codes_dev : device, [n][k/2] packed codes.
 *   n         : out features.
 *   codebook  : host, 16 floats (logbq_params.codebook); copied into the kernel arguments,
 *               so the call is capturable in a HIP graph. Entries are rounded to float16 after
 *               a common power-of-two scaling, exact in the result up to float16 rounding.
 *   y_dev     : device, [m][n] float32, written.
 * Accumulation is float32. Five kernels, chosen from (m, k, n) and from whether the codebook is
 * sign-symmetric (every fitted one is):
 *   - split-K dequantize-into-MFMA, m <= 32. At k in {1024, 2048, 4096, 8192}: 5 <= m <= 16, m = 4
 *     unless n <= 1024 at k = 8192, m = 3 at n >= 4096, and 17 <= m <= 32 unless m > 20 at k = 8192
 *     and n > 16384 (above m = 16 only for sign-symmetric codebooks); at k = 14336 and m <= 16, and
 *     at any other 512 <= k <= 16384 and 3 <= m <= 16 on the widths where it is the faster, for
 *     sign-symmetric codebooks. Where two workgroups share the rows (k = 8192 above m = 16,
 *     k > 8192, narrow layers) it first zeroes y and they add their halves of K into each output.
 *   - the wavefront-reduced GEMV for the rest of m <= 8 unless m >= 3 and m * n > 65536, and unless
 *     the activations do not fit its registers;
 *   - up to m = 128 for the rest: a K-quartered MFMA GEMM for sign-symmetric codebooks at m > 96 and
 *     n >= 4096 unless ceil(n / 64) <= 256, else the stepped dequantize-into-MFMA skinny GEMM;
 *   - above m = 128: the prefill MFMA GEMM (k < 2^22, n < 2^21), the K-quartered one (n >= 4096,
 *     sign-symmetric codebooks) or the stepped one, whichever a model of their times rates cheapest.
 * The stepped kernel runs in the launch shape a cost model rates cheapest among those whose grid
 * is on the chip at once (at most 256 workgroups): 64- or 128-row workgroups, batch blocks of 16
 * to 128 rows (to 64 for 8-bit codes and codebooks that are not sign-symmetric), and K in one part
 * or (from k = 4096) in two, where y is zeroed first and each part adds into it; with none that
 * fits, 128-row workgroups with the largest batch blocks. The prefill kernel's batch blocks (64 to
 * 256 rows) and K parts (one or two) come from its model likewise. logbq_linear_path reports the
 * path, and logbq_linear_kernel the kernel. Results are deterministic for every path.
 * k == 0 writes zeros. Errors: INVALID_ARG, UNSUPPORTED (k % 32, alignment, or k >= 2^24 on
 * the stepped or K-quartered MFMA kernel), HIP.
 */
int32_t logbq_linear(const uint16_t* x_dev, int64_t m, int64_t k, const uint8_t* codes_dev,
                     int64_t n, const float* codebook, float* y_dev, void* stream);

/*
 * logbq_linear_multi -- y_i = x . W_hat_i^T for 1 <= count <= 4 linears that share the same
 * activations (the query / key / value projections of a decoder layer, or its gate and up
 * projections), with one launch for the linears that take the GEMV in the same configuration
 * (wavefronts per row and chunks per lane, chosen from m, k and the linear's n) and one for
 * those that take the split-K kernel in the same configuration (chosen from m, k and the
 * linear's n, when their codebooks are sign-symmetric) (Sec. 3.3 lookup + product).
 *   x_dev, m, k : as logbq_linear; every W_i has k in features.
 *   count       : number of linears, 1..4.
 *   codes_dev   : host array of count device pointers, [n[i]][k/2] packed codes each.
 *   n           : host array of count out-feature counts (0 allowed).
 *   codebooks   : host array of count host pointers to 16 floats each.
 *   y_dev       : host array of count device pointers, [m][n[i]] float32 each.
 * Each y_i equals, bit for bit, what logbq_linear would write for the same operands.
 * Errors: INVALID_ARG (count outside 1..4, null arrays or entries), UNSUPPORTED, HIP.
 */
int32_t logbq_linear_multi(const uint16_t* x_dev, int64_t m, int64_t k, int32_t count,
                           const uint8_t* const* codes_dev, const int64_t* n,
                           const float* const* codebooks, float* const* y_dev, void* stream);

/*
 * logbq_dequantize -- Dequant (Eq. 2) of packed codes into float32 weights, by lookup.
 *   codes_dev : device, [n][k/2]; codebook: host, 16 floats; w_dev: device, [n][k] float32.
 * Bit-exact: w[n][k] = codebook[code(n, k)]. Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int32_t logbq_dequantize(const uint8_t* codes_dev, int64_t n, int64_t k, const float* codebook,
                         float* w_dev, void* stream);

/*
 * logbq_linear8 -- y = x . W_hat^T on 8-bit codes (Sec. 3.1 at n = 8, Sec. 3.3 lookup).
 *   x_dev     : device, [m][k] IEEE float16 activations.
 *   m, k      : batch rows and in features; k % 32 == 0, m <= 4194240.
 *   codes_dev : device, [n][k] 8-bit codes.
 *   n         : out features.
 *   codebook  : host, 256 floats (logbq_params.codebook of an 8-bit fit); rounded to float16
 *               after a common power-of-two scaling, as for logbq_linear.
 *   y_dev     : device, [m][n] float32, written.
 * Float32 accumulation. For k in {2048, 4096, 8192} a split-K dequantize-into-MFMA kernel
 * takes 5 <= m <= 8 unless n <= 1024 at k >= 4096, m = 3, 4 at n >= 8192, and 9 <= m <= 16
 * unless n > 16384 at k = 8192; at any other 512 <= k <= 8192 it takes 3 <= m <= 16 on the widths
 * where it is the faster. Otherwise the GEMV runs for m <= 8 unless m >= 5 and
 * m * n > 65536; up to m = 128 a K-quartered MFMA GEMM for m > 64 at n >= 16384 and the stepped
 * dequantize-into-MFMA skinny GEMM for the rest, in its cost-model launch shape (as for
 * logbq_linear; with K in two parts y is zeroed first); above m = 128 the prefill MFMA GEMM
 * (k < 2^22, n < 2^21), the K-quartered one (n >= 16384) or the stepped one, as for logbq_linear.
 * Results are deterministic.
 * Errors: as logbq_linear.
 */
int32_t logbq_linear8(const uint16_t* x_dev, int64_t m, int64_t k, const uint8_t* codes_dev,
                      int64_t n, const float* codebook, float* y_dev, void* stream);

/*
 * logbq_fit_uniform -- s, z, codebook and encoding thresholds of the asymmetric linear
 * baseline (Sec. 2, Quant(s, z, x)) for one tensor, from its full value range. Host only.
 *   w_host : host, numel float32 weights (any layout).
 *   bits   : 4.
 *   out    : host, filled on success.
 * Codes are decided in float64 as round(x / s) - z (ties up), clamped to 0 .. 15; the
 * thresholds reproduce that decision exactly with float32 comparisons.
 * Errors: INVALID_ARG (null, numel < 2), UNSUPPORTED (bits != 4), NONFINITE (NaN / Inf),
 * DEGENERATE (all weights equal).
 */
int32_t logbq_fit_uniform(const float* w_host, int64_t numel, int32_t bits, logbq_uniform* out);

/*
 * logbq_encode_uniform -- 4-bit asymmetric linear codes of float32 weights on the GPU:
 * code(x) = number of thresholds at or below x (NaN gives 0). Packing and layout as
 * logbq_encode ([n][k/2] bytes, low nibble = even k), but a nibble is the unsigned code q.
 * The codes run through logbq_linear / logbq_dequantize with u->codebook.
 *   w_dev     : device, [n][k] float32.   codes_dev : device, [n][k/2] bytes, written.
 *   u         : host, from logbq_fit_uniform (bits 4, thresholds non-decreasing).
 * Errors: INVALID_ARG, UNSUPPORTED (k % 32, alignment, bits), HIP.
 */
int32_t logbq_encode_uniform(const float* w_dev, int64_t n, int64_t k, const logbq_uniform* u,
                             uint8_t* codes_dev, void* stream);

/*
 * logbq_gptq -- GPTQ post-training calibration (the calibration used for every model in Sec. 4)
 * of one weight matrix with a fixed 4-bit codebook in its inner loop: LogbQuant (Eq. 1-2, from
 * `p`) or the asymmetric linear baseline (Sec. 2, from `uniform`). Columns are quantized in
 * order in blocks of 128; after column i, err = (w_i - q_i) / U_ii is subtracted, times U_ij,
 * from every later column j of its block, and after the block sum_i err_i U_ij from every
 * later column. All arithmetic is float32 in a fixed order, with no fused multiply-add:
 * err = (w - q) / U_ii; in the block w_j = w_j - err * U_ij; after it acc = acc + err_i * U_ij
 * over the block's columns in increasing i from 0, then w_j = w_j - acc.
 *   w_dev     : device, [n][k] float32, in/out. On return column i holds the value it had
 *               when it was quantized (the error-compensated weights).
 *   u_dev     : device, [k][k] float32 row-major: the upper Cholesky factor U of the damped
 *               inverse Hessian, H^-1 = U^T U (only j >= i is read; U_ii > 0).
 *   p, uniform: host; exactly one is non-NULL (bits 4). Its codebook is fixed for the whole
 *               loop (fit it on the original weights).
 *   err_dev   : device, [n][128] float32 workspace owned by the caller (overwritten).
 *   codes_dev : device, [n][k/2] packed codes, written (layout as logbq_encode; nibbles are
 *               sign + magnitude for LogbQuant, the unsigned code for the baseline).
 * Enqueues 2 * ceil(k / 128) kernels on `stream`. Errors: INVALID_ARG (null pointers, both or
 * neither of p / uniform, bad thresholds), UNSUPPORTED (bits, k % 32, alignment,
 * n > 1048560), HIP.
 */
int32_t logbq_gptq(float* w_dev, int64_t n, int64_t k, const float* u_dev, const logbq_params* p,
                   const logbq_uniform* uniform, float* err_dev, uint8_t* codes_dev,
                   void* stream);

/*
 * logbq_gptq_noalloc -- logbq_gptq without a caller-provided workspace, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc). Same arguments, results (bit for bit) and kernels as logbq_gptq, except
 * err_dev: the [n][128] float32 error workspace is a fixed array in the library's code object,
 * 8 MiB per device, held by every GPU the library runs on until the process ends.
 *   w_dev, n, k, u_dev, p, uniform, codes_dev, stream: as logbq_gptq; n <= 16384.
 * Allocates nothing (no hipMalloc, hipFree or allocating library call); the first call on a
 * device looks up the array's device address once. Every call on a GPU uses that GPU's one
 * array: calls that overlap on one GPU (e.g. on two streams) race and must be serialised by
 * the caller. Each call writes every workspace entry it reads, so no clearing is needed.
 * Errors: as logbq_gptq, and UNSUPPORTED for n > 16384.
 */
int32_t logbq_gptq_noalloc(float* w_dev, int64_t n, int64_t k, const float* u_dev,
                           const logbq_params* p, const logbq_uniform* uniform,
                           uint8_t* codes_dev, void* stream);

/* Kernel that logbq_linear (bits 4) or logbq_linear8 (bits 8) runs for a call of a shape. */
typedef enum logbq_path {
  LOGBQ_PATH_NONE = 0,     /* m or n is 0 (nothing written) or k is 0 (zeros written)        */
  LOGBQ_PATH_GEMV = 1,     /* wavefront-reduced GEMV with the LDS pair table                  */
  LOGBQ_PATH_MFMA = 2,     /* stepped dequantize-into-MFMA skinny GEMM                        */
  LOGBQ_PATH_SPLITK = 3,   /* split-K dequantize-into-MFMA kernel (4-bit, 2 <= m <= 32; 8-bit,
                              3 <= m <= 16); above m = 16 a 4-bit codebook that is not
                              sign-symmetric runs the stepped kernel instead, and where k is
                              not 1, 2, 4, 8 or 14 Ki the GEMV or the stepped kernel          */
  LOGBQ_PATH_MFMA_KQ = 4,  /* K-quartered dequantize-into-MFMA GEMM (4-bit, m > 96, n >= 4096;
                              8-bit, m > 64, n >= 16384; above m = 128 where it is rated the
                              cheapest); a 4-bit codebook that is not sign-symmetric (never a
                              fitted one) runs the stepped or the prefill kernel              */
  LOGBQ_PATH_MFMA_PF = 5   /* dequantize-into-MFMA GEMM of prefill (m > 128, k < 2^22, n < 2^21,
                              where it is rated the cheapest)                                 */
} logbq_path;

/*
 * logbq_linear_path -- the kernel a logbq_linear / logbq_linear8 call of shape (m, k, n)
 * runs with a fitted (sign-symmetric) codebook (Sec. 3.3 product; the choice is this library's,
 * not the method's). Host only: needs no device and touches none. The choice depends on (bits, m,
 * k, n) and the codebook's kind alone, so every linear of a logbq_linear_multi call runs what a
 * call of its own would run; logbq_linear_kernel tells the kernel for any codebook.
 *   bits     : 4 or 8.
 *   m, k, n  : as logbq_linear; k % 32 == 0.
 *   path_out : host, one int32, written with a logbq_path on success.
 * Errors: INVALID_ARG (null path_out, negative size), UNSUPPORTED (bits, k % 32, m too large).
 */
int32_t logbq_linear_path(int32_t bits, int64_t m, int64_t k, int64_t n, int32_t* path_out);

/*
 * logbq_linear_kernel -- name of the kernel instance (with its template arguments, as a
 * profiler lists it) that reads the codes in a logbq_linear / logbq_linear8 call of shape
 * (m, k, n), e.g. "k_gemv<4, 1, 4, false, 2>" (Sec. 3.3 product; the choice is this
 * library's); a call whose K comes in two parts launches k_fill_zero before it.
 * Host only: needs no device and touches none.
 *   bits, m, k, n : as logbq_linear_path; n fits in int32.
 *   codebook      : host, 2^bits floats, or NULL for a fitted (sign-symmetric) codebook; the
 *                   4-bit MFMA kernels dequantize in registers only for sign-symmetric ones.
 *   name_out      : host, name_len bytes, receives a NUL-terminated name ("none" for an empty
 *                   call, "k_fill_zero" for k = 0).
 * Errors: INVALID_ARG (null name_out, buffer too short, negative size, non-finite codebook
 * entry), UNSUPPORTED (bits, k % 32, m or n too large).
 */
int32_t logbq_linear_kernel(int32_t bits, int64_t m, int64_t k, int64_t n, const float* codebook,
                            char* name_out, int64_t name_len);

/*
 * logbq_dequantize8 -- Dequant (Eq. 2) of 8-bit codes: w[n][k] = codebook[codes[n][k]].
 *   codes_dev : device, [n][k]; codebook: host, 256 floats; w_dev: device, [n][k] float32.
 * Bit-exact. Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int32_t logbq_dequantize8(const uint8_t* codes_dev, int64_t n, int64_t k, const float* codebook,
                          float* w_dev, void* stream);

/*
 * ---- A serving step around the linears: paged 4-bit key/value cache, attention over it, and the
 * log probabilities of the step's tokens. The paper leaves the cache in 16 bits and names its
 * quantization as future work; the format here is this library's.
 *
 * Cache format. One layer's cache holds `pages` pages of `page` tokens each, for `heads` key/value
 * heads of `dim` channels. A token sits in slot = page id * page + offset. A row (one token's keys
 * or values of one head) is dim codes of 4 bits and one bfloat16 scale. A code is a nibble
 * sign<<3 | magnitude, as the weight codes are; it stands for
 *   +-(0, 0.5, 1, 1.5, 2, 3, 4, 6)[magnitude] * scale,
 * the values that gfx950 converts from 4 bits in one instruction.
 *   scale     = the smallest bfloat16 s with 6 s >= max |x| over the row's finite elements
 *               (0 for a row without a finite nonzero element; its codes are 0);
 *   magnitude = number of thresholds t in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5) with |x| >= t s;
 *   NaN has magnitude 0, +-Inf the largest with its sign; the sign bit is set only for a nonzero
 *   magnitude.
 * Buffers (device, 16-byte aligned, owned by the caller):
 *   k_codes   [pages][heads][page][dim/2]            low nibble = even channel
 *   v_codes   [pages][heads][page/8][16][8][dim/32]  8 tokens interleaved: 16 groups of dim/16
 *                                                    channels, each with its 8 tokens in turn
 *   k_scales, v_scales  [pages][heads][page]         bfloat16
 * dim is 64, 128 or 256; page a power of two, 16 to 1024; 1 <= heads <= 1024.
 * Device-held indices (slots, page ids, lengths, starts) are checked in the kernels: no value of
 * theirs makes a call read or write outside the buffers.
 */
typedef enum logbq_dtype {
  LOGBQ_DTYPE_F32 = 0,
  LOGBQ_DTYPE_F16 = 1,
  LOGBQ_DTYPE_BF16 = 2
} logbq_dtype;

typedef struct logbq_kv4 {
  uint8_t* k_codes;
  uint8_t* v_codes;
  uint16_t* k_scales;
  uint16_t* v_scales;
  int64_t pages;
  int32_t heads;
  int32_t page;
  int32_t dim;
  int32_t reserved;
} logbq_kv4;

/*
 * logbq_batch_tables -- block tables, slot map and starts of a step from its requests' lengths,
 * in one launch.
 *   cached_dev : device, [requests] int32, tokens that each request has in the cache.
 *   new_dev    : device, [requests] int32, tokens that it adds in this step. Negative lengths
 *                count as 0.
 *   requests   : 0 .. 4096.
 *   free_dev   : device, [free_count] int32 ids of free pages, taken from the front, request by
 *                request.
 *   table_dev  : device, [requests][width] int32, in/out. Request r has its ceil(cached / page)
 *                first entries; entries up to ceil((cached + new) / page) are written.
 *   page       : tokens in a page, a power of two, 16 .. 1024.
 *   tokens     : entries of slots_dev and positions_dev (at least the sum of new; tokens past the
 *                sum get slot -1 and position 0).
 *   slots_dev     : device, [tokens] int64, written: slot of each new token, request by request.
 *   positions_dev : device, [tokens] int32, written: its position in its request.
 *   q_starts_dev  : device, [requests + 1] int32, written: first token of each request (at most
 *                   `tokens`).
 *   seq_lens_dev  : device, [requests] int32, written: cached + new.
 *   info_dev      : device, [4] int32, written: sum of new, pages taken from the free list,
 *                   largest cached + new, and a sum of 1 (free pages were short), 2 (a request
 *                   needs more than `width` pages) and 4 (`tokens` is less than the sum of new).
 * A token without a page has slot -1, and a missing page's entry is -1. Lengths, positions and
 * sums saturate at 2^31 - 1.
 * A second call on the same input lengths gives the same results. No output may overlap an input
 * (cached_dev, new_dev, free_dev).
 * Errors: INVALID_ARG (null pointer, negative size, overlap), UNSUPPORTED (page, requests > 4096, width or
 * free_count or tokens above 2^31 - 1), HIP.
 */
int32_t logbq_batch_tables(const int32_t* cached_dev, const int32_t* new_dev, int64_t requests,
                           const int32_t* free_dev, int64_t free_count, int32_t* table_dev,
                           int64_t width, int32_t page, int64_t tokens, int64_t* slots_dev,
                           int32_t* positions_dev, int32_t* q_starts_dev, int32_t* seq_lens_dev,
                           int32_t* info_dev, void* stream);

/*
 * logbq_tree_tables -- ancestor masks and positions of a step's drafted trees (speculative decode), from the
 * nodes' parents. The new tokens of a request are the nodes of its tree, in an order in which parents come
 * before their children, at most 64.
 *   parents_dev  : device, [tokens] int32: the parent's index among the request's tokens. A negative one, or one
 *                  that is not before the node itself, stands for the request's last cached token.
 *   tokens       : entries of parents_dev and of the outputs.
 *   q_starts_dev : device, [requests + 1] int32, first token of each request.
 *   seq_lens_dev : device, [requests] int32, cached tokens with the nodes.
 *   masks_dev    : device, [tokens] uint64, written: bit j is set where node j of the request is the node
 *                  itself or an ancestor.
 *   positions_dev : device, [tokens] int32, written: the node's position in its text, seq_len - nodes + depth
 *                  (0 where that is negative). Its slot in the cache goes by its index instead (logbq_batch_tables).
 * Tokens of a request past its 64th have mask 0 and position 0; what belongs to no request is left as it was.
 * No output may overlap an input or the other output.
 * Errors: INVALID_ARG (null pointer, negative size, overlap), UNSUPPORTED (sizes), HIP.
 */
int32_t logbq_tree_tables(const int32_t* parents_dev, int64_t tokens, const int32_t* q_starts_dev,
                          const int32_t* seq_lens_dev, int64_t requests, uint64_t* masks_dev,
                          int32_t* positions_dev, void* stream);

/*
 * logbq_kv4_append -- keys and values of `tokens` tokens, quantized into their slots.
 *   k_dev, v_dev : device, row t of head h at element t * stride + h * dim; 16-byte aligned, and
 *                  so is every row (stride in elements, at least heads * dim).
 *   dtype        : logbq_dtype of both.
 *   tokens       : fewer than 2^28 - 16.
 *   cache        : host, the buffers; codes and scales of the slots are written.
 *   slots_dev    : device, [tokens] int64, distinct. A token whose slot is negative or past the
 *                  cache is left out. What a slot holds that two tokens name is not specified: its
 *                  codes and scales, of keys and values and of each head, are stored one by one and
 *                  may be of either token. No other slot is touched.
 * Errors: INVALID_ARG, UNSUPPORTED (dim, page, dtype, tokens, alignment, stride), HIP.
 */
int32_t logbq_kv4_append(const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                         int32_t dtype, int64_t tokens, const logbq_kv4* cache,
                         const int64_t* slots_dev, void* stream);

/* Rotation of queries and keys by their positions. Pair i of a head's first 2 * pairs channels is turned by
 * position * inv_freq[i] and multiplied by `factor`; the channels after them stay as they are.
 *   (u, v) -> factor (u cos - v sin, v cos + u sin)
 */
typedef struct logbq_rotation {
  const float* inv_freq;   /* device, [pairs]                                               */
  int32_t pairs;           /* 0 .. dim / 2, a multiple of dim / 16; 0 turns nothing          */
  int32_t interleaved;     /* 0: pair i is channels i and i + pairs; 1: 2 i and 2 i + 1      */
  double factor;
} logbq_rotation;

/*
 * logbq_qk_rotate -- RMS norm of each head of the queries and keys, and their rotation, in one pass.
 *   q_dev, k_dev : device, row t of head h at element t * stride + h * dim; 16-byte aligned, and so is every
 *                  row. k_heads (or q_heads) 0 leaves keys (queries) out.
 *   q_weight_dev, k_weight_dev : device, [dim] float32, 16-byte aligned: x / sqrt(mean(x^2) + eps) * weight
 *                  before the rotation; NULL: no norm.
 *   dtype        : logbq_dtype of q and k.
 *   tokens       : fewer than 2^26 - 4.
 *   dim          : 64, 128 or 256.
 *   eps          : finite, not negative.
 *   positions_dev : device, [tokens] int32 (may be NULL if the rotation has no pairs).
 *   rotation     : host. |position * inv_freq| up to 2^31 is reduced exactly.
 *   q_out_dev, k_out_dev : device, [tokens][heads][dim] of out_dtype, written; 16-byte aligned. An output may be its
 *                  own input (same type, no gaps between the tokens), and overlaps nothing else that the call reads
 *                  or writes.
 * Everything is computed in 64 bits and rounded to float32, and then to out_dtype.
 * Errors: INVALID_ARG (null pointer, negative size, eps, overlap), UNSUPPORTED (dim, pairs, dtypes, heads > 16384
 * (keys: 1024), tokens, alignment, stride), HIP.
 */
int32_t logbq_qk_rotate(const void* q_dev, int64_t q_stride, int32_t q_heads, const float* q_weight_dev,
                        const void* k_dev, int64_t k_stride, int32_t k_heads, const float* k_weight_dev,
                        int32_t dtype, int64_t tokens, int32_t dim, double eps,
                        const int32_t* positions_dev, const logbq_rotation* rotation, void* q_out_dev,
                        void* k_out_dev, int32_t out_dtype, void* stream);

/*
 * logbq_kv4_append_rotated -- logbq_qk_rotate with the keys going into the cache, and the values with them, in one
 * launch: what logbq_kv4_append would make of float32 rotated keys, and the rotated queries.
 *   q_dev .. dtype, eps, positions_dev, rotation : as logbq_qk_rotate; q_heads 0 leaves queries out. Keys and values
 *                  have the cache's heads and dim.
 *   v_dev        : device, as k_dev; values are neither normed nor turned.
 *   cache, slots_dev : as logbq_kv4_append. A token without a slot still has its query turned.
 *   q_out_dev    : device, [tokens][q_heads][dim] of out_dtype, written; q itself (as in logbq_qk_rotate) or
 *                  apart from whatever else the call reads.
 * The codes are those of the 64-bit result rounded to float32 once, so they do not depend on an order of sums.
 * Errors: as logbq_qk_rotate and logbq_kv4_append.
 */
int32_t logbq_kv4_append_rotated(const void* q_dev, int64_t q_stride, int32_t q_heads,
                                 const float* q_weight_dev, const void* k_dev, int64_t k_stride,
                                 const float* k_weight_dev, const void* v_dev, int64_t v_stride,
                                 int32_t dtype, int64_t tokens, double eps,
                                 const int32_t* positions_dev, const logbq_rotation* rotation,
                                 const logbq_kv4* cache, const int64_t* slots_dev, void* q_out_dev,
                                 int32_t out_dtype, void* stream);

/*
 * logbq_kv4_read -- the values that the cache holds in given slots, e.g. to export a prefix.
 *   slots_dev    : device, [tokens] int64; a slot that is negative or past the cache gives zeros.
 *   tokens       : fewer than 2^28 - 16.
 *   k_dev, v_dev : device, [tokens][heads][dim], written; 16-byte aligned.
 *   dtype        : logbq_dtype of both. Exact in float32, and in float16 within its range;
 *                  rounded to nearest in bfloat16.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int32_t logbq_kv4_read(const logbq_kv4* cache, const int64_t* slots_dev, int64_t tokens,
                       void* k_dev, void* v_dev, int32_t dtype, void* stream);

/* Bytes of workspace with which logbq_kv4_attention runs any call. */
#define LOGBQ_KV4_WORKSPACE_BYTES 268435456

/*
 * logbq_kv4_attention -- softmax attention of a step's queries over the 4-bit cache, for requests
 * of one token (decode), a few (speculative decode), a chunk or a whole prompt, in one call.
 *   q_dev      : device, query head h of token t at element t * q_stride + h * dim; 16-byte
 *                aligned, and so is every row.
 *   q_dtype    : logbq_dtype.
 *   tokens     : rows of q.
 *   q_heads    : a multiple of cache->heads, at most 16 times it; query head h reads key/value
 *                head h / (q_heads / heads).
 *   table_dev  : device, [requests][width] int32 page ids; a negative entry, or one past the
 *                cache, hides its page. width * page <= 2^30, and
 *                requests * heads * (width * page / 128 + 1) < 2^31.
 *   seq_lens_dev : device, [requests] int32, cached tokens with this step's, which are already
 *                appended.
 *   q_starts_dev : device, [requests + 1] int32, first token of each request.
 *   max_new    : upper bound of a request's tokens (host). Tokens of a request past it are left out:
 *                nothing is written for them, and the others are as they would be beside them.
 *   scale      : factor on the products q . k.
 *   window     : a token sees itself and the window - 1 positions before it; 0: all.
 *   out_dev    : device, [tokens][q_heads][dim], written for the tokens that belong to a request.
 *   out_dtype  : logbq_dtype.
 *   lse_dev    : device, [tokens][q_heads] float32, or NULL: log of the sum of exp(scale q . k).
 *   work_dev   : device, work_bytes bytes, 16-byte aligned, overwritten; LOGBQ_KV4_WORKSPACE_BYTES
 *                are enough for any call.
 * Token i of n new ones of a request of length s has position p = s - n + i and sees positions
 * max(0, p - window + 1) .. p (0 .. p without a window). A token that sees nothing has output 0
 * and lse -inf. What a token does not see reaches nothing of its own, whatever its scales hold.
 * Products of q are taken in float16 (float32 queries as a sum of two float16 values), all sums and
 * the softmax in float32; its weights times the values' scales are rounded to 16 bits for the
 * product with the values' codes. Logits may have any size that float32 holds; so must the products
 * of keys with queries brought below 2 (they do where |k| < 2^112), and 2^8 times the sum of |v|.
 * Requests of up to 16 query rows (tokens times q_heads / heads; 32 for dim 128, 64 for dim 64 if no
 * request of the call has more) share their positions out over the whole chip; the others go in
 * tiles of 128 rows, whose positions are split where there are few. Which way is taken goes by
 * max_new and width: a table no wider than the step's longest request serves short ones faster.
 * Results do not change from call to call. Enqueues one to four kernels.
 * Errors: INVALID_ARG, UNSUPPORTED (dim, page, heads, dtypes, alignment, sizes, a workspace that
 * is too small), HIP.
 */
int32_t logbq_kv4_attention(const void* q_dev, int64_t q_stride, int32_t q_dtype, int64_t tokens,
                            int32_t q_heads, const logbq_kv4* cache, const int32_t* table_dev,
                            int64_t requests, int64_t width, const int32_t* seq_lens_dev,
                            const int32_t* q_starts_dev, int64_t max_new, float scale,
                            int32_t window, void* out_dev, int32_t out_dtype, float* lse_dev,
                            void* work_dev, int64_t work_bytes, void* stream);

/*
 * logbq_kv4_tree_attention -- logbq_kv4_attention for a step whose new tokens are the nodes of drafted trees.
 *   masks_dev : device, [tokens] uint64 (logbq_tree_tables): bit j is set where the token sees the j-th new token of
 *               its request. Bits past the request's tokens (max_new of them at most) count for nothing. Any masks
 *               do, a tree's or not.
 *   max_new   : upper bound of a request's tokens (host), at most 64.
 *   window    : 0, or 64 at least: a token of depth d = (bits of its mask) - 1 (-1 for a mask without any) sees the
 *               cached positions past cached + d - window, and all the new tokens of its mask.
 *   The others, what is written and what a row without anything to see gets: as logbq_kv4_attention, but
 *               requests * heads * ceil(max_new * (q_heads / heads) / 128) * (width * page / 64 + 1) < 2^28.
 * A new token of a request sees all of its cached tokens (seq_len less its new tokens) that the window holds, and new
 * tokens by its mask. The new tokens' keys and values lie in the cache behind the cached ones, in order, as
 * logbq_batch_tables gives their slots. A chain (parents i - 1) gets what logbq_kv4_attention computes.
 * Errors: as logbq_kv4_attention, and UNSUPPORTED for max_new > 64 and 0 < window < 64.
 */
int32_t logbq_kv4_tree_attention(const void* q_dev, int64_t q_stride, int32_t q_dtype, int64_t tokens,
                                 int32_t q_heads, const logbq_kv4* cache, const int32_t* table_dev,
                                 int64_t requests, int64_t width, const int32_t* seq_lens_dev,
                                 const int32_t* q_starts_dev, const uint64_t* masks_dev, int64_t max_new,
                                 float scale, int32_t window, void* out_dev, int32_t out_dtype,
                                 float* lse_dev, void* work_dev, int64_t work_bytes, void* stream);

/* Most ranks of an adapter. */
#define LOGBQ_ADAPTERS_MAX_RANK 128

/* Bytes of workspace that logbq_linear_adapters needs for a call of these sizes; 0 for sizes that it does not
 * take. Host only. Grows with tokens. */
int64_t logbq_linear_adapters_workspace(int64_t tokens, int32_t count, int32_t rank);

/*
 * logbq_linear_adapters -- low-rank adapters of many requests beside up to four projections that share their
 * activations: out_i[t] = y_i[t] + scales[a] (x[t] A_i[a]^T) B_i[a]^T with a the adapter of t's request, and y_i what
 * logbq_linear or logbq_linear_multi gave.
 *   x_dev    : device, [tokens][k] float16, 16-byte aligned; k % 32 == 0.
 *   count    : projections, 1 .. 4.
 *   a_dev, b_dev : host arrays of device pointers, 16-byte aligned: A_i [adapters][rank][k], B_i
 *              [adapters][n_i][rank].
 *   n        : host array, out features of the projections (0 leaves one out; fewer than 2^24 - 1024 in all).
 *   dtype    : logbq_dtype of A and B, float16 or bfloat16.
 *   adapters : adapters in the pool.
 *   rank     : ranks that the pool has room for, a multiple of 8, at most LOGBQ_ADAPTERS_MAX_RANK.
 *   ranks_dev : device, [adapters] int32: rows of A and columns of B that an adapter has (0 .. rank; what
 *              lies past them is not used, whatever it holds). NULL: all of them have `rank`.
 *   scales_dev : device, [adapters] float32. NULL: 1.
 *   q_starts_dev : device, [requests + 1] int32, first token of each request, ascending (else what is written to the
 *              outputs is not specified).
 *   adapter_dev : device, [requests] int32: the request's adapter; one outside the pool: none.
 *   max_new  : upper bound of a request's tokens (host). Tokens of a request past it are left out.
 *   y_dev, out_dev : host arrays of device pointers, [tokens][n_i] float32. out_i may be y_i (in place), and
 *              overlaps nothing else that the call reads or writes.
 *   work_dev : device, 16-byte aligned, logbq_linear_adapters_workspace bytes at least; overwritten. Calls that
 *              overlap need one each.
 * Rows of requests without an adapter are copied (in place: left alone); rows that belong to no request are left as
 * they were. Sums are float32; x A^T goes into the second product as two float16 numbers about its largest (22
 * bits) or as three bfloat16 ones.
 * An infinity in x or y reaches the outputs as in the formula; weights are finite (an infinite one may give NaN in
 * its place). Results do not change from call to call. Enqueues one or two kernels.
 * Errors: INVALID_ARG (null pointer, negative size, count, overlap), UNSUPPORTED (dtype, k % 32, rank, alignment,
 * sizes, a workspace that is too small), HIP.
 */
int32_t logbq_linear_adapters(const uint16_t* x_dev, int64_t tokens, int64_t k, int32_t count,
                              const void* const* a_dev, const void* const* b_dev, const int64_t* n,
                              int32_t dtype, int64_t adapters, int32_t rank, const int32_t* ranks_dev,
                              const float* scales_dev, const int32_t* q_starts_dev,
                              const int32_t* adapter_dev, int64_t requests, int64_t max_new,
                              const float* const* y_dev, float* const* out_dev, void* work_dev,
                              int64_t work_bytes, void* stream);

/* Bytes of workspace that logbq_token_logprobs needs, whatever the call. */
#define LOGBQ_LOGPROBS_WORKSPACE_BYTES 4194304
/* Most alternatives that it returns. */
#define LOGBQ_LOGPROBS_MAX_TOP 32

/*
 * logbq_token_logprobs -- log probabilities of given tokens, entropy and top alternatives of
 * `tokens` rows of logits.
 *   logits_dev : device, row t at element t * stride, vocab elements; aligned to its type.
 *   dtype      : logbq_dtype.
 *   tokens     : fewer than 2^24.
 *   targets_dev : device, [tokens] int64; a target outside 0 .. vocab - 1 asks for nothing and
 *                 gives log probability 0.
 *   top        : 0 .. LOGBQ_LOGPROBS_MAX_TOP, at most vocab.
 *   logprob_dev, entropy_dev : device, [tokens] float32, written: x[target] - L and
 *                 L - sum_j exp(x_j - L) x_j with L = log sum_j exp(x_j), in nats.
 *   top_index_dev, top_logprob_dev : device, [tokens][top] int32 / float32, written: the largest
 *                 logits in descending order (equal ones by index) and their x - L. May be NULL
 *                 if top is 0.
 *   work_dev   : device, LOGBQ_LOGPROBS_WORKSPACE_BYTES bytes, 16-byte aligned. Zero before the
 *                first call; each call leaves it so. Calls that overlap need one each.
 * A logit of -inf (a forbidden token) has probability 0 and adds nothing to the entropy; it is
 * returned among the top ones only when fewer than `top` others are left, with log probability
 * -inf. Rows with a NaN, a +inf or nothing but -inf have log probabilities and entropy NaN; NaN
 * ranks above every number.
 * Sums are float32, of terms about the row's maximum: the logits' size, or an offset common to a
 * row, adds no error.
 * Errors: INVALID_ARG (null pointer, negative size, top > vocab), UNSUPPORTED (dtype, alignment,
 * tokens, vocab >= 2^31, top, stride, a workspace that is too small), HIP.
 */
int32_t logbq_token_logprobs(const void* logits_dev, int32_t dtype, int64_t tokens, int64_t vocab,
                             int64_t stride, const int64_t* targets_dev, int32_t top,
                             float* logprob_dev, float* entropy_dev, int32_t* top_index_dev,
                             float* top_logprob_dev, void* work_dev, int64_t work_bytes,
                             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LOGBQ_H */
