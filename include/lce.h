/*
 * lce.h - C ABI of the MI355X (gfx950) bitpacked binary 2-D convolution, and of
 * a 4-bit key/value cache with the attention that reads it (its own section
 * below, "4-bit key/value cache").
 *
 * The operator is LceBConv2d of Larq Compute Engine (arXiv 2011.09398,
 * Section 3.2, "Operator implementations"), preceded by the sign
 * binarization and bitpacking of LceQuantize (same section):
 *
 *   1. bitpack:   bit = 1 (standing for -1.0) iff x < 0, else 0 (+1.0);
 *                 channel c goes to 32-bit word c/32, bit c%32; the channel
 *                 count is padded up to a multiple of 32 with 0 bits.
 *   2. im2col over the bitpacked NHWC tensor, padded locations read as
 *      0 bits, i.e. +1.0 ("one-padding"), or, on request, as 0.0
 *      (TensorFlow's zero padding, through a correction step).
 *   3. XOR + POPCOUNT GEMM against bitpacked +-1 filters:
 *          dot = K - 2 * sum_k popcount(a_k XOR w_k),  K = KH*KW*C_in.
 *   4. fused output transform on the integer accumulator:
 *          c = min(max(dot, clamp_min), clamp_max)   (fused activation)
 *          float32 output:   y = fmaf((float)c, multiplier[co], bias[co])
 *          bitpacked output: bit = 1 iff c < thresholds[co] (exact compare),
 *                            optionally inverted per channel
 *
 * Conventions shared by every entry point:
 *   - All tensor pointers are DEVICE pointers owned by the caller.  The
 *     library never allocates, frees or synchronizes; all work is enqueued
 *     asynchronously on `stream` (NULL = the default stream).  Entry points
 *     that need scratch memory take it as a workspace argument.
 *   - Activations are NHWC, filters OHWI (the TensorFlow Lite orders), and a
 *     bitpacked tensor stores ceil(C/32) int32 words per pixel (or filter
 *     tap) with its packed-channel axis innermost.  Bits beyond the real
 *     channel count MUST be zero in every bitpacked input; lce_bitpack and
 *     lce_bconv2d's bitpacked output always write them as zero.
 *   - Outputs must not alias inputs.
 *   - Arguments are validated on the host before anything is launched; on
 *     any error nothing is written or launched, the status is returned, and
 *     lce_last_error() describes it.  Asynchronous device faults surface at
 *     the caller's next synchronization.  No C++ exception crosses the ABI.
 */
#ifndef LCE_H_
#define LCE_H_

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LCE_OK = 0,
    LCE_EINVAL = 1,        /* null pointer, bad size or enum, empty output   */
    LCE_EUNSUPPORTED = 2,  /* well-formed request the library does not run   */
    LCE_EALIGN = 3,        /* pointer not aligned to its element type        */
    LCE_EHIP = 4           /* the HIP runtime reported an error at launch    */
} lce_status;

/* Spatial padding, TensorFlow semantics: SAME gives ceil(H/stride) outputs
 * with floor(total/2) padding before and the rest after; VALID none. */
typedef enum { LCE_PADDING_VALID = 0, LCE_PADDING_SAME = 1 } lce_padding;

/* Value read at padded locations.  ONE (0 bits, +1.0) is the one-padding of
 * Section 3.2, the fast path.  ZERO is TensorFlow's zero padding, which the
 * same section supports through a correction step: the padded taps are
 * computed as +1.0 and their filter sums are taken out again, using the
 * table of lce_bconv2d_pad_correction. */
typedef enum { LCE_PAD_ONE = 0, LCE_PAD_ZERO = 1 } lce_pad_value;

/* Output of lce_bconv2d:
 *   FLOAT32   float  [N][OH][OW][C_out]
 *   BITPACKED int32  [N][OH][OW][ceil(C_out/32)]
 *   INT32     int32  [N][OH][OW][C_out], the clamped accumulator c itself */
typedef enum { LCE_OUT_FLOAT32 = 0, LCE_OUT_BITPACKED = 1, LCE_OUT_INT32 = 2 } lce_out_type;

/* One binary convolution.  Every field is a plain int32 (enums by value). */
typedef struct {
    int32_t n, h, w, c_in;          /* input activations, NHWC, >= 1          */
    int32_t c_out, kh, kw;          /* filters, OHWI, >= 1                    */
    int32_t stride_h, stride_w;     /* >= 1                                   */
    int32_t padding;                /* lce_padding                            */
    int32_t pad_value;              /* lce_pad_value                          */
    int32_t clamp_min, clamp_max;   /* fused activation bounds on the integer
                                       accumulator; clamp_min <= clamp_max.
                                       INT32_MIN/INT32_MAX = no activation    */
    int32_t out_type;               /* lce_out_type                           */
} lce_bconv2d_desc;

/* Number of 32-bit words holding `channels` packed channels: ceil(c/32)
 * (Section 3.2, LceQuantize: the channel count is padded up to a multiple of
 * 32 and every 32 channels become one word).  Returns -1 when channels < 0. */
int32_t lce_packed_words(int32_t channels);

/* Output height/width of `desc`.  LceBConv2d extends TensorFlow Lite's
 * convolution (Section 3, Section 3.2), so its geometry is TensorFlow's:
 * SAME gives ceil(H/stride) rows, VALID floor((H-KH)/stride)+1, and likewise
 * for the width.  Validates the descriptor exactly as lce_bconv2d does,
 * except for pointers.
 * Errors: LCE_EINVAL (null desc/oh/ow, bad field, no output). */
lce_status lce_bconv2d_out_shape(const lce_bconv2d_desc *desc, int32_t *oh, int32_t *ow);

/* LceQuantize (Section 3.2): sign-binarize and bitpack a row-major float
 * array x[rows][channels] into out[rows][ceil(channels/32)].
 * Bit c%32 of word c/32 is 1 iff x[r][c] < 0.0f (so -0.0 and NaN give 0,
 * i.e. +1.0); the bits past `channels` are written as 0.
 * For activations rows = N*H*W; for OHWI filters (the 1-bit weight storage
 * of Section 3.1) rows = C_out*KH*KW with channels = C_in.
 * rows == 0 is a no-op (pointers may then be NULL).  x must be 4-byte
 * aligned (16-byte alignment and a channel count that is a multiple of 32
 * take the fastest path), out 4-byte.
 * Errors: LCE_EINVAL (null pointer, rows < 0, channels < 1),
 *         LCE_EALIGN, LCE_EHIP. */
lce_status lce_bitpack(const float *x, int32_t *out, int64_t rows, int32_t channels,
                       hipStream_t stream);

/* LceBConv2d (Section 3.2): bitpacked binary convolution with the fused
 * output transform.
 *   x_packed   int32 [N][H][W][ceil(C_in/32)]          (device)
 *   w_packed   int32 [C_out][KH][KW][ceil(C_in/32)]    (device)
 *              The bits of a last word past C_in must be 0 in both, as
 *              lce_bitpack and a bitpacked output write them: the XOR counts
 *              every bit of a word.
 *   multiplier float [C_out] or NULL (= 1.0)   used by FLOAT32 output only
 *   bias       float [C_out] or NULL (= 0.0)   used by FLOAT32 output only
 *   thresholds float [C_out], required by BITPACKED output only
 *   flip       int32 [ceil(C_out/32)] or NULL, used by BITPACKED output
 *              only: output bits of the channels whose bit is set here are
 *              inverted (bit = NOT(c < thresholds[co])), the direction that
 *              lce_fold_thresholds derives from a negative multiplier.  Bits
 *              past C_out are ignored.
 *   pad_correction int32 table from lce_bconv2d_pad_correction for these
 *              filters; required when pad_value is ZERO and some window
 *              reaches outside the image (SAME with a nonzero total padding),
 *              ignored (may be NULL) otherwise
 *   out        see lce_out_type; shape from lce_bconv2d_out_shape
 * Dilation and groups are not part of the operator (always 1).
 * Filter shapes without a specialized XOR/POPCOUNT instance run on the matrix
 * cores (below; the same integers) where that is priced as the faster way.
 * All pointers must be 4-byte aligned.
 * Errors: LCE_EINVAL (null desc or required pointer, bad field, no output,
 *         c_out > 2^20, a tensor of 2^31 or more words/elements; with zero
 *         padding also K >= 2^29), LCE_EALIGN, LCE_EHIP. */
lce_status lce_bconv2d(const lce_bconv2d_desc *desc,
                       const int32_t *x_packed, const int32_t *w_packed,
                       const float *multiplier, const float *bias,
                       const float *thresholds, const int32_t *flip,
                       const int32_t *pad_correction, void *out, hipStream_t stream);

/* LceQuantize followed by the LceBConv2d that consumes it, in one launch
 * (Section 3.2: the float activation is sign-binarized and bitpacked, then
 * convolved).  The result equals lce_bitpack of x followed by lce_bconv2d
 * on the packed tensor, bit for bit, with no packed copy written to memory:
 * each workgroup binarizes the input rows its own windows read.  That work
 * is repeated by every filter group, so this pays at small batches, where
 * a separate lce_bitpack launch costs more than it.
 *   x          float32 [N][H][W][C_in]  (device, 16-byte aligned); the sign
 *              test is lce_bitpack's (x < 0.0f is a 1 bit = -1.0, so -0.0
 *              and NaN give +1.0)
 *   w_packed, multiplier, bias, thresholds, flip, out: as lce_bconv2d
 * Covered: C_in a multiple of 32, 3x3 filters over 32 to 192, 256 or 512
 * channels and 5x5 over 32 to 192 or 256, one padding (or a geometry with
 * no padded taps), and an input band (the input rows that the windows of
 * 64 consecutive output pixels read) that fits the LDS of a workgroup.
 * Other requests return LCE_EUNSUPPORTED before anything is launched, and
 * the caller runs lce_bitpack and lce_bconv2d instead.
 * Errors: as lce_bconv2d, plus LCE_EUNSUPPORTED (above) and LCE_EALIGN for
 *         an x that is not 16-byte aligned. */
lce_status lce_quantize_bconv2d(const lce_bconv2d_desc *desc, const float *x,
                                const int32_t *w_packed, const float *multiplier,
                                const float *bias, const float *thresholds,
                                const int32_t *flip, void *out, hipStream_t stream);

/* Number of int32 elements of the zero-padding correction table of `desc`:
 * (KH+1) * KW*(KW+1)/2 * C_out.  Validates the descriptor as lce_bconv2d
 * does.
 * Errors: LCE_EINVAL (null desc/elements, bad field). */
lce_status lce_bconv2d_pad_correction_size(const lce_bconv2d_desc *desc, int64_t *elements);

/* The correction step of zero padding (Section 3.2), prepared once per
 * filter tensor.  With S(co, ky, kx) the sum of the +-1 weights of one tap
 * and I = [x0, x1) one of the NI = KW*(KW+1)/2 non-empty column intervals
 * (numbered by x0, then x1: I = x0*(2*KW - x0 + 1)/2 + x1 - x0 - 1),
 *   pad_correction[(y*NI + I)*C_out + co] = sum over ky < y, kx in I of
 *                                           S(co, ky, kx),   y in [0, KH].
 * The in-image taps of any window form rows [y0, y1) x an interval I, so
 * lce_bconv2d takes their sum as the difference of two entries and removes
 * the padded taps' share.  w_packed as for lce_bconv2d (device, 4-byte aligned);
 * pad_correction: device int32 array of lce_bconv2d_pad_correction_size
 * elements, written asynchronously on `stream`.
 * Errors: LCE_EINVAL (null pointer, bad field, table of 2^31 or more
 *         elements), LCE_EALIGN, LCE_EHIP. */
lce_status lce_bconv2d_pad_correction(const lce_bconv2d_desc *desc, const int32_t *w_packed,
                                      int32_t *pad_correction, hipStream_t stream);

/* Converter-side threshold derivation (Sections 3.1 and 3.2: a binary
 * convolution whose float output only feeds the next layer's binarization
 * can write bits instead, compared against thresholds computed ahead of
 * time).  For each channel it returns thresholds[co] and flip bit co such
 * that, for every clamped accumulator c a convolution with K = k and
 * [clamp_min, clamp_max] can produce,
 *     (c < thresholds[co]) XOR flip[co]  ==  fmaf((float)c, m[co], b[co]) < 0,
 * i.e. lce_bconv2d's bitpacked output with (thresholds, flip) equals
 * lce_bitpack of its float output with (multiplier, bias).  A negative
 * multiplier sets the flip bit; a zero one gives a constant (+-infinity).
 * HOST pointers: multiplier, bias float [c_out] or NULL (= 1.0 / 0.0);
 * thresholds float [c_out] and flip int32 [ceil(c_out/32)] written (pad
 * bits 0).  Synchronous, no GPU work.
 * Errors: LCE_EINVAL (null output, c_out < 1, k outside [1, 2^24],
 *         clamp_min > clamp_max, a non-finite multiplier or bias). */
lce_status lce_fold_thresholds(const float *multiplier, const float *bias, int32_t c_out,
                               int32_t k, int32_t clamp_min, int32_t clamp_max,
                               float *thresholds, int32_t *flip);

/* ---- The same convolution on the matrix cores --------------------------
 *
 * LceBConv2d's dot (Section 3.2) is a dense contraction of +-1 values.  The
 * paper's XOR + POPCOUNT (lce_bconv2d) is how a CPU multiplies them; gfx950's
 * MFMA multiplies 4-bit floats, in which +1.0, -1.0 and 0.0 are exact, and
 * accumulates in fp32, exact for |dot| < 2^24, at eight times the VALU's
 * xor+popcount rate.  lce_bconv2d_mfma computes the identical result from the
 * same bitpacked activations: each bit is widened to a 4-bit +-1.0 only inside
 * the kernel.  The filters are widened once, ahead of time, into a caller-owned
 * buffer (lce_bconv2d_mfma_weights).  Zero padding needs no correction table
 * there: padded locations simply widen to 0.0. */

/* Bytes of the widened filter buffer of `desc` (20 bytes per 32 weights:
 * KH*KW x Cw' words x C_out' filters, Cw' = ceil(C_in/32) rounded up to an
 * even word count or a multiple of 4, C_out' = C_out rounded up to 32; 16
 * bytes widened and 4 bytes packed per word).
 * Errors: LCE_EINVAL (null pointer, bad field). */
lce_status lce_bconv2d_mfma_weights_size(const lce_bconv2d_desc *desc, int64_t *bytes);

/* Widen packed filters w_packed (as for lce_bconv2d, device, 4-byte aligned)
 * into w_fp4 (device, 16-byte aligned, lce_bconv2d_mfma_weights_size bytes),
 * asynchronously on `stream`.  Layout: 16-byte element (t*Cw' + j)*C_out' + co
 * holds word j of tap t of filter co as 32 e2m1 codes (+1.0 = 0x2,
 * -1.0 = 0xA), channel 32j + c in 32-bit word c % 4, nibble c / 4.  Channels
 * past C_in and filters past C_out widen to 0.0.  Then, from byte
 * 16*KH*KW*Cw'*C_out' on, the same elements as packed 32-bit words (bit 1 =
 * -1; channels past C_in, words past Cw and filters past C_out 0): the
 * streaming schedule reads these alone, for every C_in, and the
 * filter-stationary one where C_in = 32*Cw', and they widen them themselves.
 * Run once per filter tensor.
 * Errors: LCE_EINVAL, LCE_EALIGN, LCE_EHIP. */
lce_status lce_bconv2d_mfma_weights(const lce_bconv2d_desc *desc, const int32_t *w_packed,
                                    void *w_fp4, hipStream_t stream);

/* LceBConv2d on the matrix cores: arguments, output and every rounding as
 * lce_bconv2d (multiplier/bias for FLOAT32, thresholds and optional flip for
 * BITPACKED), with the widened filters in place of w_packed and either
 * pad_value (no correction table).  Bits of x_packed past C_in are ignored.
 * The work is split by shape between four schedules: filter-stationary
 * (each wave keeps its filters in registers and runs through about one
 * CU's share of pixel blocks; by default up to 36 K steps of 64
 * channels, up to 72 when an instance is forced), K-split
 * (the waves of a workgroup divide K; long K), pixel-split (the rest), and
 * streaming (tiles of pixels x filters with the filters read from the packed
 * copy step by step, any K; where many tiles make it the faster one).
 * lce_set_tuning can force a schedule, an instance or a tile for tests and
 * tuning; every choice gives the identical output.
 * w_fp4 must be the output of lce_bconv2d_mfma_weights for a descriptor with
 * the same c_in, c_out, kh and kw, 16-byte aligned and at least
 * lce_bconv2d_mfma_weights_size(desc) bytes: the kernels read the widened
 * filters and the packed copy behind them at offsets derived from `desc`
 * (the library cannot see the buffer's size; a smaller one is read past its
 * end).
 * Errors: as lce_bconv2d, plus LCE_EUNSUPPORTED when K = KH*KW*C_in >= 2^24
 * or when the input region a workgroup stages exceeds the LDS of one
 * workgroup (very wide images). */
lce_status lce_bconv2d_mfma(const lce_bconv2d_desc *desc, const int32_t *x_packed,
                            const void *w_fp4, const float *multiplier, const float *bias,
                            const float *thresholds, const int32_t *flip, void *out,
                            hipStream_t stream);

/* LceQuantize followed by the LceBConv2d that consumes it, on the matrix
 * cores in one launch (Section 3.2: the float activation is sign-binarized
 * and bitpacked, then convolved).  The result equals lce_bitpack of x
 * followed by lce_bconv2d_mfma (and so lce_bconv2d) on the packed tensor,
 * bit for bit, with no packed copy written to memory: each workgroup of the
 * filter-stationary, the K-split or the streaming schedule binarizes the
 * input region its windows read while staging it.
 *   x          float32 [N][H][W][C_in]  (device, 16-byte aligned); the sign
 *              test is lce_bitpack's (x < 0.0f is a 1 bit = -1.0, so -0.0
 *              and NaN give +1.0)
 *   w_fp4, multiplier, bias, thresholds, flip, out: as lce_bconv2d_mfma
 * Covered: C_in a multiple of 32, input below 2 GiB, and the shapes the
 * filter-stationary schedule takes (up to 72 K steps of 64 channels that
 * one of its instances covers with at most 1/8 padding; tried first up to
 * 36 K steps, and beyond where the K split's grid would not fill the CUs)
 * or, from 20 K steps, the K-split one (every 3x3 and 5x5 filter), with an
 * input region per workgroup that fits its LDS.  Other requests (e.g. 1x1
 * filters over few channels) return LCE_EUNSUPPORTED before anything is
 * launched, and the caller runs lce_bitpack and lce_bconv2d_mfma instead.
 * LCE_TUNE_MFMA_SCHEDULE 1 or 2 restricts the choice to that schedule (2
 * then takes any K); 4 takes the streaming schedule for the shapes covered
 * above; 3, the pixel split, has no fused form and is refused.
 * Errors: as lce_bconv2d_mfma, plus LCE_EUNSUPPORTED (above) and LCE_EALIGN
 *         for an x that is not 16-byte aligned. */
lce_status lce_quantize_bconv2d_mfma(const lce_bconv2d_desc *desc, const float *x,
                                     const void *w_fp4, const float *multiplier,
                                     const float *bias, const float *thresholds,
                                     const int32_t *flip, void *out, hipStream_t stream);

/* LceBMaxPool2d (Section 3.2): max pooling of +-1 activations held as
 * bits.  Since max(sign(x)) = sign(max(x)), a max pooling that feeds a
 * binarized layer can run after the binarization, on the packed tensor,
 * where the maximum of +-1 values is the bitwise AND of the window's words
 * (bit 1 = -1.0 survives only if every value in the window is -1).
 * Locations outside the image take no part (TensorFlow max pooling).  The
 * window geometry follows lce_padding like the convolution's. */
typedef struct {
    int32_t n, h, w, channels;     /* input, NHWC bitpacked, >= 1             */
    int32_t kh, kw;                /* window, >= 1                            */
    int32_t stride_h, stride_w;    /* >= 1                                    */
    int32_t padding;               /* lce_padding                             */
} lce_bmaxpool2d_desc;

/* Output height/width of `desc`.
 * Errors: LCE_EINVAL (null pointer, bad field, no output). */
lce_status lce_bmaxpool2d_out_shape(const lce_bmaxpool2d_desc *desc, int32_t *oh, int32_t *ow);

/*   x_packed int32 [N][H][W][ceil(channels/32)]    (device)
 *   out      int32 [N][OH][OW][ceil(channels/32)]  (device); pad bits 0
 * Pointers 4-byte aligned (16-byte alignment and a word count that is a
 * multiple of 4 take the widest loads).
 * Errors: LCE_EINVAL (null pointer, bad field, no output, a tensor of 2^31
 *         or more words), LCE_EALIGN, LCE_EHIP. */
lce_status lce_bmaxpool2d(const lce_bmaxpool2d_desc *desc, const int32_t *x_packed,
                          int32_t *out, hipStream_t stream);

/* LceDequantize (Section 3.2): bitpacked x_packed[rows][ceil(channels/32)]
 * back to float out[rows][channels]: -1.0f where the bit is 1, +1.0f where
 * it is 0 (the inverse of lce_bitpack's sign binarization on +-1 data).
 * rows == 0 is a no-op (pointers may then be NULL).  Pointers 4-byte
 * aligned (a channel count that is a multiple of 32 with out 16-byte aligned
 * takes the widest stores).
 * Errors: LCE_EINVAL (null pointer, rows < 0, channels < 1), LCE_EALIGN,
 *         LCE_EHIP. */
lce_status lce_dequantize(const int32_t *x_packed, float *out, int64_t rows, int32_t channels,
                          hipStream_t stream);

/* ---- 4-bit key/value cache ----------------------------------------------
 *
 * The state of a transformer held the way this library holds activations:
 * quantized as it is written, multiplied in its packed form, and read back on
 * request.  Keys and values of past tokens are 4-bit floats (e2m1: 0, 0.5, 1,
 * 1.5, 2, 3, 4, 6 and a sign) that share one power of two per 32 channels, the
 * format gfx950's matrix cores multiply directly, and every key also leaves
 * its 1-bit signs (lce_bitpack's: 1 iff x < 0), from which lce_kv4_select
 * scores pages.
 *
 * Quantization of 32 channels x of one token and head:
 *     e = max(floor(log2(max |x|)) - 2, -127)
 *     code = x / 2^e rounded to the nearest e2m1 value, ties to the even code,
 *            |x| / 2^e > 6 to 6;  the value held is code * 2^e
 * (the shared-scale 4-bit format of the OCP Microscaling specification).  A
 * group that holds an infinity or a NaN gets codes 0 and the scale NaN (255),
 * and a token with such a group in its key or its value gets key codes 0 and
 * key scales NaN: every row that attends to it is NaN, and no other row.
 *
 * The cache is one device buffer of pages of LCE_KV4_PAGE = 64 tokens, each
 * page holding a record of 76*D bytes per head (D = head_dim, G = D/32), with
 * token t of the page at
 *     key codes    byte  t*D/2 + c/2                           (channel c, low
 *     value codes  byte  32*D + ((t/4*16 + r)*4 + t%4)*G + w/2  nibble first;
 *                        r = c / (D/16), w = c % (D/16))
 *     key scales   byte  64*D + (t%16*G + c/32)*4 + t/16       (2^(byte-127))
 *     value scales byte  66*D + (c/32)*64 + t%16/4*16 + t/16*4 + t%4
 *     key signs    byte  68*D + t*D/8 + c/8, bit c%8
 * The order of the value codes is that of the matrix cores' operand: a lane
 * finds D/16 channels of four consecutive tokens in 4*G consecutive bytes.
 * Tokens are addressed by slot = page*64 + t.  A sequence is a row of page
 * numbers (its table) and a length; its token j is in slot
 * table[j/64]*64 + j%64. */
#define LCE_KV4_PAGE 64

typedef enum { LCE_FLOAT32 = 0, LCE_FLOAT16 = 1, LCE_BFLOAT16 = 2 } lce_float_type;

typedef struct {
    int32_t pages;       /* pages of the buffer, >= 1                        */
    int32_t kv_heads;    /* heads of keys and values, >= 1                   */
    int32_t head_dim;    /* channels of a head: 64, 128 or 256               */
} lce_kv4_cache_desc;

/* Bytes of the cache buffer of `desc`: pages * kv_heads * 76 * head_dim.  Its
 * contents need no initialization: slots that were never written may hold
 * anything as long as no length covers them.
 * Errors: LCE_EINVAL (null pointer, bad field), LCE_EUNSUPPORTED (head_dim). */
lce_status lce_kv4_cache_size(const lce_kv4_cache_desc *desc, int64_t *bytes);

/* Quantize `tokens` keys and values into the cache.
 *   cache  buffer of lce_kv4_cache_size bytes             (device, 16-byte aligned)
 *   k, v   [tokens][kv_heads][head_dim] of `type`         (device, 16-byte aligned),
 *          channels contiguous; token and head strides in elements, each a
 *          multiple of 16 bytes
 *   slots  int64 [tokens], where each goes (device, 8-byte aligned); a slot
 *          outside [0, 64*pages) drops its token.  A slot must not be named
 *          twice in one call.
 * tokens == 0 is a no-op (pointers may then be NULL).
 * Errors: LCE_EINVAL (null pointer, bad field, tokens < 0 or >= 2^31),
 *         LCE_EUNSUPPORTED (head_dim, kv_heads > 65535), LCE_EALIGN (pointer
 *         or stride), LCE_EHIP. */
lce_status lce_kv4_append(const lce_kv4_cache_desc *desc, void *cache, int32_t type,
                          const void *k, int64_t k_token_stride, int64_t k_head_stride,
                          const void *v, int64_t v_token_stride, int64_t v_head_stride,
                          const int64_t *slots, int64_t tokens, hipStream_t stream);

/* Read tokens back: k and v [tokens][kv_heads][head_dim] of `type`, contiguous
 * (device, 16-byte aligned), get the values that the cache holds for `slots`,
 * zeros for a slot outside the cache.  float32 and bfloat16 hold every value
 * exactly; float16 rounds those below 2^-23 to the nearest multiple of 2^-24 and
 * has infinities for those of 65536 and more.
 * Errors: as lce_kv4_append. */
lce_status lce_kv4_read(const lce_kv4_cache_desc *desc, const void *cache, const int64_t *slots,
                        int64_t tokens, int32_t type, void *k, void *v, hipStream_t stream);

/* New tokens that attend over cached sequences: `tokens` query rows, those of
 * sequence b at q_start[b] .. q_start[b+1]-1, which are the sequence's last
 * ones: with n of them, number i stands at position p = lengths[b] - n + i
 * (the cache already holds their own keys and values). */
typedef struct {
    int32_t tokens;        /* query tokens over all sequences, >= 0                    */
    int32_t q_heads;       /* a multiple of kv_heads; head hq reads cache head
                              hq / (q_heads / kv_heads)                                */
    int32_t seqs;          /* sequences, >= 1                                          */
    int32_t table_width;   /* page numbers per row of the table, >= 1                  */
    int32_t type;          /* LCE_FLOAT16 or LCE_BFLOAT16: q and out                   */
    int32_t causal;        /* 1: position p sees tokens j <= p; 0: all of the sequence */
    int32_t window;        /* > 0: only tokens j > p - window; 0: no such bound        */
    int32_t list;          /* > 0: page numbers per token and head in `pages`          */
    int32_t max_q;         /* hints for the split of the work, 0 = unknown: the most   */
    int32_t max_len;       /* new tokens, the longest length.  Wrong ones cost speed.  */
    float scale;           /* of the scores, finite and > 0                            */
    int64_t q_token_stride, q_head_stride;   /* elements, multiples of 8               */
} lce_kv4_query_desc;

/* Bytes of workspace that lce_kv4_attention, lce_kv4_select, or both calls with
 * these tokens or fewer, q_heads, seqs and table_width can need (the other
 * fields do not matter): 128 KiB, and for attention at most 36 MB (heads of 64:
 * 18, of 256: 69) of partial results, for selection 2 bytes for each token, cache
 * head and page of the table.  The workspace is 16-byte aligned device memory
 * whose first LCE_KV4_WORKSPACE_ZERO bytes are zero before its first use; each
 * call leaves them zero.  Calls that may run at the same time need one each.
 * Errors: LCE_EINVAL (null pointer, bad field), LCE_EUNSUPPORTED (head_dim, as
 *         lce_kv4_attention). */
#define LCE_KV4_WORKSPACE_ZERO 131072
lce_status lce_kv4_attention_workspace_size(const lce_kv4_cache_desc *desc,
                                            const lce_kv4_query_desc *query, int64_t *bytes);
lce_status lce_kv4_select_workspace_size(const lce_kv4_cache_desc *desc,
                                         const lce_kv4_query_desc *query, int64_t *bytes);
lce_status lce_kv4_workspace_size(const lce_kv4_cache_desc *desc, const lce_kv4_query_desc *query,
                                  int64_t *bytes);

/* Attention of new tokens over the cache: per token and query head
 *     s_j = scale * (q . k_j) over the visible tokens j,
 *     out = sum_j softmax(s)_j v_j,   lse = log sum_j exp(s_j)
 * with k and v as the cache holds them.  Products of queries and keys are exact
 * of channels that are at least 2^-13 of the largest |q| of their group (of 32
 * channels, as they share a scale in a key); smaller ones are held to 2^-21 of
 * it (float16: 2^-25).  Sums, the running maximum and the running sum are
 * float32; softmax weights are rounded to `type` where they multiply the values
 * (float16: with a last place of at most 2^-31 of a row's largest weight), and
 * out is rounded to it once.
 * A row that sees nothing is 0 with lse -infinity.
 *   q       [tokens][q_heads][head_dim] of query->type (device, 16-byte aligned)
 *   table   int32 [seqs][table_width]  (device): a row's pages; entries past a
 *           length are not read; tokens on a page outside the cache are hidden
 *   q_start int32 [seqs+1], not decreasing, lengths int32 [seqs] (device);
 *           values outside [0, tokens] and [0, 64*table_width] are taken as the
 *           nearest bound
 *   pages   with query->list > 0, int32 [tokens][kv_heads][list] (device): only
 *           tokens j on the pages j/64 named here are visible; numbers that
 *           are negative or past the length name nothing; naming a page twice
 *           counts it twice.  Otherwise ignored
 *   out     [tokens][q_heads][head_dim] of query->type, contiguous (device,
 *           16-byte aligned); rows of no sequence are left as they are
 *   lse     float32 [tokens][q_heads] or NULL
 *   workspace, workspace_bytes: see lce_kv4_attention_workspace_size
 * A query row that holds an infinity or a NaN gives NaN.  With LCE_FLOAT16,
 * cached values of 65536 and more count as 65504, the largest float16 (and
 * -65536 and less as -65504), not as the infinities that lce_kv4_read makes of
 * them; what shares a scale with them is not affected.  Those below 2^-23 count
 * as the nearest multiple of 2^-24.
 * Errors: LCE_EINVAL (null pointer, bad field, small workspace),
 *         LCE_EUNSUPPORTED (head_dim, type, more than 65535 kv_heads, a
 *         table_width or a list over 2^24, more rows or tiles than a grid
 *         holds),
 *         LCE_EALIGN, LCE_EHIP. */
lce_status lce_kv4_attention(const lce_kv4_cache_desc *desc, const void *cache,
                             const lce_kv4_query_desc *query, const void *q, const int32_t *table,
                             const int32_t *q_start, const int32_t *lengths, const int32_t *pages,
                             void *out, float *lse, void *workspace, int64_t workspace_bytes,
                             hipStream_t stream);

/* Choose query->list pages for each new token and cache head, by the signs of
 * queries and keys.  A page scores
 *     max over its visible tokens j of  sum over the query heads g of the
 *     cache head, and the channels c, of  sgn(q_gc) * sgn(k_jc)
 * (an XOR and a population count; sgn = -1 iff x < 0).  With n pages up to the
 * last visible token, the pages below keep_first and those from n - keep_last
 * on rank before all others; then higher scores, and lower page numbers among
 * equal ones.  pages int32 [tokens][kv_heads][list] (device) gets the chosen
 * page numbers in ascending order, then -1.  Pages on which the window leaves
 * nothing, or that the table names outside the cache, are not chosen.
 * The other arguments as for lce_kv4_attention (workspace: see
 * lce_kv4_select_workspace_size).
 * Errors: as lce_kv4_attention, plus LCE_EINVAL (list < 1, keep < 0) and
 *         LCE_EUNSUPPORTED (q_heads / kv_heads * head_dim > 65280). */
lce_status lce_kv4_select(const lce_kv4_cache_desc *desc, const void *cache,
                          const lce_kv4_query_desc *query, const void *q, const int32_t *table,
                          const int32_t *q_start, const int32_t *lengths, int32_t keep_first,
                          int32_t keep_last, int32_t *pages, void *workspace,
                          int64_t workspace_bytes, hipStream_t stream);

/* ---- 8-bit key/value cache ----------------------------------------------
 *
 * The same cache with a byte a channel, for models that lose too much in four bits:
 * 8-bit floats (e4m3: a sign, four bits of exponent, three of mantissa; multiples of
 * 2^-9 up to 448) that share one power of two per LCE_KV8_BLOCK = 16 tokens of a head,
 * one for its keys and one for its values.
 *
 * A block's scale is the smallest power of two, of 2^-126 and more, with which no
 * channel of the tokens that one call appends to it is past 448, or the scale that the
 * block had, where it holds older tokens and that is larger:
 *     code = x / scale rounded to the nearest e4m3 value, ties to even;
 *     the value held is code * scale.
 * Where a call raises the scale of a block that holds older tokens, their codes are
 * rounded once more, to the new scale's values (which changes only those below 2^-6 of
 * it).  A token that holds an infinity or a NaN in its key or its value gets the NaN
 * code in all channels of its key, and 0 for what is not finite in its value: every row
 * that attends to it is NaN, and no other row.
 *
 * The cache is one device buffer of pages of LCE_KV8_PAGE = 64 tokens, each page
 * holding a record of 128*D + 128 bytes per head (D = head_dim), with token t of the
 * page at
 *     key codes     byte  t*D + c                       (channel c)
 *     value codes   byte  64*D + (t/4*D + c)*4 + t%4
 *     key scales    byte  128*D + t/16                  (2^(byte-127))
 *     value scales  byte  128*D + 4 + t/16
 * and 120 bytes that nothing uses, so that records begin with a line of memory.  A
 * sequence is a row of page numbers (its table) and a length; its token j is in slot
 * table[j/64]*64 + j%64. */
#define LCE_KV8_PAGE 64
#define LCE_KV8_BLOCK 16

typedef struct {
    int32_t pages;       /* pages of the buffer, >= 1                        */
    int32_t kv_heads;    /* heads of keys and values, >= 1                   */
    int32_t head_dim;    /* channels of a head: 64, 128 or 256               */
} lce_kv8_cache_desc;

/* Bytes of the cache buffer of `desc`: pages * kv_heads * 128 * (head_dim + 1).  Its
 * contents need no initialization: what was never written may be anything as long as
 * no length covers it.
 * Errors: LCE_EINVAL (null pointer, bad field), LCE_EUNSUPPORTED (head_dim). */
lce_status lce_kv8_cache_size(const lce_kv8_cache_desc *desc, int64_t *bytes);

/* Quantize the last tokens of sequences into the cache: `tokens` rows of keys and
 * values, those of sequence b at q_start[b] .. q_start[b+1]-1; with n of them, number i
 * is the sequence's token lengths[b] - n + i (lengths count the new tokens).
 *   cache  buffer of lce_kv8_cache_size bytes             (device, 16-byte aligned)
 *   k, v   [tokens][kv_heads][head_dim] of `type`         (device, 16-byte aligned),
 *          channels contiguous; token and head strides in elements, each a
 *          multiple of 16 bytes
 *   table, q_start, lengths   as for lce_kv8_attention
 * Tokens before a sequence's beginning (n > lengths[b]) and tokens on a page outside
 * the cache are dropped.  Older tokens of a block are those before its first new one;
 * what a block holds behind the last new one is lost.  No two sequences may append to
 * one block in a call, nor one that has a page twice.  Appending the same tokens again, nothing having been appended
 * behind them, changes nothing.
 * tokens == 0 is a no-op (pointers may then be NULL).
 * Errors: LCE_EINVAL (null pointer, bad field, tokens < 0), LCE_EUNSUPPORTED
 *         (head_dim, kv_heads > 65535, table_width over 2^24, more blocks than a grid
 *         holds), LCE_EALIGN (pointer or stride), LCE_EHIP. */
lce_status lce_kv8_append(const lce_kv8_cache_desc *desc, void *cache, int32_t type,
                          const void *k, int64_t k_token_stride, int64_t k_head_stride,
                          const void *v, int64_t v_token_stride, int64_t v_head_stride,
                          int32_t tokens, int32_t seqs, int32_t table_width, const int32_t *table,
                          const int32_t *q_start, const int32_t *lengths, hipStream_t stream);

/* Read tokens back: k and v [tokens][kv_heads][head_dim] of `type`, contiguous
 * (device, 16-byte aligned), get the values that the cache holds for `slots` (int64
 * [tokens], device), zeros for a slot outside the cache.  float32 holds every value
 * exactly, bfloat16 those of 2^-126 and more; float16 rounds those below 2^-20 to the
 * nearest multiple of 2^-24 and has infinities for those of 65536 and more.
 * Errors: LCE_EINVAL (null pointer, bad field, tokens < 0 or >= 2^31), LCE_EUNSUPPORTED
 *         (head_dim, kv_heads > 65535), LCE_EALIGN, LCE_EHIP. */
lce_status lce_kv8_read(const lce_kv8_cache_desc *desc, const void *cache, const int64_t *slots,
                        int64_t tokens, int32_t type, void *k, void *v, hipStream_t stream);

/* New tokens that attend over cached sequences (see lce_kv4_query_desc). */
typedef struct {
    int32_t tokens;        /* query tokens over all sequences, >= 0                    */
    int32_t q_heads;       /* a multiple of kv_heads; head hq reads cache head
                              hq / (q_heads / kv_heads)                                */
    int32_t seqs;          /* sequences, >= 1                                          */
    int32_t table_width;   /* page numbers per row of the table, >= 1                  */
    int32_t type;          /* LCE_FLOAT16 or LCE_BFLOAT16: q and out                   */
    int32_t causal;        /* 1: position p sees tokens j <= p, and a prefix; 0: all   */
    int32_t window;        /* > 0: only tokens j > p - window; 0: no such bound        */
    int32_t max_q;         /* hints for the split of the work, 0 = unknown: the most   */
    int32_t max_len;       /* new tokens, the longest length.  Wrong ones cost speed
                              (and max_q says how weights are rounded: see below)      */
    float scale;           /* of the scores, finite and > 0                            */
    float softcap;         /* 0: none, or what scores are capped at, 1e-30 .. 1e30     */
    int64_t q_token_stride, q_head_stride;   /* elements, multiples of 8               */
} lce_kv8_query_desc;

/* Bytes of workspace that lce_kv8_attention calls with these tokens or fewer, q_heads,
 * seqs and table_width can need (the other fields do not matter): 128 KiB, and at most
 * 36 MB (heads of 64: 18, of 256: 69) of partial results.  The workspace is 16-byte
 * aligned device memory whose first LCE_KV8_WORKSPACE_ZERO bytes are zero before its
 * first use; each call leaves them zero.  Calls that may run at the same time need one
 * each.
 * Errors: LCE_EINVAL (null pointer, bad field), LCE_EUNSUPPORTED (head_dim, as
 *         lce_kv8_attention). */
#define LCE_KV8_WORKSPACE_ZERO 131072
lce_status lce_kv8_workspace_size(const lce_kv8_cache_desc *desc, const lce_kv8_query_desc *query,
                                  int64_t *bytes);

/* Attention of new tokens over the cache: per token (position p) and query head
 *     s_j = scale * (q . k_j)                        over the visible tokens j,
 *     s_j = softcap * tanh(s_j / softcap)            with a softcap,
 *     s_j = s_j - slopes[head] * |p - j|             with slopes,
 *     out = sum_j softmax(s)_j v_j,   lse = log sum_j exp(s_j)
 * with k and v as the cache holds them.  Token j is visible where j <= p or j <
 * prefix[b] (causal) or anywhere in the sequence (not causal), and j > p - window where
 * there is a window.  Sums, scores, the running maximum and the running sum are
 * float32, and out is rounded to `type` once (float16: what is past 65504 to that).
 * Softmax weights are rounded to `type` where they multiply the values (float16: with a last
 * place of at most 2^-31 of a row's largest weight).  Where max_q (0: the mean number of) new
 * tokens make up to 64 rows of a cache head, results are divided by the sum of the rounded
 * weights; and of a sequence's rows of a cache head (its tokens times the query heads that
 * share it, in that order) the last ones, if they are up to 8 more than a multiple of 16,
 * have weights of two parts of `type`, which is next to float32 ones.  A row's bits may so
 * depend on how many rows its sequence has and on max_q, as on the split of the work.
 * With LCE_FLOAT16, keys are multiplied as multiples of 2^-32 times the largest scale of
 * their page, or of less, values as multiples of 2^-32 times the largest scale that a row's
 * sequence has: this rounds only what is under a scale 2^-22 times as large.  With
 * LCE_BFLOAT16 the same holds of 2^-126, and products are summed in float32 before their
 * scales are multiplied in: queries of 2^111 and more may pass its range.
 * A row that sees nothing is 0 with lse -infinity.
 *   q       [tokens][q_heads][head_dim] of query->type (device, 16-byte aligned)
 *   table   int32 [seqs][table_width]  (device): a row's pages; entries past a
 *           length are not read; tokens on a page outside the cache are hidden
 *   q_start int32 [seqs+1], not decreasing, lengths int32 [seqs] (device);
 *           values outside [0, tokens] and [0, 64*table_width] are taken as the
 *           nearest bound
 *   slopes  float32 [q_heads] (device) or NULL
 *   prefix  int32 [seqs] (device) or NULL; values outside [0, length] as the nearest
 *   out     [tokens][q_heads][head_dim] of query->type, contiguous (device,
 *           16-byte aligned); rows of no sequence are left as they are
 *   lse     float32 [tokens][q_heads] or NULL
 *   workspace, workspace_bytes: see lce_kv8_workspace_size
 * A query row that holds an infinity or a NaN gives NaN.
 * Errors: LCE_EINVAL (null pointer, bad field, small workspace),
 *         LCE_EUNSUPPORTED (head_dim, type, more than 65535 kv_heads, a
 *         table_width over 2^24, more rows or tiles than a grid holds),
 *         LCE_EALIGN, LCE_EHIP. */
lce_status lce_kv8_attention(const lce_kv8_cache_desc *desc, const void *cache,
                             const lce_kv8_query_desc *query, const void *q, const int32_t *table,
                             const int32_t *q_start, const int32_t *lengths, const float *slopes,
                             const int32_t *prefix, void *out, float *lse, void *workspace,
                             int64_t workspace_bytes, hipStream_t stream);

/* ---- Rotary positions -----------------------------------------------------
 *
 * Queries and keys turned by their tokens' positions, before keys are appended to a
 * cache and queries attend to it.  Of a head's first rot_dim channels, pair i is
 * channels (i, i + rot_dim/2), or (2i, 2i + 1) interleaved; at position p
 *     (a, b) -> scale * (a cos(p f_i) - b sin(p f_i), b cos(p f_i) + a sin(p f_i)),
 * the channels behind them stay as they are.  Frequencies f_i are radians a position:
 * the caller's own, or those of lce_rotary_frequencies. */
typedef enum {
    LCE_ROTARY_PLAIN = 0,    /* f_i = base^(-2i / rot_dim)                             */
    LCE_ROTARY_LINEAR = 1,   /* f_i / factor                                           */
    LCE_ROTARY_NTK = 2,      /* base times factor^(rot_dim / (rot_dim - 2))            */
    LCE_ROTARY_YARN = 3      /* by parts: pairs that turn more than 32 times over
                                `original` positions keep f_i, those that turn less than
                                once have f_i / factor, a linear mixture by pair number
                                between; scale = 0.1 ln(factor) + 1                    */
} lce_rotary_scaling;

/* Frequencies (host, double [rot_dim/2]) of a scaling for contexts `factor` >= 1 times
 * as long as trained (`original` positions; yarn alone looks at it), and the scale
 * that goes with them.  Yarn's `original` is 7 or more: the first pair's whole turn.
 * Errors: LCE_EINVAL. */
lce_status lce_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                                  double original, double *freqs, float *scale);

/* The form in which lce_rotary takes frequencies (both host, [count]): turns a position
 * in multiples of 2^-64, whole turns left out.  Frequencies of up to one turn a position are
 * rounded to the nearest, larger ones to the last place of a 64-bit mantissa; position times
 * what that leaves is exact.
 * Errors: LCE_EINVAL (null pointer, count < 1, a frequency that is not finite). */
lce_status lce_rotary_turns(const double *freqs, int32_t count, uint64_t *turns);

typedef struct {
    int32_t tokens;        /* >= 0                                                     */
    int32_t head_dim;      /* channels of a head, 2 .. 65536                           */
    int32_t rot_dim;       /* of which so many are turned: even, 2 .. head_dim         */
    int32_t type;          /* lce_float_type of x and y                                */
    int32_t interleaved;   /* 0: pairs (i, i + rot_dim/2); 1: (2i, 2i + 1)             */
    int32_t backward;      /* 1: the other way: x are gradients of the results, y those
                              of what was turned                                       */
    float scale;           /* finite                                                   */
} lce_rotary_desc;

/* Heads of one tensor, read from x and written to y: channels contiguous, strides in
 * elements.  y may be x (with the same strides); other overlaps are not allowed.  Rows of
 * y do not lie between each other: its smaller stride is head_dim or more, its larger one
 * all that the rows of the other axis take, or more.  Of two tensors, neither's y overlaps
 * the other's x or y. */
typedef struct {
    int32_t heads;         /* >= 1                                                     */
    const void *x;
    void *y;
    int64_t x_token_stride, x_head_stride, y_token_stride, y_head_stride;
} lce_rotary_rows;

/* Turn `q`, and `k` unless it is NULL, in one launch.
 *   turns      uint64 [rot_dim/2] (device): see lce_rotary_turns
 *   positions  int64 [tokens] (device), any values
 * Angles of position p are known to 2^-33 + 0.6 |p| 2^-64 turns (frequencies of up to one
 * turn a position: 2^-32 for the first 2^32 positions), and products are float32, rounded
 * once to `type`.
 * rot_dim a multiple of 32 bytes, head_dim of 16, and x, y and strides of 16 bytes take
 * the widest loads; others work.
 * tokens == 0 is a no-op (pointers may then be NULL).
 * Errors: LCE_EINVAL (null pointer, bad field), LCE_EUNSUPPORTED (more than 2^20 heads
 *         or than a grid holds), LCE_EALIGN (pointers not aligned to their type),
 *         LCE_EHIP. */
lce_status lce_rotary(const lce_rotary_desc *desc, const uint64_t *turns, const int64_t *positions,
                      const lce_rotary_rows *q, const lce_rotary_rows *k, hipStream_t stream);

/* ---- Schedule overrides, for tests and tuning ----------------------------
 *
 * Every convolution picks its work split by itself.  These process-wide
 * overrides force one instead; each choice gives the identical output (of
 * lce_kv4_attention and lce_kv8_attention: the same but for the order of their
 * float32 sums), only
 * the speed changes.  0 (the initial value of every key) restores the
 * library's own choice.  Callers are tests, benchmarks and tuning scripts,
 * not production code.  Values are read once per launch with atomic loads,
 * so setting them while other threads launch is safe (a launch sees either
 * the old or the new value).  An out-of-range value falls back to the
 * automatic choice where the key's comment says so. */
typedef enum {
    LCE_TUNE_XOR_NB = 0,          /* lce_bconv2d: blocks of 8 filters per wave, 1..4    */
    LCE_TUNE_XOR_KS = 1,          /* lce_bconv2d: waves sharing a block's K range 1/2/4 */
    LCE_TUNE_MFMA_SCHEDULE = 2,   /* lce_bconv2d_mfma and lce_quantize_bconv2d_mfma:
                                     1 filter-stationary (where an instance fits),
                                     2 K split, 3 pixel split (not fused), 4 streaming
                                     (where a tile fits)                                */
    LCE_TUNE_MFMA_FS_KS = 3,      /* filter-stationary instance: K steps per wave       */
    LCE_TUNE_MFMA_FS_S = 4,       /* filter-stationary instance: waves per filter block */
    LCE_TUNE_MFMA_FS_WPC = 5,     /* filter-stationary and streaming grids: 1 or 2 workgroups
                                     per CU                                             */
    LCE_TUNE_MFMA_FS_PAD = 6,     /* -1: no LDS claim that spreads workgroups over CUs  */
    LCE_TUNE_MFMA_PACKED = 7,     /* -1: load widened filters where packed ones would do */
    LCE_TUNE_MFMA_TILE_M = 8,     /* K-split / pixel-split tile: 32-pixel blocks;
                                     streaming: 32-pixel blocks per wave, 2 or 4        */
    LCE_TUNE_MFMA_TILE_N = 9,     /* K-split / pixel-split / streaming tile: 32-filter
                                     blocks                                             */
    LCE_TUNE_MFMA_FS_WINDOW = 10, /* -1: filter-stationary workgroups stage whole padded
                                     rows, also where a share's window of columns would do */
    LCE_TUNE_XOR_STREAM = 11,     /* lce_bconv2d, filter shapes without a specialized XOR
                                     instance: 1 the streaming schedule (where a tile
                                     fits; tile and grid keys as above), -1 the XOR kernel */
    LCE_TUNE_KV4_CHUNK = 12,      /* lce_kv4_attention, lce_kv4_select: pages per
                                     workgroup, >= 1 (raised where the workspace has no
                                     room for that many workgroups)                     */
    LCE_TUNE_KV4_ROWS = 13,       /* lce_kv4_attention without a list: 16, 32 or 128 query
                                     rows per tile, where there is such a kernel (heads
                                     of up to 128; 32 not of 128 in float16)            */
    LCE_TUNE_KV8_CHUNK = 14,      /* lce_kv8_attention: pages per workgroup, as above      */
    LCE_TUNE_KV8_ROWS = 15,       /* lce_kv8_attention: 16, 32 or 128 query rows per tile, where
                                     there is such a kernel                                */
    LCE_TUNE_COUNT = 16
} lce_tuning_key;

/* Set override `key` to `value` (0 = automatic).
 * Errors: LCE_EINVAL (unknown key). */
lce_status lce_set_tuning(int32_t key, int32_t value);

/* Current value of override `key` (0 for an unknown key). */
int32_t lce_get_tuning(int32_t key);

/* Message describing the last error on the calling thread ("" if none). */
const char *lce_last_error(void);

/* What the calling thread's last convolution or lce_kv4_attention or
 * lce_kv8_attention call that got as far as a launch ran, for tests and tuning: "xor", "xor-generic",
 * "xor-quantize", "filter-stationary", "k-split", "pixel-split", "streaming" or
 * "streaming-stored" (lce_bconv2d on the matrix cores); "kv4-16", "kv4-32" or
 * "kv4-128" by the rows of a tile, "kv4-list", "kv8-16", "kv8-32" or "kv8-128", each
 * with "-split" behind it where a tile's pages may be divided; "" before any. */
const char *lce_last_schedule(void);

#ifdef __cplusplus
}
#endif

#endif /* LCE_H_ */
