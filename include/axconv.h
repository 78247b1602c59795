/*
 * axconv -- table-lookup quantized conv2d / dense for AMD MI355X (gfx950).
 *
 * Emulates a DNN accelerator whose MAC unit has an 8-bit (approximate) multiplier and a
 * 32-bit accumulator: every product of an 8-bit activation code and an 8-bit filter code
 * is taken from a truth table of 256 x 256 16-bit entries (128 kB), summed exactly in
 * int32, then dequantized (paper: Sec. II, Eq. (1)-(4) and the MAC model; Sec. III,
 * tensor layouts and the table addressed by the two stitched codes).
 *
 * Conventions for every entry point
 *   - Tensor pointers (x, w, lut, acc_out, y_out, workspace) are DEVICE pointers owned by
 *     the caller.  `q` is a HOST pointer and is read before the call returns.
 *   - Calls only enqueue work on `hip_stream` (a hipStream_t passed as void*, NULL = the
 *     default stream).  They never synchronize, allocate or free.
 *   - Outputs are overwritten completely.  Either of acc_out / y_out may be NULL to skip
 *     it (not both).  Inputs must not alias outputs or the workspace.
 *   - `workspace` holds per-call scratch (re-laid-out table, packed operands, partial
 *     sums).  Its contents need not be preserved between calls, but two calls that run
 *     concurrently on different streams need separate workspaces.  The required size is
 *     returned by the matching *_workspace_bytes function; a smaller buffer is an error.
 *   - Return value: AX_OK (0) or a negative AX_ERR_* code; ax_strerror() gives text.
 *     Nothing is printed, thrown or aborted.
 *   - The library keeps no mutable process-wide state: tuning overrides travel with the call
 *     (ax_tune_t) or with a layer handle, so calls from several host threads do not interact.
 *
 * Micro-benchmarks and kernel timing helpers are declared in axconv_probe.h, not here.
 */
#ifndef AXCONV_H
#define AXCONV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define AX_OK 0
#define AX_ERR_NULL (-1)       /* a required pointer is NULL                                   */
#define AX_ERR_SHAPE (-2)      /* non-positive dimension, stride < 1, pad < 0, empty output,
                                  or a tensor with 2^31 or more elements                       */
#define AX_ERR_QUANT (-3)      /* zero point / pad code outside [0,255] (pad_code may be -1),
                                  scale not finite or not positive                             */
#define AX_ERR_K_OVERFLOW (-4) /* KH*KW*Cin > 32768: the int32 accumulator could overflow
                                  (32769 * 65535 > 2^31 - 1)                                   */
#define AX_ERR_WORKSPACE (-5)  /* workspace NULL, too small or not 256-byte aligned            */
#define AX_ERR_HIP (-6)        /* a HIP runtime call failed (launch, attribute, event)         */
#define AX_ERR_ALIGN (-7)      /* a tensor pointer is not aligned to its element size          */
#define AX_ERR_OPTION (-8)     /* a flag, round mode or tuning value out of range              */
#define AX_ERR_STATE (-9)      /* layer handle used before ax_layer_prepare                    */

/* Affine quantization parameters, real = scale * (code - zero_point)  (Eq. (1)).
 * x_* are alpha_1 / beta_1 of the activations, w_* are alpha_2 / beta_2 of the filters
 * (Eq. (3)).  pad_code is the activation code that taps outside the image feed through
 * the multiplier table; -1 selects x_zp, the code of the real value zero (Sec. II). */
typedef struct {
  float x_scale;
  int32_t x_zp;
  float w_scale;
  int32_t w_zp;
  int32_t pad_code;
} ax_quant_t;

/*
 * Approximate 2-D convolution (Sec. III, Algorithm 1 without the float quantization step:
 * operands arrive as 8-bit codes).
 *
 *   x        [N, H, W, Cin]       uint8, channels fastest
 *   w        [KH, KW, Cin, Cout]  uint8, filter count fastest
 *   lut      [65536]              uint16, entry index = x_code * 256 + w_code
 *   acc_out  [N, OH, OW, Cout]    int32:  acc = sum over the KH*KW*Cin taps of lut[...]
 *   y_out    [N, OH, OW, Cout]    float:  y = x_scale * w_scale *
 *                (acc - w_zp * Sp - x_zp * Sf + K * x_zp * w_zp),
 *            Sp = sum of the patch's activation codes (padded taps included), Sf = sum of
 *            the channel's filter codes, K = KH*KW*Cin: the integer expansion of Eq. (3)
 *            with the table in place of the product (Eq. (4)).
 *   OH = floor((H + 2*pad_h - KH) / stride_h) + 1, OW likewise.  Dilation is 1.
 *
 * acc_out is bit-exact; y_out is float(corr) * (x_scale * w_scale) in float arithmetic.
 */
int ax_conv2d(const uint8_t* x, int N, int H, int W, int Cin, const uint8_t* w, int KH, int KW,
              int Cout, const uint16_t* lut, int stride_h, int stride_w, int pad_h, int pad_w,
              const ax_quant_t* q, int32_t* acc_out, float* y_out, void* workspace,
              size_t workspace_bytes, void* hip_stream);

size_t ax_conv2d_workspace_bytes(int N, int H, int W, int Cin, int KH, int KW, int Cout,
                                 int stride_h, int stride_w, int pad_h, int pad_w);

/*
 * Approximate dense layer / matrix product (Eq. (2)-(4)); identical to ax_conv2d with
 * H = W = KH = KW = 1, Cin = K, Cout = N and M images.
 *   x [M, K] uint8 row major, w [K, N] uint8 row major, acc_out / y_out [M, N].
 */
int ax_dense(const uint8_t* x, int M, int K, const uint8_t* w, int N, const uint16_t* lut,
             const ax_quant_t* q, int32_t* acc_out, float* y_out, void* workspace,
             size_t workspace_bytes, void* hip_stream);

size_t ax_dense_workspace_bytes(int M, int K, int N);

/* ---- operator variants (Sec. III, Algorithm 1: the layer's dilation parameter next to the
 * strides; Sec. II: signed multipliers with codes in [-128, 127] next to unsigned ones, and an
 * approximate twin for each kind of 2-D convolution, of which the depthwise and the grouped ones
 * are built here and the transposed one further down) ----- */

/* pad_code value that selects the activation zero point in both the unsigned and the signed
 * form (-1 selects it too, but only for unsigned codes, where -1 is no code). */
#define AX_PAD_DEFAULT INT32_MIN

typedef struct {
  int32_t N, H, W, Cin; /* input  [N, H, W, Cin]                                              */
  int32_t KH, KW, Cout; /* filters [KH, KW, Cin, Cout], or [KH, KW, Cin, Cout/Cin] (depthwise) */
  int32_t stride_h, stride_w, pad_h, pad_w;
  int32_t dilation_h, dilation_w; /* >= 1; tap (ky, kx) reads pixel (oy*stride_h - pad_h +
                                     ky*dilation_h, ox*stride_w - pad_w + kx*dilation_w);
                                     OH = floor((H + 2*pad_h - dilation_h*(KH-1) - 1)/stride_h) + 1 */
  int32_t depthwise;    /* 0: ordinary convolution.  1: output channel ci*mult + m (mult =
                           Cout/Cin, Cout a multiple of Cin) sums over the KH*KW taps of input
                           channel ci only, so K = KH*KW in the correction                     */
  int32_t signed_codes; /* 0: x, w uint8, lut uint16.  1: x, w int8, lut int16 with entry index
                           (uint8_t)x_code * 256 + (uint8_t)w_code (the two's-complement patterns
                           stitched together); zero points and pad_code in [-128, 127]         */
  int32_t groups;       /* 0 or 1: ordinary.  n >= 2 (depthwise must be 0): grouped convolution,
                           Cin and Cout multiples of n; input and output channels are cut into n
                           contiguous blocks and output block g sums over the taps of input block
                           g only: filters [KH, KW, Cin/n, Cout], K = KH*KW*Cin/n in the
                           correction.  Grouped layers run on the direct kernel (functional, not
                           tuned); the backward pass does not take them.                        */
} ax_conv_desc_t;

/*
 * Tuning overrides for one call or one layer handle.  Every field 0 (or a NULL pointer where a
 * tune is accepted) selects the automatic choice; results never depend on them (integer addition
 * is associative), only run time does.  The tests force them to reach every kernel path.
 *   variant      1 = direct kernel: table read from global memory, one thread per output or, for
 *                    few outputs, 4, 16 or 64
 *                2 = table-tile kernel, lanes over output pixels
 *                3 = table-tile kernel, lanes over output channels
 *   split_k      n >= 1 (at most 64): n equal workgroup shares per output tile (n slices of the
 *                sum over the taps)
 *   tile         n >= 1: table-tile configuration n (greatest height of a tile in lane elements)
 *   row_tiles    1 = as few tiles along the lane dimension as fit, n >= 2 = n tiles (clamped to
 *                what the layer allows; at most 2^20)
 *   share_order  1 = workgroups take their shares of the work in launch order, 2 = XCD by XCD
 *                (every XCD, with its own L2, gets a contiguous run of tiles)
 *   combine      output tiles whose sum over the taps is shared by several workgroups:
 *                1 = a second kernel adds the pieces, 2 = the workgroup that finishes a tile's
 *                last piece adds the others inside the main kernel
 *   tables       the per-tap lookup tables of the table-tile kernel (variant 2, one multiplier
 *                table): 1 = assembled inside the kernel from the rows of the multiplier table,
 *                2 = ready-made in the prepared block (4 KiB per tap and eight output channels)
 * A value out of range gives AX_ERR_OPTION.
 */
typedef struct {
  int32_t variant, split_k, tile, row_tiles, share_order, combine, tables;
} ax_tune_t;

/* ax_conv2d generalized by the descriptor; outputs, workspace rules and errors as for ax_conv2d
 * (AX_ERR_OPTION for a flag that is neither 0 nor 1).  acc_out is the exact (signed) sum.
 * tune may be NULL. */
int ax_conv2d_ex(const ax_conv_desc_t* desc, const ax_tune_t* tune, const void* x, const void* w,
                 const void* lut, const ax_quant_t* q, int32_t* acc_out, float* y_out,
                 void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_conv2d_ex_workspace_bytes(const ax_conv_desc_t* desc, const ax_tune_t* tune);

/*
 * Transposed convolution (Sec. II: an approximate twin for every kind of 2-D convolution; the
 * paper does not define this one).  Reading taken: zero insertion, as an accelerator with a fixed
 * MAC array runs it.  The input is spread out by the strides, every inserted position holding the
 * activation zero point (the code of the real value zero), and every output sums the table
 * entries of all its KH*KW*Cin taps: taps on an input pixel feed its code, taps on an inserted
 * position feed x_zp, taps outside the spread-out image feed pad_code.  With the exact
 * multiplier and the default pad code this is the transposed convolution of the common
 * frameworks on the dequantized tensors (the adjoint of ax_conv2d_ex with the same descriptor).
 *
 *   desc      N, H, W, Cin describe the INPUT, Cout the output channels, filters [KH, KW, Cin, Cout];
 *             depthwise must be 0 and groups 0 or 1 (AX_ERR_OPTION otherwise)
 *   acc_out / y_out  [N, OH, OW, Cout], OH = (H-1)*stride_h + 1 + dilation_h*(KH-1) - 2*pad_h
 *             (pad_h <= dilation_h*(KH-1), AX_ERR_SHAPE otherwise), OW likewise
 *   tap (ky, kx) of output (oy, ox) looks at position (oy + pad_h - ky*dilation_h,
 *             ox + pad_w - kx*dilation_w) of the spread-out image, whose pixel
 *             (iy*stride_h, ix*stride_w) is input pixel (iy, ix); K = KH*KW*Cin in the correction
 *
 * The workspace also holds the spread-out image and the flipped filters; the layer itself then
 * runs as an ordinary stride-1 layer (table-tile kernels included).  Other rules as for
 * ax_conv2d_ex.  Layer handles, the float form and the backward pass do not take this kind.
 */
int ax_conv2d_transpose(const ax_conv_desc_t* desc, const ax_tune_t* tune, const void* x, const void* w,
                        const void* lut, const ax_quant_t* q, int32_t* acc_out, float* y_out,
                        void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_conv2d_transpose_workspace_bytes(const ax_conv_desc_t* desc, const ax_tune_t* tune);

/*
 * One layer against several multiplier tables in one call: the use the paper builds the
 * emulator for is evaluating many candidate approximate multipliers on the same network
 * (Sec. I, Sec. V).  luts holds num_luts (1 .. 65536) tables of 65536 entries back to back;
 * acc_out / y_out hold num_luts result tensors back to back ([num_luts][N, OH, OW, Cout]),
 * each exactly what ax_conv2d gives for that table.  The operands are prepared once, and the
 * tiles of all tables form one pool of work, so that the machine is filled without cutting
 * output tiles along K.
 */
int ax_conv2d_multi_lut(const uint8_t* x, int N, int H, int W, int Cin, const uint8_t* w, int KH,
                        int KW, int Cout, const uint16_t* luts, int num_luts, int stride_h,
                        int stride_w, int pad_h, int pad_w, const ax_quant_t* q, int32_t* acc_out,
                        float* y_out, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_conv2d_multi_lut_workspace_bytes(int N, int H, int W, int Cin, int KH, int KW, int Cout,
                                           int num_luts, int stride_h, int stride_w, int pad_h,
                                           int pad_w);

/* ---- layer handles: filters and table prepared once, then many calls ---------------------
 *
 * Filters, multiplier table and quantization coefficients of a layer do not change from batch
 * to batch (Sec. III, Algorithm 1 derives everything that depends on them once per layer; Sec. I:
 * the emulator runs whole data sets through one network and one candidate multiplier).  A handle
 * fixes the layer's geometry, coefficients, number of tables and tuning; ax_layer_prepare turns
 * filters and tables into the form the kernels consume (re-laid-out table, packed filters, filter
 * sums) in a caller-owned device block; ax_layer_run then only needs the activations.  Results
 * are those of ax_conv2d_ex / ax_conv2d_multi_lut, bit for bit.
 *
 * The handle is a small host object (malloc / free); device memory stays with the caller:
 *   prepared   ax_layer_prepared_bytes() bytes, 256-byte aligned, written by ax_layer_prepare and
 *              read by every ax_layer_run until the next ax_layer_prepare (which may be given
 *              another block: e.g. two blocks to prepare the next table while the current one
 *              is still in use on another stream).  May be 0 bytes (NULL is then accepted).
 *   workspace  ax_layer_workspace_bytes() bytes of per-call scratch, as for ax_conv2d.
 * w and luts given to ax_layer_prepare must stay valid and unchanged while the handle is used:
 * layers that take the direct kernel, the depthwise kernel or the one for few output pixels
 * (ax_layer_plan: variant 1; most layers of a network at batch 1) copy nothing and read them in
 * every call.
 * A handle may be used from one host thread at a time.  Runs that use the same prepared block
 * must not overlap in time on the device (one stream, or streams ordered by events): where
 * several workgroups share an output tile the main kernel keeps the tile's arrival counter in
 * the prepared block, at zero between runs.
 */
typedef struct ax_layer ax_layer_t;

/* num_luts >= 1 tables as in ax_conv2d_multi_lut (1 for a plain layer); q and tune are copied
 * (tune may be NULL).  Errors as for ax_conv2d_ex; *layer_out is NULL on error. */
int ax_layer_create(const ax_conv_desc_t* desc, int num_luts, const ax_quant_t* q,
                    const ax_tune_t* tune, ax_layer_t** layer_out);
void ax_layer_destroy(ax_layer_t* layer); /* NULL is ignored */
size_t ax_layer_prepared_bytes(const ax_layer_t* layer);
size_t ax_layer_workspace_bytes(const ax_layer_t* layer);
/* w: filters, luts: num_luts tables back to back (device pointers, types as the descriptor says). */
int ax_layer_prepare(ax_layer_t* layer, const void* w, const void* luts, void* prepared,
                     size_t prepared_bytes, void* hip_stream);
/* x: activations; acc_out / y_out: [num_luts][N, OH, OW, Cout], either may be NULL (not both).
 * AX_ERR_STATE before the first ax_layer_prepare. */
int ax_layer_run(const ax_layer_t* layer, const void* x, int32_t* acc_out, float* y_out,
                 void* workspace, size_t workspace_bytes, void* hip_stream);
/*
 * ax_layer_run for callers that cannot allocate device memory or hand in a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The per-call scratch
 * is a device array inside the library (ax_static_scratch_bytes() = 64 MiB, held by every GPU the
 * library runs on until the process ends); the call allocates and frees nothing.  Inputs, outputs
 * and results as for ax_layer_run.  AX_ERR_WORKSPACE when the call needs more scratch than the
 * array holds (what it needs is at most ax_layer_workspace_bytes(), less when the activations can
 * be read in place: 16-byte aligned, unsigned, channel count a multiple of 16).  All calls on one
 * GPU share that GPU's array: calls that overlap in time on one GPU (different streams) race.
 */
int ax_layer_run_static(const ax_layer_t* layer, const void* x, int32_t* acc_out, float* y_out,
                        void* hip_stream);
size_t ax_static_scratch_bytes(void);

/* What the handle's calls run (host arithmetic only): variant as in ax_tune_t (1, 2 or 3), tile
 * configuration (0 for the kernels that prepare nothing: direct, few output pixels, depthwise,
 * all variant 1), grid size of the main kernel and number of partial tile pieces it produces.
 * Any output pointer may be NULL. */
int ax_layer_plan(const ax_layer_t* layer, int* variant, int* tile, int* workgroups, int* pieces);
/* The two remaining choices of the plan, in the values of ax_tune_t: combine (0: no shared tiles,
 * 1: second kernel, 2: inside the main kernel) and tables (0: not a table-tile layer, 1: assembled
 * in the kernel, 2: ready-made in the prepared block).  Any output pointer may be NULL. */
int ax_layer_plan_paths(const ax_layer_t* layer, int* combine, int* tables);

/* ---- float-in / float-out form of the layer (Sec. II: the approximate layer reads two float
 * tensors plus the range of each and returns a float tensor; Sec. III, Algorithm 1:
 * ComputeCoeffs, quantization, lookup-MAC, dequantization) ---------------------------------
 *
 * Arithmetic, every step a single IEEE float32 operation in this order:
 *   lo = min(range[0], 0), hi = max(range[1], 0)     the range is widened to hold r = 0, which
 *                                                    makes zero exactly representable (Sec. II)
 *   alpha = (hi - lo) / 255, or 1 if that is not positive
 *   beta  = clamp(round(-lo / alpha), 0, 255)
 *   code(r) = clamp(round(r / alpha) + beta, 0, 255)          (Eq. (1) solved for the code)
 * round_mode 0 rounds halves to even, 1 rounds halves away from zero (the layer's "round mode"
 * parameter, Sec. II); other values give AX_ERR_OPTION.  relu != 0 replaces r by max(r, 0)
 * first: the activation between two chained layers, fused into the pass that reads the tensor.
 * Tensor values must be finite.  Ranges live in DEVICE memory as two floats (min, max), the
 * way the minimum / maximum operators in front of the layer deliver them (Sec. II, design flow).
 */

/* One (alpha, beta) pair of Eq. (1) as the quantization kernels store it in device memory. */
typedef struct {
  float scale;
  int32_t zero_point;
} ax_coeffs_t;

/* Minimum and maximum of x[0..n), n >= 1 (AX_ERR_SHAPE otherwise): range_out[0] = min,
 * range_out[1] = max, of max(x, 0) when relu != 0.  Evaluated once per batch in front of each
 * layer (Sec. II, design flow).  workspace: ax_range_workspace_bytes(n) bytes, 256-byte aligned. */
int ax_range_f32(const float* x, size_t n, int relu, float* range_out, void* workspace,
                 size_t workspace_bytes, void* hip_stream);
size_t ax_range_workspace_bytes(size_t n);

/* codes_out[i] = code(x[i]) with the coefficients derived from `range` (device, two floats).
 * coeffs_out (device, may be NULL) receives alpha and beta.  n >= 1.  No workspace. */
int ax_quantize_f32(const float* x, size_t n, const float* range, int relu, int round_mode,
                    uint8_t* codes_out, ax_coeffs_t* coeffs_out, void* hip_stream);

/*
 * The whole layer of Algorithm 1 on float tensors:
 *   x [N,H,W,Cin] float, w [KH,KW,Cin,Cout] float, x_range / w_range device float[2],
 *   lut as for ax_conv2d; relu applies to x only.
 *   Either range pointer may be NULL: the layer then takes that tensor's minimum and maximum
 *   itself (of max(x, 0) for x when relu != 0), once per call, which is what the operators in
 *   front of the layer would deliver and saves their separate launches.
 *   (alpha1, beta1) from x_range, (alpha2, beta2) from w_range; both tensors are quantized
 *   (into the workspace); taps outside the image carry the real value 0, i.e. the code beta1;
 *   acc_out (optional) and y_out are those of ax_conv2d for these codes and coefficients:
 *   y = float(corr) * (alpha1 * alpha2), the product of the scales taken in float32.
 * workspace: ax_conv2d_f32_workspace_bytes(...) bytes; it also holds the codes and the
 * coefficients, which never visit the host.
 */
int ax_conv2d_f32(const float* x, int N, int H, int W, int Cin, const float* w, int KH, int KW,
                  int Cout, const uint16_t* lut, int stride_h, int stride_w, int pad_h, int pad_w,
                  const float* x_range, const float* w_range, int relu, int round_mode,
                  int32_t* acc_out, float* y_out, void* workspace, size_t workspace_bytes,
                  void* hip_stream);
size_t ax_conv2d_f32_workspace_bytes(int N, int H, int W, int Cin, int KH, int KW, int Cout,
                                     int stride_h, int stride_w, int pad_h, int pad_w);

/* The float layer with the layer's full parameter set (Sec. III, Algorithm 1: strides,
 * dilations, padding; Sec. II: signed or unsigned multiplier, round mode) and the depthwise kind,
 * given by the descriptor of ax_conv2d_ex; tune may be NULL.  signed_codes = 1: the same alpha; codes and zero points are
 * the unsigned ones lowered by 128 (they span [-128, 127], real zero stays representable), lut is
 * int16 addressed by the codes' two's-complement patterns.  Everything else as ax_conv2d_f32. */
int ax_conv2d_f32_ex(const ax_conv_desc_t* desc, const ax_tune_t* tune, const float* x,
                     const float* w, const void* lut, const float* x_range, const float* w_range,
                     int relu, int round_mode, int32_t* acc_out, float* y_out, void* workspace,
                     size_t workspace_bytes, void* hip_stream);
size_t ax_conv2d_f32_ex_workspace_bytes(const ax_conv_desc_t* desc, const ax_tune_t* tune);

/* Dense form: x [M,K] float, w [K,N] float (Eq. (2)-(4) after the same quantization). */
int ax_dense_f32(const float* x, int M, int K, const float* w, int N, const uint16_t* lut,
                 const float* x_range, const float* w_range, int relu, int round_mode,
                 int32_t* acc_out, float* y_out, void* workspace, size_t workspace_bytes,
                 void* hip_stream);
size_t ax_dense_f32_workspace_bytes(int M, int K, int N);

/* ---- backward pass -------------------------------------------------------------------------
 *
 * The paper says the transformed network serves training as well as inference (Sec. II, design
 * flow) but defines no gradient of the approximate layer.  Reading taken (straight-through): the
 * backward pass treats the layer as the exact convolution of the dequantized tensors of Eq. (1),
 * xr = x_scale * (x_code - x_zp), wr = w_scale * (w_code - w_zp) -- the layer with the exact
 * multiplier (Sec. IV) -- where a tap outside the image carries x_scale * (pad_code - x_zp).
 * Quantization and the multiplier's error are passed straight through.  With gy = dL/dy:
 *
 *   gx_out [N, H, W, Cin]       dL/dxr = sum over (ky, kx, co) and the output pixels (oy, ox) whose
 *                               tap (ky, kx) reads input pixel (iy, ix) of gy * wr[ky, kx, ci, co]
 *   gw_out [KH, KW, Cin, Cout]  dL/dwr = sum over (n, oy, ox) of xr(tap) * gy[n, oy, ox, co]
 *
 * x, w: codes as for ax_conv2d_ex (uint8, or int8 with signed_codes); gy: float [N, OH, OW, Cout].
 * Either output may be NULL (not both).  Sums are accumulated in float32 on the matrix cores (gy
 * split exactly into three bf16 pieces, the other operand a small integer that bf16 holds
 * exactly); each output is within 2e-5 times the sum of the absolute values of its terms of the
 * exact value.  Depthwise descriptors give AX_ERR_OPTION (not built).  workspace (always
 * needed: it holds the bf16 pieces of gy, the converted filters and the partial filter
 * gradients): ax_conv2d_backward_workspace_bytes(desc) bytes, 256-byte aligned.
 */
int ax_conv2d_backward(const ax_conv_desc_t* desc, const ax_quant_t* q, const void* x, const void* w,
                       const float* gy, float* gx_out, float* gw_out, void* workspace,
                       size_t workspace_bytes, void* hip_stream);
size_t ax_conv2d_backward_workspace_bytes(const ax_conv_desc_t* desc);

/* ---- feed-forward operators ----------------------------------------------------------------
 *
 * What a network needs around its quantized layers to be trained and to answer: the norm in front
 * of a feed-forward block with an output in 8-bit codes, matrix products with bias, activation and
 * residual in their epilogue on float tensors or on 8-bit codes, the gated block, and the step of
 * the optimizer.  They work on exact products (the matrix cores), next to the table-lookup layers.
 *
 * Element types are named by the values below.  Matrices are row major; *_ld are row pitches in
 * elements (at least the row's length).  Sums, norms and optimizer states are held in float32 (int32
 * for products of codes); results are rounded once, to nearest even, where they are stored.  Zero
 * rows (M or rows = 0) are valid: nothing is written but the sums over rows, which are zero.
 * Everything else follows the conventions above: the calls only enqueue work, outputs are
 * overwritten completely and alias no input unless that is said, 16-bit and 32-bit pointers are
 * aligned to their element.
 */
#define AX_F32 0
#define AX_BF16 1

#define AX_ACT_NONE 0
#define AX_ACT_RELU 1
#define AX_ACT_SILU 2 /* z / (1 + exp(-z)) */
#define AX_ACT_GELU 3 /* z * (1 + erf(z / sqrt 2)) / 2 */
/* Float32 results are evaluated to within 14 2^-24 (gelu) and 8 2^-24 (silu) of themselves, the far tails of gelu
 * included; results in bf16 to within 1.2e-4 and 1.2e-5 in front of their rounding. */

/*
 * Root-mean-square norm of rows with the residual's addition in front:
 *   t = x + residual            (x alone where residual is NULL), in float32
 *   rstd = 1 / sqrt(mean of t^2 over the row + eps)
 *   y = t * rstd * weight
 */
typedef struct {
  int64_t rows, cols; /* 0 <= rows < 2^31, 1 <= cols < 2^31 - 32768                             */
  int64_t x_ld, residual_ld, sum_ld, y_ld;
  int32_t dtype;      /* of x, residual, sum and y; in the backward pass of all the matrices    */
  int32_t w_dtype;    /* of weight                                                              */
  float eps;          /* >= 0 and finite                                                        */
  int32_t normalize;  /* 1.  0 (ax_rmsnorm_q8 alone): rstd = 1, plain quantization of rows      */
} ax_norm_desc_t;

/* sum_out (may be NULL; needs a residual): t, the residual stream behind the addition, rounded to
 * dtype (the norm itself takes it unrounded); it may be x or residual itself, with that tensor's
 * row pitch.  rstd_out [rows] (may be NULL): kept for the backward pass. */
int ax_rmsnorm(const ax_norm_desc_t* desc, const void* x, const void* residual, const void* weight,
               void* sum_out, void* y_out, float* rstd_out, void* hip_stream);

/*
 * The same rows as 8-bit codes, symmetric, one scale a row: with v = t * weight (one float32
 * product; v = t where weight is NULL) and amax the row's largest |v|,
 *   codes = round(v * (127 / amax)), ties to even, in [-127, 127]        scales = amax * rstd / 127
 * The codes do not depend on the order of the norm's sum: rstd scales the whole row.  A row whose
 * amax is below 2^-120 (where 127 / amax leaves float32) has codes zero.  A row that holds a NaN or an infinity has scale NaN or
 * infinity and codes zero.  codes_out [rows, cols] and scales_out [rows] are what ax_matmul_q8 and
 * ax_gated_q8 take.  values_out (may be NULL) [rows, cols] float32, pitch cols: code * scale.
 */
int ax_rmsnorm_q8(const ax_norm_desc_t* desc, const void* x, const void* residual, const void* weight,
                  void* sum_out, int8_t* codes_out, float* scales_out, float* values_out, void* hip_stream);

/*
 * Gradients of ax_rmsnorm.  t: the sum (x where there was no residual) and rstd as the forward pass
 * left them; gy [rows, cols]; gsum (may be NULL) [rows, cols]: the gradient that reaches t from the
 * residual stream.  With h = t * rstd and q = gy * weight:
 *   gx_out = rstd * (q - h * mean over the row of (q * h)) + gsum       for x and residual alike
 *   gw_out [cols] float32 = sum over the rows of gy * h
 * Pitches: desc->x_ld (t), residual_ld (gsum), sum_ld (gx_out), y_ld (gy).  gx_out may be gsum.
 * Either output may be NULL (not both, where there are rows).  The sum over rows is taken in a fixed order.
 * workspace: ax_rmsnorm_backward_workspace_bytes(desc) bytes, 256-byte aligned.
 */
int ax_rmsnorm_backward(const ax_norm_desc_t* desc, const void* gy, const void* gsum, const void* t,
                        const void* weight, const float* rstd, void* gx_out, float* gw_out,
                        void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_rmsnorm_backward_workspace_bytes(const ax_norm_desc_t* desc);

/*
 * Matrix product with its epilogue:  z = x w + bias,  y = act(z) + residual.
 *   x [M, K], w [K, N] (or [N, K] where w_transposed is 1), bias [N], residual and y [M, N],
 *   z_out (may be NULL) [M, N] with pitch N, kept for the backward pass
 * bias and residual may be NULL; y_out may be residual itself, with its pitch.  dtype is the type of x and w, out_dtype that of bias, residual, z
 * and y.  AX_BF16 products are exact in float32 and summed there.  AX_F32 operands are taken as three
 * bf16 pieces each (exact together, each rounded to nearest) and six of their nine products; what is
 * dropped is within 2^-24 (1 + 2^-8) of a product and of either sign, so results are those of a float32
 * product (but an infinity in an operand may give NaN).
 * Operands that the kernels cannot read in place (AX_F32; rows that are not 16-byte aligned or whose
 * length is no multiple of 16 bytes) are copied into the workspace first.
 * workspace: ax_matmul_workspace_bytes(desc) bytes, 256-byte aligned.
 */
typedef struct {
  int64_t M, N, K;    /* M >= 0; N, K >= 1; each at most 2^30, row pitches below 2^22 bytes      */
  int64_t x_ld, w_ld, residual_ld, y_ld;
  int32_t dtype, out_dtype;
  int32_t act;
  int32_t w_transposed;
  int32_t unaligned;  /* 0: x, w (and gy where act is AX_ACT_NONE) start on 16 bytes wherever their rows do
                         (AX_ERR_ALIGN otherwise).  1: they may start anywhere; they are copied   */
} ax_matmul_desc_t;

int ax_matmul(const ax_matmul_desc_t* desc, const void* x, const void* w, const void* bias,
              const void* residual, void* y_out, void* z_out, void* workspace, size_t workspace_bytes,
              void* hip_stream);
size_t ax_matmul_workspace_bytes(const ax_matmul_desc_t* desc);

/*
 * The product of 8-bit codes: z = (x_scales[m] * w_scales[n]) * sum over k of x[m,k] w[n,k] + bias,
 * y = act(z) + residual, the sum exact in int32.  x [M, K] and w [N, K] int8 (desc->w_transposed must
 * be 1, desc->dtype is ignored), K <= 131071 (AX_ERR_K_OVERFLOW).
 * workspace: ax_matmul_q8_workspace_bytes(desc) bytes, 256-byte aligned.
 */
int ax_matmul_q8(const ax_matmul_desc_t* desc, const int8_t* x, const float* x_scales, const int8_t* w,
                 const float* w_scales, const void* bias, const void* residual, void* y_out,
                 void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_matmul_q8_workspace_bytes(const ax_matmul_desc_t* desc);

/*
 * Gradients of ax_matmul (of its residual: gy itself).  With gz = gy * act'(z), act'(0) = 0 for relu:
 *   gx_out [M, K] = gz w^T     gw_out (the shape and pitch of w) = x^T gz     gb_out [N] float32 = sum of gz
 * gy and z [M, N] have the type desc->dtype and the pitches y_ld and N; gx_out (pitch x_ld) and gw_out
 * (pitch w_ld) too; desc->out_dtype must be desc->dtype.  z may be NULL where act is AX_ACT_NONE.  bf16: gz is
 * rounded to bf16 for the two products (their matrix instructions take 16-bit operands), not for gb_out, nor
 * for gw_out of at most 12 rows (16 where K N >= 2^22): errors of 2.3e-3 in the 2-norm where the rounding of the
 * results alone gives 1.7e-3.  Float32 operands have no such rounding.  Any output may be NULL (not all, where there are rows).
 * workspace: ax_matmul_backward_workspace_bytes(desc) bytes.
 */
int ax_matmul_backward(const ax_matmul_desc_t* desc, const void* gy, const void* x, const void* w,
                       const void* z, void* gx_out, void* gw_out, float* gb_out, void* workspace,
                       size_t workspace_bytes, void* hip_stream);
size_t ax_matmul_backward_workspace_bytes(const ax_matmul_desc_t* desc);

/*
 * Gated feed-forward block up to the product back:  g = x wg,  u = x wu,  h = act(g) * u,
 * both projections, the activation and the product in one kernel.
 *   x [M, K], wg and wu [K, N], h [M, N]; g_out, u_out [M, N] (pitch N, both or neither NULL): kept
 *   for the backward pass
 * The descriptor is that of ax_matmul: w_ld is the pitch of both weights, w_transposed must be 0,
 * residual_ld is ignored.  workspace: ax_gated_workspace_bytes(desc) bytes, 256-byte aligned.
 */
int ax_gated(const ax_matmul_desc_t* desc, const void* x, const void* wg, const void* wu, void* h_out,
             void* g_out, void* u_out, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_gated_workspace_bytes(const ax_matmul_desc_t* desc);

/* On 8-bit codes, as ax_matmul_q8: x [M, K], wg and wu [N, K] int8, w_transposed must be 1. */
int ax_gated_q8(const ax_matmul_desc_t* desc, const int8_t* x, const float* x_scales, const int8_t* wg,
                const float* wg_scales, const int8_t* wu, const float* wu_scales, void* h_out,
                void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_gated_q8_workspace_bytes(const ax_matmul_desc_t* desc);

/*
 * Gradients of ax_gated.  With gg = gh * u * act'(g) and gu = gh * act(g):
 *   gx_out [M, K] = gg wg^T + gu wu^T     gwg_out = x^T gg,  gwu_out = x^T gu     [K, N], pitch w_ld
 * gh (pitch y_ld), g, u (pitch N), gx_out (pitch x_ld): type desc->dtype; desc->out_dtype must be
 * desc->dtype.  bf16: gg and gu are rounded to bf16 for the products, as above.  gx_out may be NULL, or both
 * weight gradients.  workspace: ax_gated_backward_workspace_bytes(desc) bytes.
 */
int ax_gated_backward(const ax_matmul_desc_t* desc, const void* gh, const void* x, const void* wg,
                      const void* wu, const void* g, const void* u, void* gx_out, void* gwg_out,
                      void* gwu_out, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_gated_backward_workspace_bytes(const ax_matmul_desc_t* desc);

/*
 * One AdamW step over many tensors (decoupled weight decay, bias correction for step = 1, 2, ...).
 * For every element, each line a float32 operation at a time, factors rounded once from double:
 *   g = gradient * *grad_scale          (the gradient itself where grad_scale is NULL)
 *   m = beta1 * m + (1 - beta1) * g            v = beta2 * v + (1 - beta2) * (g * g)
 *   p = p * (1 - lr * weight_decay) - (lr / (1 - beta1^step)) * (m / (sqrt(v) * (1 / sqrt(1 - beta2^step)) + eps))
 * state_bits 32: m and v are float32.  state_bits 8: codes, one float32 scale for every 256 elements
 * in their order (AX_STATE_BLOCK; the last block of a tensor may be shorter):
 *   m = scale * r |r|, r = code / 127, code in [-127, 127], scale the block's largest |m|
 *   v = scale * (r r)^2, r = code / 255, code in [0, 255], scale the block's largest v
 * with the codes rounded to nearest in r; a v above zero never gets code 0, so that no update divides
 * by eps alone.  A block with a NaN gets scale NaN: it shows in every parameter of the block.
 */
#define AX_STATE_BLOCK 256

typedef struct {
  void* p;        /* parameters, updated in place                                              */
  const void* g;  /* gradients                                                                 */
  void* m;        /* float32, or int8 codes                                                    */
  void* v;        /* float32, or uint8 codes                                                   */
  float* m_scale; /* 8 bits: one a block                                                       */
  float* v_scale;
  void* copy;     /* may be NULL: the updated parameters once more, rounded to bf16            */
  int64_t n;      /* elements, >= 0, below 2^36                                                */
} ax_adamw_tensor_t;

typedef struct {
  double lr, beta1, beta2, eps, weight_decay;
  int64_t step;            /* >= 1                                                             */
  const float* grad_scale; /* device float, may be NULL                                        */
  int32_t p_dtype, g_dtype;
  int32_t state_bits;      /* 32 or 8                                                          */
  int32_t reserved;        /* 0                                                                */
} ax_adamw_desc_t;

/* tensors: HOST array, read before the call returns (it travels in the kernels' arguments: one launch
 * for every AX_ADAMW_LAUNCH tensors that are not empty).  Tensors must not overlap. */
#define AX_ADAMW_LAUNCH 48
int ax_adamw(const ax_adamw_desc_t* desc, const ax_adamw_tensor_t* tensors, int count, void* hip_stream);

/* The values that 8-bit states stand for, float32: m_out[i] and v_out[i] (host arrays of device
 * pointers) for tensors[i], of which p, g and copy are not looked at. */
int ax_adamw_states(const ax_adamw_tensor_t* tensors, int count, float* const* m_out, float* const* v_out,
                    void* hip_stream);

/* ---- feed-forward blocks of experts ---------------------------------------------------------
 *
 * A block whose projections come in `experts` versions, of which every token takes k: the router's choice, the products
 * of the tokens' rows with the matrix of their expert, and their sum; and, for serving, products with weights of 4 bits.  The conventions
 * are those above.
 *
 * Rows.  Every choice of a token is a row of the products.  Rows lie in the order of their experts: expert e has the rows
 * offsets[e] .. offsets[e + 1] - 1 (offsets [experts + 1], int32, device).  Sizes are ragged, an expert may have no rows;
 * rows in front of offsets[0] and from offsets[experts] on belong to nobody: they reach no product and are left as they are in the outputs, though copies
 * of operands and the elementwise part of the gradients pass over them in the workspace.  With
 * offsets that descend or leave the rows the results are not defined, but no call reads or writes outside its arrays, whatever they hold.
 */
#define AX_MAX_EXPERTS 1024
#define AX_MAX_CHOICES 16

/*
 * The router.  For every token the k largest logits, ties to the lowest expert, in descending order:
 *   experts_out [tokens, k]  int32
 *   weights_out [tokens, k]  float32: exp(l - m) / sum of exp(l - m), m the largest logit, summed over the chosen experts
 *                            (normalize = 1) or over all (0)
 *   offsets_out [experts + 1], rows_out [tokens, k], tokens_out [tokens * k], int32: the rows of the choices in the order
 *                            (expert, token, choice): the row of every choice, and the token of every row
 * A logit of minus infinity is never chosen (a mask); where fewer than k others are left, the choice is dropped: expert -1, weight 0, row
 * -1, and as many rows at the end belong to nobody (their token is -1).  Infinite logits share the weight.  A NaN is never
 * chosen either, and makes the weights of its token NaN.
 * workspace: ax_route_workspace_bytes(desc) bytes, 256-byte aligned.
 */
typedef struct {
  int64_t tokens;     /* tokens * k <= 2^30                                                     */
  int64_t ld;         /* row pitch of the logits                                                */
  int32_t experts;    /* 1 .. AX_MAX_EXPERTS                                                    */
  int32_t k;          /* 1 .. min(experts, AX_MAX_CHOICES)                                      */
  int32_t dtype;      /* of the logits and their gradient                                       */
  int32_t normalize;
} ax_route_desc_t;

int ax_route(const ax_route_desc_t* desc, const void* logits, int32_t* experts_out, float* weights_out,
             int32_t* offsets_out, int32_t* rows_out, int32_t* tokens_out, void* workspace,
             size_t workspace_bytes, void* hip_stream);
size_t ax_route_workspace_bytes(const ax_route_desc_t* desc);

/*
 * The gradient of the logits from that of the weights, through what the forward pass left.  With inner = sum over j of gw_j w_j:
 *   normalize = 1: gl[e_j] = w_j (gw_j - inner), zero elsewhere (logits may be NULL)
 *   normalize = 0: gl = p (g - inner), p the softmax over all experts, g_e_j = gw_j and zero elsewhere
 * A dropped choice has no gradient.  glogits_out [tokens, experts] at pitch glogits_ld.  No workspace.
 */
int ax_route_backward(const ax_route_desc_t* desc, const float* gweights, const void* logits, const int32_t* experts,
                      const float* weights, void* glogits_out, int64_t glogits_ld, void* hip_stream);

/*
 * Products of rows with the matrix of their expert.  Row r is row index[r] of x (an index outside x: a row of zeros), or row
 * r of x where index is NULL and desc->indexed is 0; w holds the experts' matrices one behind the other, [experts, K, N] or
 * [experts, N, K] (w_transposed), all rows at pitch w_ld:
 *   z = x w_e,  y_out = act(z),  z_out (may be NULL, pitch N) kept for the backward pass
 *   h_out = act(x wg_e) * (x wu_e),  g_out and u_out (both or neither NULL, pitch N) kept
 * Types, sums and roundings as in ax_matmul and ax_gated.
 * More than 2^23 tiles (2^29 float32 rows, say) are refused: AX_ERR_SHAPE, as in the gradients and in the products with 4-bit weights.
 * workspace: ax_*_experts_workspace_bytes(desc) bytes, 256-byte aligned.
 */
typedef struct {
  int64_t rows;       /* of the products, at most 2^30                                          */
  int64_t x_rows;     /* of x; rows where it is not indexed                                     */
  int64_t N, K;       /* experts * N and experts * K below 2^31                                 */
  int64_t x_ld, w_ld, y_ld;
  int64_t gx_ld;      /* of the rows' gradient                                                  */
  int32_t experts;    /* 1 .. AX_MAX_EXPERTS                                                    */
  int32_t dtype;      /* of all matrices                                                        */
  int32_t act;
  int32_t w_transposed; /* must be 0 for the gated pair                                         */
  int32_t indexed;    /* 1: index is given                                                      */
  int32_t unaligned;  /* as in ax_matmul_desc_t                                                 */
} ax_experts_desc_t;

int ax_matmul_experts(const ax_experts_desc_t* desc, const void* x, const int32_t* index, const int32_t* offsets,
                      const void* w, void* y_out, void* z_out, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_matmul_experts_workspace_bytes(const ax_experts_desc_t* desc);
int ax_gated_experts(const ax_experts_desc_t* desc, const void* x, const int32_t* index, const int32_t* offsets,
                     const void* wg, const void* wu, void* h_out, void* g_out, void* u_out, void* workspace,
                     size_t workspace_bytes, void* hip_stream);
size_t ax_gated_experts_workspace_bytes(const ax_experts_desc_t* desc);

/*
 * Their gradients.  gx_out [rows, K] (pitch gx_ld) is that of the rows of the products, in their order; the gradient of an indexed
 * x is the sum over its rows (ax_combine without weights).  gw_out (gwg_out, gwu_out): the experts' matrices one behind the other, at
 * the pitch of w; an expert without rows gets zeros.  Formulas, roundings and what may be NULL as in
 * ax_matmul_backward and ax_gated_backward, without the bias; bf16: gz (gg, gu) is rounded to bf16 for all products.  Without rows
 * gx_out may be NULL whatever else is.
 */
int ax_matmul_experts_backward(const ax_experts_desc_t* desc, const void* gy, const void* x, const int32_t* index,
                               const int32_t* offsets, const void* w, const void* z, void* gx_out, void* gw_out,
                               void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_matmul_experts_backward_workspace_bytes(const ax_experts_desc_t* desc);
int ax_gated_experts_backward(const ax_experts_desc_t* desc, const void* gh, const void* x, const int32_t* index,
                              const int32_t* offsets, const void* wg, const void* wu, const void* g, const void* u,
                              void* gx_out, void* gwg_out, void* gwu_out, void* workspace, size_t workspace_bytes,
                              void* hip_stream);
size_t ax_gated_experts_backward_workspace_bytes(const ax_experts_desc_t* desc);

/*
 * Back to the tokens: y_out[t] = residual[t] + sum over j of weights[t, j] * h[rows[t, j]], in float32 in the order of j.
 *   h [h_rows, cols], rows [tokens, k] int32 (a row outside h is left out), weights [tokens, k] float32 (NULL: one each),
 *   residual (may be NULL) and y_out [tokens, cols]; y_out may be residual itself, with its pitch
 */
typedef struct {
  int64_t tokens;     /* tokens * k <= 2^30                                                     */
  int64_t h_rows, cols;
  int64_t h_ld, residual_ld, y_ld;
  int64_t gh_ld;      /* of h's gradient                                                        */
  int32_t k;          /* 1 .. AX_MAX_CHOICES                                                    */
  int32_t dtype;      /* of h, residual, y and their gradients                                  */
} ax_combine_desc_t;

int ax_combine(const ax_combine_desc_t* desc, const void* h, const int32_t* rows, const float* weights,
               const void* residual, void* y_out, void* hip_stream);

/*
 * Gradients: gh_out[rows[t, j]] = weights[t, j] * gy[t] (gy at pitch y_ld; rows must differ from one another; rows of gh_out that no
 * choice names are left as they are), gweights_out[t, j] = sum over the columns of gy[t] * h[rows[t, j]], float32, zero for a row
 * outside h.  Either may be NULL (not both, where there are tokens); h is needed for gweights_out alone.  The residual's gradient is gy.
 */
int ax_combine_backward(const ax_combine_desc_t* desc, const void* gy, const void* h, const int32_t* rows,
                        const float* weights, void* gh_out, float* gweights_out, void* hip_stream);

/*
 * Weights of 4 bits with a scale for every group of a row: w[n, k] = scale[n, k / group] * code[n, k], codes -8 .. 7, scales bf16,
 * group 32, 64 or 128, [N, K] for each of `experts` matrices (1 for a plain one).  They are kept in a layout of the
 * library's own, codes and scales apart, ax_q4_codes_bytes and ax_q4_scales_bytes bytes, 16-byte aligned, at most 2^24
 * blocks of 16 x 128 in all.
 *
 * ax_quantize_q4: from float weights [experts * N, K] at pitch w_ld: scale = (largest |w| of the group / 7) rounded to bf16, code =
 * w / scale rounded to nearest, ties to even, in -8 .. 7; a group whose scale is zero or not finite has codes zero.
 * ax_pack_q4: from codes int8 [experts * N, K] (others are taken to the nearest of -8 .. 7) and scales bf16 [experts * N, ceil(K / group)].
 * ax_q4_values: the weights, float32 [experts * N, K].
 */
size_t ax_q4_codes_bytes(int64_t experts, int64_t N, int64_t K);
size_t ax_q4_scales_bytes(int64_t experts, int64_t N, int64_t K, int32_t group);
int ax_quantize_q4(const void* w, int32_t dtype, int64_t w_ld, int64_t experts, int64_t N, int64_t K, int32_t group,
                   uint8_t* codes_out, void* scales_out, void* hip_stream);
int ax_pack_q4(const int8_t* codes, const void* scales, int64_t experts, int64_t N, int64_t K, int32_t group,
               uint8_t* codes_out, void* scales_out, void* hip_stream);
int ax_q4_values(const uint8_t* codes, const void* scales, int64_t experts, int64_t N, int64_t K, int32_t group,
                 float* values_out, void* hip_stream);

/*
 * Products with such weights: y_out = act(x w^T + bias) + residual, h_out = act(x wg^T) * (x wu^T).  bias [N], residual and y_out
 * [rows, N] (both may be NULL; y_out may be residual itself) have x's type.  With several experts the rows are grouped as above (index
 * and offsets; offsets may be NULL for one expert, whose rows are then all).  The weights are exact: products with the
 * codes are exact and summed in float32, each group's sum times its scale in float32 (some sums of bf16 rows run over codes with 24 added, taken
 * off again in float32: they round as sums of terms up to six times as large, and an infinity in x, or a value beyond 2^117, may come out as a NaN).  Only for more than 600 bf16
 * rows an expert on the average, every weight is rounded to bf16 for the matrix instructions: errors of 2.1e-3 in the 2-norm where the rounding of the
 * results alone gives 1.7e-3, and a row's result depends on how many rows the call has.  Float32 rows never meet rounded weights, nor do calls of up to 600 rows.
 * workspace: ax_*_q4_workspace_bytes(desc) bytes, 256-byte aligned.
 */
typedef struct {
  int64_t rows;       /* of the products, at most 2^30                                          */
  int64_t x_rows;     /* of x; rows where it is not indexed                                     */
  int64_t N, K;
  int64_t x_ld, residual_ld, y_ld;
  int32_t experts;
  int32_t group;
  int32_t dtype;      /* of x, bias, residual and the output                                    */
  int32_t act;
  int32_t indexed;
  int32_t unaligned;
} ax_q4_desc_t;

int ax_matmul_q4(const ax_q4_desc_t* desc, const void* x, const int32_t* index, const int32_t* offsets,
                 const uint8_t* codes, const void* scales, const void* bias, const void* residual, void* y_out,
                 void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_matmul_q4_workspace_bytes(const ax_q4_desc_t* desc);
int ax_gated_q4(const ax_q4_desc_t* desc, const void* x, const int32_t* index, const int32_t* offsets,
                const uint8_t* g_codes, const void* g_scales, const uint8_t* u_codes, const void* u_scales, void* h_out,
                void* workspace, size_t workspace_bytes, void* hip_stream);
size_t ax_gated_q4_workspace_bytes(const ax_q4_desc_t* desc);

const char* ax_strerror(int code);

/* Library version, major * 10000 + minor * 100 + patch. */
int ax_version(void);

#ifdef __cplusplus
}
#endif
#endif /* AXCONV_H */
