/*
 * escoin.h -- C ABI of the MI355X (gfx950) direct sparse convolution library.
 *
 * The library computes one pruned convolution layer without lowering it to a matrix
 * product: the M x (C*R*S) filter matrix is held in CSR, one row per output channel
 * (Section 2.3), its column indices are "stretched" once into offsets of a zero-padded
 * 1-D input array (Section 3.1), and the output is accumulated nonzero by nonzero as in
 * Algorithm 2.  Shape names follow Table 1: N batch, M filters / ofmap channels, C ifmap
 * channels, H/W ifmap height/width, R/S filter height/width, E/F ofmap height/width.
 *
 * Conventions for every entry point
 *   - All tensors are contiguous fp32 NCHW (filters MCRS); all indices are int32.
 *   - Hp = H + 2*pad, Wp = W + 2*pad, E = (Hp - R)/stride + 1, F = (Wp - S)/stride + 1.
 *   - "host" pointers are ordinary CPU memory; "device" pointers are HIP device memory on
 *     the current device.  The library owns no memory: every buffer is the caller's and
 *     must stay valid until the stream work that uses it has finished.
 *   - Device entry points enqueue on `hip_stream` (a hipStream_t passed as void*; NULL is
 *     the default stream), never synchronise and never allocate.
 *   - Every call returns ESCOIN_OK (0) or a negative code; nothing throws or aborts.  On an
 *     error no kernel is launched and no output is written.
 *   - Output buffers are overwritten (no accumulation into their previous contents) and
 *     must not alias any input.
 */
#ifndef ESCOIN_H
#define ESCOIN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct escoin_conv_desc {
    int32_t N, C, H, W; /* input  N x C x H x W (unpadded)                     */
    int32_t M, R, S;    /* filter M x C x R x S                                */
    int32_t stride;     /* same stride on both axes, >= 1                      */
    int32_t pad;        /* symmetric zero padding on all four sides, >= 0      */
} escoin_conv_desc;

enum {
    ESCOIN_OK = 0,
    ESCOIN_EINVAL = -1, /* null pointer, non-positive dim, malformed CSR, bad flags   */
    ESCOIN_ERANGE = -2, /* an index would not fit int32 (C*Hp*Wp, M*E*F or nnz)       */
    ESCOIN_EHIP = -3,   /* a HIP call (launch, attribute query) failed                */
    ESCOIN_ESIZE = -4   /* a caller-provided buffer is too small                      */
};

enum {
    ESCOIN_F_BIAS = 1u, /* add bias[m] to every element of output channel m          */
    ESCOIN_F_RELU = 2u  /* clamp the result at zero: x > 0 ? x : 0                    */
};

/* Human-readable text for a return code (static storage, never NULL). */
const char *escoin_strerror(int code);

/* Validates a descriptor: ESCOIN_EINVAL for non-positive dims / stride < 1 / pad < 0 /
 * filter larger than the padded input, ESCOIN_ERANGE when C*Hp*Wp or M*E*F reaches 2^31. */
int escoin_check_desc(const escoin_conv_desc *desc);

/* Output extent E, F (Eq. 1 generalised by padding and stride).  Returns a code. */
int escoin_output_dims(const escoin_conv_desc *desc, int32_t *E, int32_t *F);

/* Element counts of the padded input N*C*Hp*Wp and of the output N*M*E*F; 0 on a bad desc. */
size_t escoin_padded_elems(const escoin_conv_desc *desc);
size_t escoin_output_elems(const escoin_conv_desc *desc);

/*
 * Weight stretching (Section 3.1).  Host, pure, run once per (layer, input size).
 * Each column index j = (c*R + r)*S + s of the M x CRS filter matrix is rewritten to the
 * CHW layout offset f(c, r, s) = (c*Hp + r)*Wp + s of the padded input; `value` and
 * `rowptr` are unchanged and the map is element-wise and order-preserving (entries may be
 * in any order inside a row and may repeat).
 *   rowptr            host, M+1 entries, rowptr[0] == 0, non-decreasing
 *   colidx            host, nnz = rowptr[M] entries, each in [0, C*R*S)
 *   colidx_stretched  host, nnz entries, caller-owned; may alias colidx (in-place)
 * ESCOIN_EINVAL on a malformed CSR (nothing useful is written then).
 */
int escoin_sconv_pack(const escoin_conv_desc *desc, const int32_t *rowptr, const int32_t *colidx,
                      int32_t *colidx_stretched);

/*
 * pad_in (Sections 3.1 and 4.2): the zero-padded 1-D input array
 *   padded[n][c][y + pad][x + pad] = in[n][c][y][x], +0.0f elsewhere.
 *   d_in      device, N*C*H*W floats
 *   d_padded  device, N*C*Hp*Wp floats, fully overwritten
 * With pad == 0 this is a plain copy.
 */
int escoin_pad_in(const escoin_conv_desc *desc, const float *d_in, float *d_padded,
                  void *hip_stream);

/*
 * sconv, Algorithm 2 as stated, for any filter size / stride and any CSR entry order:
 *   out[n][m][h][w] = sum over j in row m of
 *       value[j] * padded[n][ colidx_stretched[j] + h*stride*Wp + w*stride ]
 * optionally followed by the fused epilogue out = relu(out + bias[m]) (flags).
 *   d_rowptr, d_colidx_stretched, d_value   device CSR (stretched by escoin_sconv_pack)
 *   d_padded  device, N*C*Hp*Wp floats (from escoin_pad_in; the input itself when pad==0)
 *   d_out     device, N*M*E*F floats, overwritten
 *   d_bias    device, M floats; may be NULL unless ESCOIN_F_BIAS is set
 * The CSR on the device is trusted (it was validated by escoin_sconv_pack): offsets outside
 * the padded image are the caller's error.
 */
int escoin_sconv_forward(const escoin_conv_desc *desc, const int32_t *d_rowptr,
                         const int32_t *d_colidx_stretched, const float *d_value,
                         const float *d_padded, float *d_out, const float *d_bias,
                         uint32_t flags, void *hip_stream);

/* ------------------------------------------------------------------------------------------
 * LDS-tiled sconv: the same result as escoin_sconv_forward, computed from the UNPADDED input
 * (the zero frame of pad_in is produced while the input window is staged on chip, so the
 * padded array of Section 3.1 only ever exists tile by tile in LDS).  It needs a plan: a
 * kernel-specific re-encoding of the stretched CSR (nonzeros regrouped by input-channel chunk
 * and row bin, offsets re-stretched to the on-chip window; Section 3.3's "weights stationary,
 * inputs streamed" with Section 4.3's tiling).  The stretched CSR stays the externally
 * visible, bit-exact packing result; the plan is derived data and opaque.
 * ------------------------------------------------------------------------------------------ */

/* Tiling knobs; a zero field means "choose for me".  Out-of-range combinations make the plan
 * calls return ESCOIN_EINVAL / ESCOIN_ERANGE (e.g. a window that does not fit LDS). */
typedef struct escoin_sconv_tuning {
    int32_t K;  /* output channels accumulated per wave: 1, 2, 4 or 8               */
    int32_t Q;  /* 16-byte position groups per lane, 1 or 2                         */
    int32_t B;  /* nonzeros per record batch, 2 or 4 (not every K/Q/B mix exists)   */
    int32_t WM; /* waves per workgroup along the output-channel axis (WS included)  */
    int32_t CC; /* input channels staged per LDS chunk                              */
    int32_t NB; /* images per workgroup                                             */
    int32_t TH; /* output rows per tile                                             */
    int32_t CS; /* workgroups sharing one output tile, each taking every CS-th      */
                /* channel chunk and adding its partial sums with float atomics     */
    int32_t WS; /* every output channel's nonzeros are split over at least WS waves */
                /* of a workgroup, whose partial sums are added in LDS (rows much   */
                /* longer than a wave's share are split further by the library)     */
    int32_t CC0;/* input channels of the first chunk, <= CC (a short first chunk    */
                /* lets the arithmetic start before the whole window has arrived)   */
} escoin_sconv_tuning;

/* Bytes the plan blob needs.  Host; rowptr / colidx_stretched as returned by
 * escoin_sconv_pack (any order inside a row, duplicates allowed); tuning may be NULL. */
int escoin_sconv_plan_size(const escoin_conv_desc *desc, const int32_t *rowptr,
                           const int32_t *colidx_stretched, const escoin_sconv_tuning *tuning,
                           size_t *plan_bytes);

/* Builds the plan into caller-owned host memory `plan` (plan_bytes from the size query, else
 * ESCOIN_ESIZE).  A plan is valid for every batch size (only C, H, W, M, R, S, stride and pad are
 * checked at launch); desc->N only guides the default tiling.  The caller then copies the blob
 * verbatim to device memory (256-byte aligned) and keeps the host copy for escoin_sconv_forward_tiled.
 * ESCOIN_EINVAL if an offset is not one weight stretching can produce for this desc. */
int escoin_sconv_plan_build(const escoin_conv_desc *desc, const int32_t *rowptr,
                            const int32_t *colidx_stretched, const float *value,
                            const escoin_sconv_tuning *tuning, void *plan, size_t plan_bytes);

/*
 * out[n][m][h][w] = sum_j value[j] * Ipad[n][...]  (Algorithm 2 / Eq. 1 with zero padding and
 * stride), optional fused epilogue as in escoin_sconv_forward.
 *   plan_host  host copy of the blob (only its header is read, synchronously)
 *   d_plan     device copy of the same blob
 *   d_in       device, N*C*H*W floats, UNPADDED
 *   d_out      device, N*M*E*F floats, overwritten
 * ESCOIN_EINVAL if the plan was built for another layer geometry.
 *
 * By default a launch that would leave compute units idle (small batches) splits every output
 * channel's nonzeros over several waves of a workgroup and adds their partial sums on chip: one
 * kernel, and the same bits on every run.
 *
 * A plan with CS > 1 (only on request, through the tuning) splits the input channels of a tile
 * over CS workgroups instead.  The call then enqueues three kernels: a zero fill of d_out, the
 * convolution, whose workgroups add their partial sums with fp32 atomics (the order of those
 * additions, and with it the last bits of the result, may differ from run to run), and, with
 * ESCOIN_F_RELU, the clamp as a pass of its own.
 *
 * A plan made without tuning for a layer of stride 1 or 2, or of few input channels and any even stride, may also hold its
 * weights for the matrix cores, and a call on a batch large enough to be faster there multiplies all of them, zeros too.  Two forms:
 *   - pairs of fp16 numbers, for layers of up to some 90 % sparsity whose rows have 32 nonzeros or more, 60 to some hundred on
 *     the average, and whose filters reach at most 127 positions of the flat padded map (two rows of 62, four of 30; at
 *     stride 2 of the outputs' map), or with fewer than 16 input channels and an even stride, where 256 outputs of an image need
 *     no more than some 12 000 words of whole padded input rows (3 channels, 7x7 filters, stride 2: up to 250 columns).  Inputs are scaled by a
 *     power of two, the same for a workgroup's window, weights by one a row.  A pair holds 22 to 23 bits: an output of n
 *     products is off by up to 2^-21 of sum|w*x|, 0.8e-7 to 1.5e-7 of the result in the mean.  Where half of the inputs are zeros that is
 *     less than a chain of fp32 sums is off by from about 60 nonzeros on, and shorter rows are summed in fp32; an output that meets
 *     fewer than some 30 inputs other than zero is less exact than in fp32 (a single product by up to 2^-21, not 2^-24).  A plan made
 *     with a tuning keeps to fp32 multiply-adds.  Weights of a row more than 2^27 apart keep a layer from the pairs;
 *   - three bf16 parts each, for layers of stride 1 pruned little (roughly 50-70 %) where the sums are too short for the pairs or the filters
 *     reach further.  Results stay within fp32 rounding of the sums over the nonzeros.  Weights outside 2^-50 .. 2^30 keep a layer
 *     from it.
 * In both, tiny inputs, Inf and NaN behave as in the sums over the nonzeros: outputs that meet an Inf or a NaN, or whose
 * inputs are all far smaller than others of their window (2^-70 in the second form), are computed from the nonzeros
 * and slow such a call down.  Repeated columns keep a layer on the tiled kernel.  The sections add 4 and 6 bytes
 * per weight of the unpruned filter bank (channels rounded up to 64 and 16) and 12 per nonzero to the plan, whatever
 * batch it is for.
 *
 * escoin_sconv_tiled_on_matrix_cores (host) tells which kernel a call with this descriptor and a 16-byte
 * aligned d_plan takes: 1 for the matrix cores, 0 for the tiled kernel, or an error code as the call itself would return.
 * escoin_sconv_tiled_kernel tells it further: 0 for the tiled kernel, 1 for the one of three bf16 parts,
 * 100*a + 10*b + c for the one of pairs with workgroups of a*b*c waves over a*64 output channels, b*64 positions and c
 * shares of the input channels (141: the form for fewer than 16 input channels and an even stride).
 *
 * d_in and d_plan that are 16-byte aligned let the kernel stage with 16-byte loads (or with
 * global -> LDS copies); any 4-byte aligned pointer is accepted.
 */
int escoin_sconv_forward_tiled(const escoin_conv_desc *desc, const void *plan_host,
                               const void *d_plan, const float *d_in, float *d_out,
                               const float *d_bias, uint32_t flags, void *hip_stream);
int escoin_sconv_tiled_on_matrix_cores(const escoin_conv_desc *desc, const void *plan_host);
int escoin_sconv_tiled_kernel(const escoin_conv_desc *desc, const void *plan_host);

/* ---------------------------------------------------------------------------------------
 * Pruned feed-forward blocks: linear layers on token-major activations, and the norms between them.
 *
 * Conventions beside those at the top of this file
 *   - Activations are T x features, one row a token, features contiguous; rows may lie further apart (ld_*, in
 *     elements; 0: next to each other).  Every tensor of a call, parameters too, has the descriptor's type; pointers are
 *     aligned to it.  Sums and statistics are fp32, an output is rounded once (to nearest even).
 *   - T == 0 is a call that does nothing and returns ESCOIN_OK.  Rows from T on are neither read nor written.
 *   - ESCOIN_ERANGE also where a launch would have 2^32 threads (some four million rows of a long norm).
 */
enum { ESCOIN_T_F32 = 0, ESCOIN_T_F16 = 1, ESCOIN_T_BF16 = 2 };

enum {
    /* ESCOIN_F_BIAS and ESCOIN_F_RELU as above, and: */
    ESCOIN_F_RESIDUAL = 4u,   /* add residual[t][m] to the result                               */
    ESCOIN_F_SILU = 8u,       /* z / (1 + exp(-z))                                              */
    ESCOIN_F_GELU = 16u,      /* z/2 * erfc(-z / sqrt(2))                                       */
    ESCOIN_F_GELU_TANH = 32u  /* z/2 * (1 + tanh(sqrt(2/pi) * (z + 0.044715 z^3)))              */
};

typedef struct escoin_linear_desc {
    int32_t T, K, M; /* tokens, input features, output features                             */
    int32_t type;    /* ESCOIN_T_*                                                          */
    int32_t gated;   /* 0, or 1: act(gate) * up, from a CSR of 2*M rows, the gates' first   */
    int64_t ld_in, ld_out, ld_residual; /* elements from row to row; 0: K, M, M             */
} escoin_linear_desc;

/* Validates a descriptor: ESCOIN_EINVAL for T < 0, K or M < 1, an unknown type or a row pitch shorter than its row,
 * ESCOIN_ERANGE where K reaches 2^22, 2*M 2^30 or a pitch 2^40, or the 16 by 128 tiles of the weights 2^31. */
int escoin_linear_check_desc(const escoin_linear_desc *desc);

/*
 * Pruned linear layer.  With W (M x K, or 2*M x K gated) given by its nonzeros as CSR,
 *   out[t][m] = act(sum_k W[m][k] * in[t][k] + bias[m]) + residual[t][m]
 *   gated:      act(sum_k W[m][k] * in[t][k] + bias[m]) * (sum_k W[M+m][k] * in[t][k] + bias[M+m]) + residual[t][m]
 * The plan (host blob, then uploaded, as for the convolution) holds the weights rounded to the descriptor's type
 * (beyond its range: infinite), each with a bit for its place, in the order in which the matrix cores take them; plans for
 * more tokens than escoin_linear_few_tokens tells hold them a second time with their zeros.  `T` of the descriptor that a plan is
 * built with is the most tokens that calls with it may have.
 *   rowptr, colidx, value  host CSR, columns of a row in any order; repeated ones are added up in fp32
 *   plan_size     an upper bound on the blob's size, from the descriptor and the number of nonzeros
 *   plan_build    fills it, by up to eight threads; equal calls give equal bytes.  ESCOIN_ESIZE if it is smaller than plan_size
 *                 tells (or there is no memory for 32 rows a thread), ESCOIN_EINVAL on a malformed CSR
 * Both run on the host and need no GPU.
 */
int escoin_linear_plan_size(const escoin_linear_desc *desc, const int32_t *rowptr, const int32_t *colidx, size_t *plan_bytes);
int escoin_linear_plan_build(const escoin_linear_desc *desc, const int32_t *rowptr, const int32_t *colidx,
                             const float *value, void *plan, size_t plan_bytes);

/*
 * One forward call.  Up to escoin_linear_few_tokens tokens a kernel reads each kept weight once and multiplies it on the
 * matrix cores as it comes, beyond that the weights are multiplied in tiles, zeros too.  Pruned weights count as zeros: an Inf
 * or NaN in a token's input can make every output of that token NaN (or what the epilogue makes of it), and of no other token.
 * The order of the sums depends on T, never on timing: equal calls give equal bits.
 *   plan_host     host pointer to the blob (its header is read at the call), d_plan its copy on the device, 16-byte aligned
 *   d_bias        device, M (gated: 2*M) elements, with ESCOIN_F_BIAS
 *   d_residual    device, with ESCOIN_F_RESIDUAL; may be d_out itself with the same pitch (each element is read before it is
 *                 written), and must not overlap it otherwise
 *   flags         ESCOIN_F_BIAS, ESCOIN_F_RESIDUAL and at most one activation
 * Inputs whose rows start on 16-byte boundaries, and hold a multiple of 16 bytes, are read with wide loads; any other is accepted.
 */
int escoin_linear_forward(const escoin_linear_desc *desc, const void *plan_host, const void *d_plan, const void *d_in,
                          void *d_out, const void *d_bias, const void *d_residual, uint32_t flags, void *hip_stream);
/* host: up to how many tokens a call with this plan reads the kept weights only; or an error code */
int escoin_linear_few_tokens(const escoin_linear_desc *desc, const void *plan_host);

/* host: the kernel that a call with this descriptor and plan takes, for reports and tests.  All zeros for a call without tokens. */
typedef struct escoin_linear_kernel_info {
    int32_t kept;         /* 1: reads the kept weights; 0: the whole ones, tile by tile               */
    int32_t rows, tokens; /* of weights and of activations, to a workgroup                            */
    int32_t waves;
    int32_t inputs;       /* 0: from any place, by way of registers; 1: 16 bytes a lane to registers; */
                          /* 2: 16 bytes a lane copied to LDS                                         */
    int32_t pieces;       /* kept: 16-byte pieces that a lane loads of a tile's values                */
    int32_t lane_words;   /* kept: 32-bit words of LDS that are a lane's own                          */
    int32_t steps;        /* whole: steps along the columns that LDS holds                            */
    int32_t step_bytes;   /* whole: bytes of a row to a step                                          */
    int32_t lds_bytes;    /* of a workgroup                                                           */
} escoin_linear_kernel_info;
/* d_in: where the call's input will lie (its alignment counts; nothing is read) */
int escoin_linear_kernel(const escoin_linear_desc *desc, const void *plan_host, const void *d_in, escoin_linear_kernel_info *info);

enum { ESCOIN_NORM_NONE = 0, ESCOIN_NORM_RMS = 1, ESCOIN_NORM_LAYER = 2 };

typedef struct escoin_norm_desc {
    int32_t T, D;        /* tokens, features                                                    */
    int32_t type;        /* ESCOIN_T_*                                                          */
    int32_t post, pre;   /* ESCOIN_NORM_*: of the block's output y, and of the sum h            */
    int32_t gate_rows;   /* 0: one gate vector for all tokens; 1: a row for each token          */
    float eps;           /* added to the mean square (or variance), >= 0                        */
    float alpha, beta;   /* scales of the residual stream and of the block's output             */
    float weight_offset; /* added to every norm weight (1 where weights are kept as w - 1)      */
    int64_t ld_x, ld_y, ld_gate, ld_h, ld_n; /* elements from row to row; 0: D                  */
} escoin_norm_desc;

int escoin_norm_check_desc(const escoin_norm_desc *desc);

/*
 * The residual stream between two blocks, in one pass over it:
 *   h[t] = alpha * x[t] + beta * gate * post(y[t])       n[t] = pre(h[t])
 *   RMS(v) = v / sqrt(mean(v^2) + eps) * (weight + weight_offset) + bias
 *   LAYER(v): of v - mean(v), with the variance in place of the mean square;   NONE(v) = v
 * n is the norm of h before h is rounded.
 *   d_x                  device, T x D
 *   d_y, d_gate          device; d_y NULL: h = alpha * x (post must be NONE then, and d_gate NULL); d_gate NULL: 1
 *   d_post_*, d_pre_*    device, D elements each; a weight NULL: no factor (weight_offset is then unused), a bias NULL: none; NULL for a
 *                        norm that is NONE
 *   d_h, d_n             device, T x D each; either may be NULL.  Each may be d_x or d_y itself with the same pitch; h and n
 *                        must not be the same.
 */
int escoin_norm_forward(const escoin_norm_desc *desc, const void *d_x, const void *d_y, const void *d_gate,
                        const void *d_post_weight, const void *d_post_bias, const void *d_pre_weight, const void *d_pre_bias,
                        void *d_h, void *d_n, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ESCOIN_H */
