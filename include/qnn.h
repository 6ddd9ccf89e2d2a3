/*
 * qnn.h - C ABI of the GB300 (sm_103a) quantized HWC convolution library.
 *
 * Method: PULP-NN, "Accelerating Quantized Neural Networks on Parallel
 * Ultra-Low-Power RISC-V Processors" (arXiv 1908.11263).  The library runs the
 * data-parallel hot path of that method on one GPU: im2col + integer MatMul
 * with 32-bit accumulation (Sec. III-B, Eq. 2 and Eq. 6), compression of the
 * accumulator back to Q bits (Sec. III-A), max-pooling and the fully connected
 * layer (Sec. IV-A), for INT-8 and packed INT-4 / INT-2 data (Sec. IV-A,
 * "Sub-byte Extensions").  Also: the staircase (threshold) compression of
 * Eq. 4, the INT-1 XNOR / popcount convolution of Eq. 5, and a convolution
 * with its 2x2 max-pooling fused into one kernel.
 *
 * Conventions shared by every entry point
 *  - Plain C types only.  Pointers marked "device" must point to memory of the
 *    current CUDA device; the caller allocates and owns every buffer, and keeps
 *    it alive until the work queued on `stream` has finished.
 *  - `stream` is a cudaStream_t passed as void*; NULL means the legacy default
 *    stream.  Every call only enqueues work and returns; device-side problems
 *    surface at the caller's next synchronisation, or through
 *    qnn_device_status().
 *  - Arguments are validated before anything is launched; a call that returns
 *    an error has enqueued nothing.  Nothing is thrown across the ABI.
 *  - Tensors are dense and contiguous; there are no stride arguments (the
 *    language-model block operators at the end take row strides).  Input and
 *    output buffers must not overlap.
 *  - Sub-byte storage: element e of a packed Q-bit stream sits in byte
 *    e / (8/Q) at bits [(e mod (8/Q)) * Q, +Q), the first element in the least
 *    significant bits.  Activations are unsigned, weights two's-complement.
 *  - Thread safety: calls may be made from several host threads; the only
 *    shared host state is a per-device cache of queried device properties.
 *    A workspace belongs to one call at a time, on one stream too: calls of
 *    several threads interleave their launches, and a call may hold data in
 *    its workspace from one launch to the next.
 */
#ifndef QNN_H
#define QNN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    QNN_OK = 0,
    QNN_EINVAL = 1,        /* NULL pointer, non-positive size, empty output, shift out of [0,62], bad struct_size */
    QNN_EUNSUPPORTED = 2,  /* bits not in {8,4,2}; mixed bit-widths; C, M or a count not a whole number of bytes
                              at Q bits; accumulator bound above int32; forced algorithm that cannot run the shape */
    QNN_EALIGN = 3,        /* a tensor pointer that must be 16-byte aligned is not */
    QNN_ECUDA = 4,         /* a CUDA runtime call or kernel launch failed */
    QNN_ETIMEOUT = 5,      /* a bounded device-side wait gave up (reported by qnn_device_status) */
    QNN_EWORKSPACE = 6,    /* workspace missing or smaller than qconv_hwc_workspace_size() */
    QNN_ESCRATCH = 7       /* qconv_hwc_noalloc(): the layer needs more than QNN_NOALLOC_SCRATCH_BYTES */
} qnn_status;

/* Convolution algorithm choice (qnn_conv_desc.algo). */
enum {
    QNN_ALGO_AUTO = 0,         /* tensor-core kernel when the shape allows it, else the CUDA-core kernel */
    QNN_ALGO_DIRECT = 1,       /* CUDA-core kernel (dp4a), any stride / padding */
    QNN_ALGO_TENSORCORE = 2,   /* tcgen05 implicit GEMM (the window kernel when its plan fits, else the
                                  general one); QNN_EUNSUPPORTED when neither fits the shape */
    QNN_ALGO_TC_WINDOW = 3,    /* the window kernel only: stride 1, m <= 128, INT-8 with c a multiple of 8
                                  or INT-4/INT-2 with c a multiple of 32, c <= 64 (INT-8) or 128 (sub-byte),
                                  kh, kw <= 8; one launch per call, filters read in place */
    QNN_ALGO_TC_GENERAL = 4    /* the general tensor-core kernel only (filter preparation kernel plus
                                  convolution kernel, any stride-1 shape with whole 16-byte input rows) */
};

/*
 * One convolution layer (Sec. III-B).  Input x is NHWC [n][h][w][c]; filters
 * are [m][kh][kw][c] with c innermost, so each bank W(m) is stored in im2col
 * order (Eq. 6).  Output y is NHWC [n][oh][ow][m] with
 * oh = (h + 2*pad_h - kh) / stride_h + 1 and ow likewise (floor).  Padding
 * reads as activation 0.  x, w and y all use `bits` per element.
 */
typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_conv_desc) */
    int32_t n, h, w, c;        /* input batch, height, width, channels; n may be 0 (no work) */
    int32_t m, kh, kw;         /* output channels, kernel height and width */
    int32_t stride_h, stride_w;
    int32_t pad_h, pad_w;
    int32_t bits;              /* Q in {8, 4, 2} for activations, weights and outputs alike */
    int32_t shift;             /* right shift in [0, 62], used for every channel when shifts == NULL */
    int32_t algo;              /* QNN_ALGO_* */
} qnn_conv_desc;

/*
 * Bytes of device workspace for this layer: what qconv_hwc_prepare() writes
 * and qconv_hwc_run() reads, and what qconv_hwc() needs on the general
 * tensor-core kernel (0 for the CUDA-core kernel).  For the general kernel
 * the workspace holds the filters re-laid out for the tensor cores and the
 * per-channel compression constants, rewritten by every qconv_hwc() call, so
 * one workspace must not be shared by calls that can run concurrently.  For
 * the window kernel it holds the image of the kernel's shared-memory operands
 * that qconv_hwc_prepare() builds once (the filters as the tensor-core B
 * operand, the per-channel compression records, the exact chunk count and the
 * MMA issue table); qconv_hwc_run() reads it with two bulk copies per block,
 * and qconv_hwc() builds the same operands inside its one launch and leaves
 * the workspace alone.
 */
qnn_status qconv_hwc_workspace_size(const qnn_conv_desc *d, size_t *bytes);

/*
 * Quantized convolution with fused compression (Sec. III-A, III-B, IV-A):
 *
 *   acc[n][oy][ox][o] = sum_{i<kh, j<kw, ch<c} x[n][oy*sh-ph+i][ox*sw-pw+j][ch] * w[o][i][j][ch]   (int32)
 *   y[n][oy][ox][o]   = clip( floor( ((acc + bias[o]) * kappa[o] + lambda[o]) / 2^shift_o ), 0, 2^Q - 1 )
 *
 * computed exactly (64-bit intermediate for the scaled value); the clip is
 * also the ReLU.  shift_o = shifts[o] when shifts != NULL, else d->shift.
 *
 *   x       device, packed unsigned Q-bit NHWC, 16-byte aligned
 *   w       device, packed signed Q-bit [m][kh][kw][c], 16-byte aligned
 *   bias    device int32[m], or NULL for zero
 *   kappa   device int16[m]
 *   lambda  device int32[m]
 *   shifts  device uint8[m] with values in [0, 62], or NULL
 *   y       device, packed unsigned Q-bit NHWC output, 16-byte aligned
 *   workspace, workspace_bytes: device scratch of at least
 *           qconv_hwc_workspace_size() bytes, 256-byte aligned (may be NULL
 *           when that size is 0).  When the window kernel serves the layer
 *           (qconv_hwc_tc_kernel() == QNN_ALGO_TC_WINDOW) the call is one
 *           launch that reads w, bias, kappa, lambda and shifts in place and
 *           the workspace is neither read nor written (it may be NULL).
 *
 * Requirements (else QNN_EUNSUPPORTED): c and m multiples of 8/Q, and
 * kh*kw*c*(2^Q-1)*2^(Q-1) < 2^30, so that the int32 accumulator of Eq. 2 cannot
 * overflow.  The caller keeps |bias| < 2^30 (bias values are not inspected).
 */
qnn_status qconv_hwc(const qnn_conv_desc *d, const void *x, const void *w, const int32_t *bias,
                     const int16_t *kappa, const int32_t *lambda, const uint8_t *shifts, void *y,
                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * The two halves of qconv_hwc(), for callers whose filters and compression
 * constants stay fixed across many calls (inference serving):
 *
 * qconv_hwc_prepare: writes into `workspace` the filters re-laid out for the
 *   tensor cores and the per-channel constants derived from bias, kappa,
 *   lambda and the shifts (same argument rules as qconv_hwc); one small
 *   launch.  The caller's buffers may be freed or changed afterwards.  For a
 *   descriptor that selects the CUDA-core kernel it enqueues nothing.
 * qconv_hwc_run: the convolution itself, reading a workspace prepared for the
 *   same descriptor (any other workspace content gives undefined results).
 *   Only for descriptors that select the tensor-core kernel; otherwise
 *   QNN_EUNSUPPORTED.  The window kernel launches with programmatic stream
 *   serialization: it may start while the previous kernel in the stream is
 *   still running, waits for it before touching x or y, and reads the
 *   workspace before that wait, so the workspace must not be written by the
 *   kernel launched just before it (qconv_hwc_prepare's own launch is fine:
 *   its successor starts only after it ends).
 * qconv_hwc(...) is exactly qconv_hwc_prepare(...) followed by qconv_hwc_run(...)
 * on the same stream.
 */
qnn_status qconv_hwc_prepare(const qnn_conv_desc *d, const void *w, const int32_t *bias, const int16_t *kappa,
                             const int32_t *lambda, const uint8_t *shifts, void *workspace, size_t workspace_bytes,
                             void *stream);
qnn_status qconv_hwc_run(const qnn_conv_desc *d, const void *x, void *y, const void *workspace,
                         size_t workspace_bytes, void *stream);

/*
 * Quantized convolution, compression and 2x2 max-pooling in one kernel: the
 * pooling layer of Sec. IV-A (window 2, stride 2, no padding, floor output
 * size) applied to the output of qconv_hwc(), fused into its epilogue so the
 * full-resolution output never reaches memory:
 *
 *   t[n][oy][ox][o]  = y of qconv_hwc() for the same arguments
 *   y[n][py][px][o]  = max over dy, dx in {0, 1} of t[n][2*py+dy][2*px+dx][o]
 *                      for py < oh / 2, px < ow / 2 (integer division)
 *
 * Arguments are those of qconv_hwc(); y is the pooled NHWC tensor
 * [n][oh/2][ow/2][m], packed Q-bit, 16-byte aligned.  The workspace size is
 * qconv_hwc_workspace_size() of the same descriptor.  Runs only on the
 * tensor-core kernel (stride 1, the shapes qconv_hwc_algo() reports as
 * QNN_ALGO_TENSORCORE, d->algo not QNN_ALGO_DIRECT); QNN_EUNSUPPORTED
 * otherwise, and QNN_EINVAL when oh or ow is below 2 (no pooled pixel).
 */
qnn_status qconv_hwc_pool2(const qnn_conv_desc *d, const void *x, const void *w, const int32_t *bias,
                           const int16_t *kappa, const int32_t *lambda, const uint8_t *shifts, void *y,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * qconv_hwc_pool2_run: qconv_hwc_pool2() on filters prepared with
 * qconv_hwc_prepare() for the same descriptor: the fused convolution,
 * compression and 2x2/2 max-pool, one launch that reads x, the workspace and
 * writes the pooled y ([n][oh/2][ow/2][m], packed Q-bit, 16-byte aligned).
 * Only where qconv_hwc_algo() reports the window tensor-core kernel
 * (qconv_hwc_tc_kernel() == QNN_ALGO_TC_WINDOW); QNN_EUNSUPPORTED otherwise,
 * QNN_EINVAL when oh or ow is below 2, QNN_EWORKSPACE for a workspace below
 * qconv_hwc_workspace_size() or not 256-byte aligned.  The workspace rules of
 * qconv_hwc_run() apply (it is read before the wait on the previous kernel).
 */
qnn_status qconv_hwc_pool2_run(const qnn_conv_desc *d, const void *x, void *y, const void *workspace,
                               size_t workspace_bytes, void *stream);

/*
 * Quantized convolution with staircase compression (Sec. III-A, Eq. 4), the
 * paper's compression for INT-4 and INT-2 outputs:
 *
 *   acc[n][oy][ox][o] = as in qconv_hwc() (int32, no bias)
 *   y[n][oy][ox][o]   = number of k in [0, 2^Q - 1) with thresholds[o][k] <= acc
 *
 * For thresholds sorted ascending per channel this is the index p of the
 * interval [tau_p, tau_p+1) that holds the accumulator, counted from 0 for the
 * lowest interval (unsigned outputs).  The thresholds absorb bias and batch
 * normalisation (footnote to Eq. 3), so there is no bias, kappa or lambda.
 *
 *   x, w, y     as in qconv_hwc(); d->bits must be 4 or 2 (else QNN_EUNSUPPORTED)
 *   thresholds  device int32 [m][2^Q - 1], 4-byte aligned (any values)
 *   workspace, workspace_bytes: as in qconv_hwc() (qconv_hwc_workspace_size)
 *
 * d->shift is ignored.  Same accumulator bound and other requirements as
 * qconv_hwc().
 */
qnn_status qconv_hwc_thresholds(const qnn_conv_desc *d, const void *x, const void *w, const int32_t *thresholds,
                                void *y, void *workspace, size_t workspace_bytes, void *stream);

/*
 * INT-1 convolution (Sec. III-A, Eq. 5; binary kernel of Sec. IV-A).  Values
 * +1 / -1 are bits 1 / 0, eight per byte, element e at bit e mod 8 of byte e / 8
 * (the sub-byte order above with Q = 1).
 *
 *   acc[n][oy][ox][o] = number of (i, j, ch) with the input pixel inside the
 *                       image and bit(w[o][i][j][ch]) == bit(x[n][iy][ix][ch])
 *                       (popcount of W xnor X; padding contributes nothing)
 *   y[n][oy][ox][o]   = 1 if thresholds[o] <= acc, else 0
 *
 *   d           d->bits must be 1; c and m multiples of 8; d->shift and d->algo ignored
 *   x           device, NHWC bits [n][h][w][c / 8 bytes]
 *   w           device, [m][kh][kw][c / 8 bytes]
 *   thresholds  device int32 [m], 4-byte aligned
 *   y           device, NHWC bits [n][oh][ow][m / 8 bytes]
 *
 * Runs on CUDA cores (XNOR and population count).  QNN_EUNSUPPORTED when bits
 * is not 1 or c, m are not multiples of 8.
 */
qnn_status qconv_hwc_binary(const qnn_conv_desc *d, const void *x, const void *w, const int32_t *thresholds,
                            void *y, void *stream);

/* Which kernel qconv_hwc() would run for d: QNN_ALGO_DIRECT or QNN_ALGO_TENSORCORE;
 * negative qnn_status on invalid or unsupported descriptors. */
int32_t qconv_hwc_algo(const qnn_conv_desc *d);

/* Which tensor-core kernel qconv_hwc() would run for d: QNN_ALGO_TC_WINDOW or
 * QNN_ALGO_TC_GENERAL; 0 when d selects the CUDA-core kernel; negative qnn_status
 * on invalid or unsupported descriptors. */
int32_t qconv_hwc_tc_kernel(const qnn_conv_desc *d);

/* Operand format of the tensor-core MMAs qconv_hwc() would issue for d, so that a
 * caller can take the right tensor roof: 16 for fp16 operands (tcgen05 kind::f16,
 * the exact embedding of INT-8 and of sub-byte layers with c not a multiple of 32),
 * 8 for e4m3 operands (kind::f8f6f4, twice the fp16 rate per MMA; INT-4/INT-2 with
 * c a multiple of 32), 0 when d selects the CUDA-core kernel; negative qnn_status
 * on invalid or unsupported descriptors.  Not a paper concept: a query about this
 * library's kernel choice. */
int32_t qconv_hwc_mma_operand_bits(const qnn_conv_desc *d);

/* Size of the fixed scratch array behind qconv_hwc_noalloc(): 2 MiB. */
enum { QNN_NOALLOC_SCRATCH_BYTES = 2097152 };

/*
 * qconv_hwc() without a workspace, for callers that cannot allocate device
 * memory.  The paper has no counterpart to this entry point; it serves users of
 * the library.  Typical such callers: a serving runtime that commits all device
 * memory to its own arenas up front and has none to hand to a library; a
 * latency-critical loop, where cudaMalloc / cudaFree would synchronise the
 * device and stall its other streams; a plain C caller with no device
 * allocator of its own to size, own and free a workspace.
 *
 * Arguments and results are those of qconv_hwc() minus the workspace.  The
 * re-laid-out filters and per-channel constants go to one scratch array of
 * QNN_NOALLOC_SCRATCH_BYTES compiled into the library's device image, which
 * every GPU that loads the library holds until the process exits.  The call
 * allocates nothing: no cudaMalloc, cudaFree or allocating library routine.
 *
 *  - Only for descriptors that select the tensor-core kernel (QNN_ALGO_AUTO
 *    resolving to it, or QNN_ALGO_TENSORCORE), else QNN_EUNSUPPORTED.  The
 *    CUDA-core kernel needs no scratch: call qconv_hwc() with a NULL workspace.
 *  - QNN_ESCRATCH, with nothing enqueued, when the layer needs more than
 *    QNN_NOALLOC_SCRATCH_BYTES; qconv_hwc_workspace_size() gives the need.
 *  - Set-up on first use: the first call on each device looks up the scratch
 *    array's device address (cudaGetSymbolAddress, with that device current;
 *    QNN_ECUDA if that fails), and the first tensor-core launch of each bit
 *    width and filter tile on a device raises that kernel's shared-memory
 *    limit.  Make those first calls before any stream capture.
 *  - Shared state: all calls on a device use the same array, which keeps the
 *    last call's contents.  Each call rewrites every scratch byte its
 *    convolution reads before reading it, so nothing has to be cleared between
 *    calls.  Calls that overlap on the GPU (streams with no ordering between
 *    them) race on the array and give undefined results; calls queued on one
 *    stream do not overlap.
 *  - n == 0: after validation, returns QNN_OK with nothing enqueued (the
 *    scratch array is not touched).
 */
qnn_status qconv_hwc_noalloc(const qnn_conv_desc *d, const void *x, const void *w, const int32_t *bias,
                             const int16_t *kappa, const int32_t *lambda, const uint8_t *shifts, void *y,
                             void *stream);

/*
 * Fully connected layer (Sec. IV-A, matrix-vector product split over output
 * neurons in Sec. IV-B), without compression:
 *   y[b][o] = sum_{i<k} x[b][i] * w[o][i] + bias[o]      (int32 output)
 *   x    device uint8 [n][k]      (HWC-flattened activations)
 *   w    device int8  [m][k]
 *   bias device int32 [m] or NULL
 *   y    device int32 [n][m]
 * Requirements: k * 255 * 128 < 2^30 (else QNN_EUNSUPPORTED); the caller keeps |bias| < 2^30.
 */
qnn_status qlinear(int32_t n, int32_t k, int32_t m, const uint8_t *x, const int8_t *w, const int32_t *bias,
                   int32_t *y, void *stream);

/*
 * Max-pooling (Sec. IV-A): y[b][oy][ox][ch] = max_{i,j<k} x[b][oy*s+i][ox*s+j][ch]
 * on packed unsigned Q-bit NHWC data, no padding, oh = (h-k)/s + 1 (floor).
 *   x  device, [n][h][w][c] packed at `bits`;  y  device, [n][oh][ow][c] packed at `bits`
 * Requirements: c a multiple of 8/Q; 1 <= k <= min(h, w); s >= 1.
 */
qnn_status qmaxpool(int32_t n, int32_t h, int32_t w, int32_t c, int32_t k, int32_t s, int32_t bits,
                    const void *x, void *y, void *stream);

/*
 * Sub-byte packing (Sec. IV-A, "Sub-byte Extensions": two INT-4 or four INT-2
 * values per byte, and the unpack-to-INT-8 helper of the same section).
 *   pack_subbyte:   src device int8[count] (the low Q bits of each value are stored),
 *                   dst device uint8[count*Q/8]
 *   unpack_subbyte: src device uint8[count*Q/8], dst device int8[count];
 *                   is_signed != 0 sign-extends (weights), 0 zero-extends (activations)
 * count must be a multiple of 8/Q; bits in {8,4,2} (8 is a plain copy).
 */
qnn_status pack_subbyte(const int8_t *src, void *dst, int64_t count, int32_t bits, void *stream);
qnn_status unpack_subbyte(const void *src, int8_t *dst, int64_t count, int32_t bits, int32_t is_signed,
                          void *stream);

/*
 * Synchronises `stream`, then returns and clears the library's device status
 * word: QNN_OK, or QNN_ETIMEOUT when a bounded wait inside a kernel gave up
 * (the kernel then skipped its remaining work and returned).  QNN_ECUDA when
 * the synchronisation itself fails.
 */
qnn_status qnn_device_status(void *stream);

/*
 * Diagnostics: runs the library's bounded-wait failure path on the GPU.  One
 * warp waits on an mbarrier that nothing arrives on; after `limit_cycles` SM
 * cycles the wait gives up, records QNN_ETIMEOUT in the device status word and
 * the kernel returns, leaving the context usable.  Every wait inside the
 * library's kernels is bounded the same way (a wait that never completes
 * turns into QNN_ETIMEOUT, not a hang).  The paper has no counterpart; this
 * exists so that the failure path can be tested without faulting a GPU.
 * limit_cycles must lie in [1, 2^31); QNN_EINVAL otherwise.  Read the result
 * with qnn_device_status(stream).
 */
qnn_status qnn_selftest_wait_timeout(int64_t limit_cycles, void *stream);

/* Static description of a status code. */
const char *qnn_status_string(qnn_status s);

/* Library version, for ABI checks: major * 10000 + minor * 100 + patch. */
int32_t qnn_version(void);

/* ------------------------------------------------------------------------
 * Operators of a language model's block, for serving: the norms around a
 * block, the routing to experts, the matrix product with a fused epilogue and
 * the experts' products.  Activations are floating point here; weights may be
 * packed INT-8/4/2 in the order above with one scale per output channel.
 * These entry points take row strides (elements); columns are contiguous.
 * ---------------------------------------------------------------------- */

/* Element types of activations, residuals and parameters. */
enum { QNN_F16 = 0, QNN_BF16 = 1, QNN_F32 = 2 };

/* Norm of qnn_block_norm(). */
enum {
    QNN_NORM_RMS = 0,          /* v / sqrt(mean(v^2) + eps) */
    QNN_NORM_LAYER = 1         /* (v - mean) / sqrt(var + eps), var the mean square of v - mean */
};

/*
 * One call between two blocks.  x is [t][d] with row stride ldx; residual, r
 * and h likewise.  Row i uses gate row i / (t / gates); the gate is
 * [gates][d], contiguous.  d is at most 32768.
 */
typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_norm_desc) */
    int32_t kind;              /* QNN_NORM_* of both norms */
    int32_t dtype;             /* of x and h */
    int32_t residual_dtype;    /* of residual and r: dtype or QNN_F32 */
    int32_t param_dtype;       /* of gate, weights and biases: dtype or QNN_F32 */
    int32_t post_norm;         /* 0: u = x; 1: u = N(x) * post_w + post_b */
    int32_t gates;             /* rows of the gate; t must be a multiple of it (ignored without a gate) */
    int32_t d;                 /* row length */
    int64_t t;                 /* rows; may be 0 */
    int64_t ldx, ldres, ldr, ldh;
    float scale;               /* of the gated branch */
    float eps;
} qnn_norm_desc;

/*
 *   u = post_norm ? N(x) * post_w + post_b : x
 *   r = residual + scale * gate * u
 *   h = N(r) * pre_w + pre_b
 *
 * in 32 bits, each output rounded once (h from the unrounded r).  residual,
 * gate, every weight and bias may be NULL (0, 1, 1, 0); r or h may be NULL
 * (not written), not both.  r may be the residual itself and h may be x (same
 * pointer and stride); no other overlap.  Pointers are aligned to their
 * element; 16-byte aligned rows take the faster loads.
 */
qnn_status qnn_block_norm(const qnn_norm_desc *d, const void *x, const void *residual, const void *gate,
                          const void *post_w, const void *post_b, const void *pre_w, const void *pre_b, void *r,
                          void *h, void *stream);

/* Scores and group scores of qnn_route_topk(). */
enum { QNN_SCORE_SOFTMAX = 0, QNN_SCORE_SIGMOID = 1 };
enum {
    QNN_GROUP_MAX = 0,         /* a group counts as its best expert */
    QNN_GROUP_TOP2 = 1         /* ... as the sum of its two best */
};

typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_route_desc) */
    int32_t dtype;             /* of the logits */
    int32_t experts;           /* 1 .. 1024 */
    int32_t k;                 /* experts a token goes to: 1 .. 32, at most experts */
    int32_t score;             /* QNN_SCORE_* */
    int32_t groups;            /* experts are split evenly into this many groups: 1 .. 32, dividing experts */
    int32_t top_groups;        /* groups a token may choose from: 1 .. groups */
    int32_t group_score;       /* QNN_GROUP_* */
    int32_t renormalise;       /* weights divided by their sum */
    float scale;               /* of the weights */
    int64_t t;                 /* tokens; may be 0 */
    int64_t ld;                /* row stride of the logits */
} qnn_route_desc;

/*
 * Chooses each token's k experts.  s = softmax or sigmoid of the logits; the
 * choice goes by s + bias (bias float[experts], may be NULL), first among
 * groups when top_groups < groups, in falling order, ties to the lowest index.
 * The weights are s of the chosen experts without the bias, divided by their
 * sum when renormalise is set, times scale.
 *
 * An expert whose logit is -inf or NaN cannot be chosen and counts for
 * nothing; a token that runs out of experts gets id -1 and weight 0 for the
 * rest (a row of -inf: all of them).
 *
 *   weights  device float[t][k]      ids  device int32[t][k]
 */
qnn_status qnn_route_topk(const qnn_route_desc *d, const void *logits, const float *bias, float *weights,
                          int32_t *ids, void *stream);

/*
 * The slots (token * k + choice) sorted by expert, each expert's in rising
 * order; ids outside [0, experts) are in no expert's list.
 *
 *   offsets   device int32[experts + 1]: expert e has places offsets[e] .. offsets[e+1]
 *   order     device int32[slots]: the slot at each place, -1 after the last
 *   position  device int32[slots]: the place of each slot, -1 for one left out
 *
 * slots below 2^31 - 2048, experts 1 .. 1024; workspace as
 * qnn_expert_plan_workspace_size() says (256-byte aligned; NULL when 0).
 */
qnn_status qnn_expert_plan_workspace_size(int64_t slots, int32_t experts, size_t *bytes);
qnn_status qnn_expert_plan(const int32_t *ids, int64_t slots, int32_t experts, int32_t *offsets, int32_t *order,
                           int32_t *position, void *workspace, size_t workspace_bytes, void *stream);

/* Activation of the matrix products. */
enum {
    QNN_ACT_NONE = 0,
    QNN_ACT_RELU = 1,
    QNN_ACT_SILU = 2,          /* v / (1 + exp(-v)) */
    QNN_ACT_GELU = 3,          /* v * Phi(v), with erf */
    QNN_ACT_GELU_TANH = 4      /* its tanh form */
};

/*
 * A weight matrix [rows][k], or one for each of `experts` experts; rows is m,
 * or 2 m for a gated product: m gate rows, then m up rows.  Weights are 16-bit
 * floats of type `dtype`, or packed signed 8/4/2-bit codes in the sub-byte
 * order above with one float scale a row.  experts * rows * k, with the rows
 * of an expert counted in 32s (gate and up rows in 8s each before that) and k
 * in 64s, is at most 2^40.
 */
typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_matmul_desc) */
    int32_t experts;           /* matrices: 1 for qnn_matmul_run(), 1 .. 1024 for the experts' products */
    int32_t m;                 /* output channels, at most 2^24 */
    int32_t k;                 /* input channels, at most 2^24; a multiple of 8/bits for packed weights */
    int32_t bits;              /* 16, 8, 4 or 2 */
    int32_t dtype;             /* QNN_F16 or QNN_BF16: x, residual, outputs and 16-bit weights */
    int32_t gated;             /* 1: y = act(gate) * up */
    int32_t act;               /* QNN_ACT_* */
} qnn_matmul_desc;

/*
 * Lays the weights out once, as the kernels read them, with scale and bias
 * beside them; the caller's buffers may be freed afterwards.  The image needs
 * qnn_matmul_image_size() bytes, 256-byte aligned, and may be used by any
 * number of concurrent calls.
 *
 *   w      device [experts][rows][k], 16-bit floats or packed codes (aligned to their element)
 *   scale  device float[experts][rows] or NULL (1); bias likewise or NULL (0)
 */
qnn_status qnn_matmul_image_size(const qnn_matmul_desc *d, size_t *bytes);
qnn_status qnn_matmul_prepare(const qnn_matmul_desc *d, const void *w, const float *scale, const float *bias,
                              void *image, size_t image_bytes, void *stream);

/*
 *   v = scale * (x w^T) + bias        (codes are multiplied as they are; 32-bit accumulation)
 *   y = residual + act(v)             or  residual + act(v_gate) * v_up
 *
 * rounded once.  x [t][k], residual [t][m] or NULL, y [t][m] of type dtype, or
 * float when out_f32 is set; t is at most 2^20, t * m at most 2^38.  y may be the residual itself (same pointer,
 * stride and type), no other overlap.  Workspace (256-byte aligned) as
 * qnn_matmul_workspace_size() says for the same d, t, x and ldx.
 */
qnn_status qnn_matmul_workspace_size(const qnn_matmul_desc *d, int64_t t, const void *x, int64_t ldx, size_t *bytes);
qnn_status qnn_matmul_run(const qnn_matmul_desc *d, const void *image, size_t image_bytes, int64_t t, const void *x,
                          int64_t ldx, const void *residual, int64_t ldres, void *y, int64_t ldy, int32_t out_f32,
                          void *workspace, size_t workspace_bytes, void *stream);

/*
 * The experts' products over a plan of qnn_expert_plan() (tokens * top slots,
 * at most 2^20 of them, top at most 1024, slots * m at most 2^38).
 *
 * qnn_experts_dispatch: row p of y is the product of x[order[p] / top] with
 *   the weights of the expert that place p belongs to; x [tokens][k],
 *   y [tokens * top][m].  Rows after the last place are zero.
 * qnn_experts_combine: x has a row per place, x [tokens * top][k];
 *   y[t] = residual[t] + sum_j weights[t][j] * product(position[t][j]), the sum in 32 bits in the order of j;
 *   choices without a place add nothing.  weights float[tokens][top].
 */
qnn_status qnn_experts_workspace_size(const qnn_matmul_desc *d, int64_t tokens, int32_t top, int32_t combine,
                                      const void *x, int64_t ldx, size_t *bytes);
qnn_status qnn_experts_dispatch(const qnn_matmul_desc *d, const void *image, size_t image_bytes, int64_t tokens,
                                int32_t top, const int32_t *offsets, const int32_t *order, const void *x, int64_t ldx,
                                void *y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream);
qnn_status qnn_experts_combine(const qnn_matmul_desc *d, const void *image, size_t image_bytes, int64_t tokens,
                               int32_t top, const int32_t *offsets, const int32_t *position, const float *weights,
                               const void *x, int64_t ldx, const void *residual, int64_t ldres, void *y, int64_t ldy,
                               void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------
 * The attention half of a block, for serving: rotary positions, a paged cache
 * of keys and values, attention over it, and cross attention to an encoder's
 * states.  Heads are strided (elements); a head's elements are contiguous.
 * ---------------------------------------------------------------------- */

/* Frequencies f_i of the pairs i < dim / 2 (radians a position):
 * f_i = base^(-2 i / dim), and for contexts `factor` times as long: */
enum {
    QNN_ROPE_NONE = 0,
    QNN_ROPE_LINEAR = 1,       /* f_i / factor */
    QNN_ROPE_BASE = 2,         /* base * factor^(dim / (dim - 2)) as the base (dim > 2) */
    QNN_ROPE_RAMP = 3          /* g f_i + (1 - g) f_i / factor, g = (context * f_i / 2 pi - low) / (high - low) in 0 .. 1:
                                  pairs that turn `high` times or more in the original context stay, those that turn
                                  `low` times or less are stretched */
};

typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_rope_scaling) */
    int32_t dim;               /* rotated elements of a head, even */
    int32_t scaling;           /* QNN_ROPE_* */
    int32_t context;           /* original context (QNN_ROPE_RAMP) */
    double base;               /* > 1 */
    double factor;             /* >= 1 */
    double low, high;          /* rotations (QNN_ROPE_RAMP), low < high */
} qnn_rope_scaling;

/*
 * The frequencies as the kernels take them: turns[i] (host, dim / 2 of them)
 * is f_i / 2 pi as a binary fraction of 64 bits, so that position * turns[i]
 * modulo 2^64 is the pair's phase, exact at any position of either sign.
 * Frequencies of one's own may be given the same way.
 */
qnn_status qnn_rope_turns(const qnn_rope_scaling *s, uint64_t *turns);

typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_rope_desc) */
    int32_t dtype;             /* of x and y */
    int32_t heads;
    int32_t head_dim;          /* at most 1024 */
    int32_t dim;               /* rotated elements, the first of a head: even, 0 .. head_dim */
    int32_t interleaved;       /* pairs (2 i, 2 i + 1), else (i, i + dim / 2) */
    int32_t wide;              /* positions are int64, else int32 */
    float amplitude;           /* of the rotated elements */
    int64_t t;                 /* tokens; t * heads below 2^31 */
    int64_t ldx, hx, ldy, hy;  /* strides of tokens and heads */
} qnn_rope_desc;

/*
 * y = x with every pair (a, b) of its rotated elements turned by the angle p f_i of its token's position p:
 *   amplitude * (a cos - b sin, a sin + b cos)
 * in 32 bits, rounded once; the other elements are copied.  A position -p turns back.  y may be x (same strides), no
 * other overlap.
 *   turns device uint64[dim / 2]    positions device int64 or int32 [t]
 */
qnn_status qnn_rope(const qnn_rope_desc *d, const uint64_t *turns, const void *positions, const void *x, void *y, void *stream);

/*
 * A cache of keys and values in pages.  Row r of page p and head h begins at
 * p * k_page + h * k_head + r * k_row elements of the keys (values likewise),
 * so any order of the dimensions may be given.  16-byte aligned rows: the
 * strides are multiples of 8, the pointers 16-byte aligned (else QNN_EALIGN).
 */
typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_cache_desc) */
    int32_t dtype;             /* QNN_F16 or QNN_BF16: keys, values, queries, outputs */
    int32_t kv_heads;          /* at most 1024 */
    int32_t head_dim;          /* a multiple of 8, at most 256 */
    int32_t page_size;         /* rows of a page */
    int64_t pages;
    int64_t k_page, k_head, k_row;
    int64_t v_page, v_head, v_row;
} qnn_cache_desc;

/*
 * The sequences of a call.  Sequence s has lengths[s] tokens, the call's new
 * ones included: token j of it lies in row j % page_size of page
 * table[s * ldt + j / page_size].  A table entry outside [0, pages) stands for
 * no page: nothing is written there, and its tokens are not attended to.
 * Tokens past the table's width are not in the cache.
 *
 * The call's t tokens are the sequences' new ones: ragged, sequence s has rows
 * offsets[s] .. offsets[s + 1] (rising; rows before the first and behind the
 * last are in no sequence: what they hold does not matter, and none is
 * written); else t / seqs rows each.  New token i of n is token lengths[s] - n + i.
 * The host sees t and seqs, not the offsets: rows in no sequence count when a
 * call's kernels are chosen (for speed alone), and a step of single tokens is
 * quicker without offsets.
 *
 * table int32, lengths int32[seqs], offsets int32[seqs + 1]: device.
 */
typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_batch_desc) */
    int32_t seqs;
    int32_t width;             /* pages of a row of the table; width * page_size at most 2^30 */
    int32_t ragged;            /* 1: with offsets */
    int64_t t;                 /* a multiple of seqs unless ragged */
    int64_t ldt;               /* row stride of the table */
} qnn_batch_desc;

typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_append_desc) */
    int32_t heads;             /* of q; 0: no queries */
    int32_t dim;               /* as in qnn_rope_desc; 0: nothing is rotated */
    int32_t interleaved, wide;
    float amplitude;
    int64_t ldk, hk, ldv, hv, ldq, hq, ldo, ho;  /* strides of tokens and heads: k, v, q, q_out */
} qnn_append_desc;

/*
 * Writes the sequences' new keys, rotated, and values to their places, and the
 * rotated queries to q_out (which may be q, same strides).  k and v [t][kv_heads][head_dim], q
 * [t][heads][head_dim].  The rotation goes by the token's place in its
 * sequence, or by positions[t] when given.  A token whose place is not in the
 * cache is not written.  Tokens of one call whose places are the same, and
 * keys and values in the same memory, leave the elements of either.
 */
qnn_status qnn_cache_append(const qnn_cache_desc *c, const qnn_batch_desc *b, const qnn_append_desc *d, const int32_t *table,
                            const int32_t *lengths, const int32_t *offsets, const uint64_t *turns, const void *positions,
                            const void *k, const void *v, const void *q, void *k_pages, void *v_pages, void *q_out,
                            void *stream);

typedef struct {
    uint32_t struct_size;      /* = sizeof(qnn_attention_desc) */
    int32_t heads;             /* of q, a multiple of kv_heads: query head h reads key head h / (heads / kv_heads) */
    int32_t causal;            /* 1: a new token sees the tokens up to itself; 0: all of its sequence */
    int32_t window;            /* > 0: it sees no token `window` or more before itself; 0: no limit */
    float scale;               /* of the products: normal, positive, at most FLT_MAX / 2 */
    int64_t q_seq, ldq, hq;    /* strides of q: sequences (not ragged), tokens, heads */
    int64_t o_seq, ldo, ho;    /* of out */
} qnn_attention_desc;

/*
 * out = sum_j softmax_j(scale * q . k_j) v_j over the tokens j that the new
 * token sees; zero where it sees none.  lse (or NULL), float[t][heads]: the
 * logarithm of the sum of exp(scale * q . k_j), -inf where there is none.
 *
 * table NULL: sequence s has the one page s (width at most 1), as for the
 * states of an encoder.  lengths NULL: every sequence is width * page_size
 * long.  q and out [t][heads][head_dim]; out overlaps nothing.  Rows of the
 * cache that no new token sees may hold anything, also NaN; those that one
 * sees are finite.
 *
 * 16-bit products are summed in 32 bits; the weights 2^(z - max) are rounded
 * to 16 bits before they multiply the values, the sum of them is not.
 * t * heads below 2^31.  Workspace as qnn_attention_workspace_size() says
 * (256-byte aligned; NULL when 0).
 */
qnn_status qnn_attention_workspace_size(const qnn_cache_desc *c, const qnn_batch_desc *b, const qnn_attention_desc *d,
                                        size_t *bytes);
qnn_status qnn_attention(const qnn_cache_desc *c, const qnn_batch_desc *b, const qnn_attention_desc *d, const int32_t *table,
                         const int32_t *lengths, const int32_t *offsets, const void *q, const void *k_pages,
                         const void *v_pages, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QNN_H */
