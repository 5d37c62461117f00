/*
 * eqat.h  --  C ABI of the MI355X (gfx950) quantized-linear library for
 * EfficientQAT (arXiv 2407.11062).
 *
 * The library implements the layer both training phases of the paper run on
 * every step:
 *   Block-AP (Sec. 3.2):  W_int = clamp(round(W/s) + z, 0, 2^N - 1)   Eq.(1)
 *                         What  = (W_int - z) * s                     Eq.(2)
 *                         Y = X * What^T, and the backward of App. B.
 *   E2E-QP  (Sec. 3.3):   W_int frozen and packed at N bits; only Eq.(2) runs.
 *
 * Conventions (all entry points)
 *   Layout     Row-major, contiguous.  X [T,I], W [O,I] (row = output channel),
 *              s,z [O,G] with G = I/g, Y,dY [T,O], dX [T,I], dW [O,I],
 *              ds,dz [O,G].  Group j of row o covers columns [j*g,(j+1)*g).
 *   Memory     Every pointer is a DEVICE pointer owned by the caller, 16-byte
 *              aligned.  The library never allocates or frees device memory and
 *              keeps no pointer of the caller (the optional timing aid at the end
 *              of this header creates HIP event objects while it is switched on).
 *              Each tensor must be smaller than 2 GiB.
 *   Dtypes     X,Y,dY,dX have desc.act_dtype; W,dW have desc.w_dtype; s,z,ds,dz
 *              are always fp32.  act bf16 selects the MFMA path (needs O % 8 == 0);
 *              act fp32 selects the fp32 path.
 *   Shapes     I % 32 == 0; g > 0, g % 32 == 0, g | I (group = -1 means g = I);
 *              bits in {2,3,4}; T >= 0, O >= 1; with bf16 activations I, O < 2^22.
 *   Stream     `stream` is a hipStream_t (NULL = default stream).  All work is
 *              enqueued there; no call synchronises.  Outputs are overwritten.
 *   Workspace  Caller-provided scratch of at least eqat_workspace_bytes(desc, op)
 *              bytes, 256-byte aligned; contents undefined afterwards.  The part of
 *              it that only lets workgroups share an output tile (few tokens: parts
 *              of the sums) may be missing: the codes and pairs do not depend on the
 *              token count, so that of 8192 tokens of a 4096 x 4096 layer serves one
 *              token as well.  Tiles are not shared then, and the sums are added up
 *              in another order.  Less than the call needs gives EQAT_ERR_WORKSPACE.
 *   Errors     Arguments are checked on the host before anything is launched and
 *              the first violation is returned; nothing is thrown or aborted.
 *   Numerics   round() is round-half-to-even of the correctly rounded binary32
 *              quotient w/s (bf16 weights are widened first), so integer codes
 *              and packed bytes are identical on every implementation.
 *              zbar = clamp(round(z), 0, 2^N-1) is used in place of z in every
 *              entry point (the zero point is stored at N bits when Block-AP ends,
 *              so the packed layer is exactly the layer Block-AP trained); the
 *              gradient passes straight through the rounding and the clamp.
 *              Preconditions (not checked): s a normal,
 *              finite, positive binary32 number (>= 2^-126; the min/max rule
 *              never gives less than 1e-10), |z| <= 2^20, all inputs finite.
 *   Determinism  Same inputs (and the same workspace size, if it is below
 *              eqat_workspace_bytes) give bitwise the same outputs.
 */
#ifndef EQAT_H_
#define EQAT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    EQAT_OK = 0,
    EQAT_ERR_NULL = 1,      /* a required pointer is NULL                        */
    EQAT_ERR_SHAPE = 2,     /* T < 0, I or O < 1, I % 32, O % 8 (bf16), >= 2 GiB */
                            /* or, with bf16 activations, I or O >= 2^22         */
    EQAT_ERR_BITS = 3,      /* bits not in {2,3,4}                               */
    EQAT_ERR_GROUP = 4,     /* group not -1 and (<= 0, % 32 != 0 or not | I)     */
    EQAT_ERR_DTYPE = 5,     /* unknown dtype value                               */
    EQAT_ERR_ALIGN = 6,     /* pointer not 16-byte (workspace: 256-byte) aligned */
    EQAT_ERR_WORKSPACE = 7, /* workspace missing or too small                    */
    EQAT_ERR_DEVICE = 8,    /* the HIP runtime refused a launch                  */
    EQAT_ERR_HYPER = 9      /* optimizer, attention, norm, rotary, gate constants  */
} eqat_status;

typedef enum { EQAT_F32 = 0, EQAT_BF16 = 1 } eqat_dtype;

typedef enum {
    EQAT_OP_FQ_FWD = 0, EQAT_OP_FQ_BWD = 1, EQAT_OP_Q_FWD = 2, EQAT_OP_Q_BWD = 3,
    EQAT_OP_QP_FWD = 4, EQAT_OP_QP_BWD = 5      /* eqat_qlinear_fwd_prepared / _bwd_prepared */
} eqat_op;

/* What eqat_unpack_state reads: the workspace left by eqat_fq_linear_fwd_keep, the one left by
 * eqat_qlinear_fwd_keep, or a layer prepared by eqat_qlinear_prepare. */
typedef enum { EQAT_STATE_FQ_KEPT = 0, EQAT_STATE_Q_KEPT = 1, EQAT_STATE_PREPARED = 2 } eqat_state_kind;

typedef struct eqat_desc {
    int64_t tokens;        /* T                                                  */
    int64_t in_features;   /* I                                                  */
    int64_t out_features;  /* O                                                  */
    int32_t bits;          /* N                                                  */
    int32_t group;         /* g, or -1 for one group per row (per-channel)       */
    int32_t act_dtype;     /* eqat_dtype of X, Y, dY, dX                         */
    int32_t w_dtype;       /* eqat_dtype of W, dW                                */
} eqat_desc;

/* Host-only helpers.  Sizes are 0 for an invalid descriptor. */
const char *eqat_status_string(int status);
eqat_status eqat_validate_desc(const eqat_desc *d);
size_t eqat_packed_w_bytes(const eqat_desc *d);   /* O * I*N/8                     */
size_t eqat_packed_z_bytes(const eqat_desc *d);   /* O * 4*ceil(G*N/32)            */
size_t eqat_workspace_bytes(const eqat_desc *d, int op);

/*
 * Per-group initialisation of step sizes and zero points.  The paper does not
 * say how s and z start; this is the usual asymmetric min/max rule in binary32:
 *   s = max((max - min) / (2^N - 1), 1e-10),  z = clamp(round(-min / s), 0, 2^N - 1).
 * In: W [O,I].  Out: s, z [O,G].  d->tokens is ignored.
 */
eqat_status eqat_init_minmax(const eqat_desc *d, const void *W, float *s, float *z, void *stream);

/*
 * Block-AP forward (Sec. 3.2, Eqs.(1),(2)):  Y = X * What^T.
 * What is rebuilt from W, s, z on the fly and never stored.
 */
eqat_status eqat_fq_linear_fwd(const eqat_desc *d, const void *X, const void *W, const float *s,
                               const float *z, void *Y, void *ws, size_t ws_bytes, void *stream);

/*
 * Block-AP backward (App. B, Eqs.(3)-(5), straight-through estimator):
 *   dX = dY * What
 *   dW = (dY^T X) where 0 <= round(w/s)+zbar <= 2^N-1, else 0            Eq.(5)
 *   ds[o,j] = sum over group of (dY^T X) * { round(w/s) - w/s | -zbar | 2^N-1-zbar }   Eq.(3)
 *   dz[o,j] = sum over group of (dY^T X) * { 0 in range | -s outside }                 Eq.(4)
 * Eq.(4) is printed with -1; -s is the derivative of Eq.(2) for a zero point in
 * integer units, and the printed form equals dz / s.  The appendix writes the
 * upper bound as 2^(N-1); Eq.(1)'s 2^N - 1 is used.
 * Any of dX, dW, ds, dz may be NULL and is then skipped.  dW, ds and dz do not depend on which outputs are asked for; dX asked for
 * together with any of them may come from a common launch that sums in another order than the launch for dX alone.
 */
eqat_status eqat_fq_linear_bwd(const eqat_desc *d, const void *X, const void *W, const float *s,
                               const float *z, const void *dY, void *dX, void *dW, float *ds, float *dz,
                               void *ws, size_t ws_bytes, void *stream);

/*
 * The same pair for a training step that runs both on unchanged (W, s, z): the forward leaves what Eq.(1) produced
 * (codes, which weights were clamped, the (s, zbar) pairs) in the workspace and the backward uses it instead of
 * running Eq.(1) a second time.  Both take a workspace of EQAT_OP_FQ_BWD size.  Precondition of _bwd_kept (not
 * checked): `ws` is untouched since eqat_fq_linear_fwd_keep ran on the same descriptor (any token count), W, s and z.
 * Results are bitwise those of eqat_fq_linear_fwd / eqat_fq_linear_bwd.  (With fp32 activations nothing is kept and
 * the backward works from W as always.)
 */
eqat_status eqat_fq_linear_fwd_keep(const eqat_desc *d, const void *X, const void *W, const float *s,
                                    const float *z, void *Y, void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_fq_linear_bwd_kept(const eqat_desc *d, const void *X, const void *W, const float *s,
                                    const float *z, const void *dY, void *dX, void *dW, float *ds, float *dz,
                                    void *ws, size_t ws_bytes, void *stream);

/*
 * The forward of the pair above from kept state: `ws` holds what eqat_fq_linear_fwd_keep or eqat_fq_quantize_batched
 * left for the same descriptor, W, s and z (not checked), and Eq.(1) is not run again.  Bitwise eqat_fq_linear_fwd.
 */
eqat_status eqat_fq_linear_fwd_kept(const eqat_desc *d, const void *X, const void *W, const float *s,
                                    const float *z, void *Y, void *ws, size_t ws_bytes, void *stream);

/*
 * Several matrices in ONE launch.  The linears of a decoder block are a few tens of megabytes each; the memory-bound
 * passes over them (min/max, Eq.(1), packing) last 10-25 microseconds apiece when launched one by one, a good part of it
 * filling and draining the chip.  n: 1 .. EQAT_MAX_BATCH; descs: n descriptors (host); every other argument: a HOST
 * array of n device pointers (or sizes), entry i belonging to descs[i].  All descriptors must agree in bits
 * (EQAT_ERR_BITS) and in the dtypes (EQAT_ERR_DTYPE); shapes and group sizes may differ.  Results are bitwise those of
 * n single calls.
 *   eqat_init_minmax_batched   as eqat_init_minmax.
 *   eqat_pack_batched          as eqat_pack.
 *   eqat_fq_quantize_batched   Eq.(1) of n linears before their Block-AP forward and backward: leaves every ws[i]
 *                              (EQAT_OP_FQ_BWD size for descs[i], tokens included) as eqat_fq_linear_fwd_keep would, for
 *                              eqat_fq_linear_fwd_kept / eqat_fq_linear_bwd_kept.  With fp32 activations nothing is kept
 *                              and nothing is launched.
 */
#define EQAT_MAX_BATCH 8
eqat_status eqat_init_minmax_batched(int n, const eqat_desc *descs, const void *const *W, float *const *s,
                                     float *const *z, void *stream);
eqat_status eqat_pack_batched(int n, const eqat_desc *descs, const void *const *W, const float *const *s,
                              const float *const *z, uint8_t *const *Wpacked, uint8_t *const *zpacked, void *stream);
eqat_status eqat_fq_quantize_batched(int n, const eqat_desc *descs, const void *const *W, const float *const *s,
                                     const float *const *z, void *const *ws, const size_t *ws_bytes, void *stream);

/*
 * Freeze after Block-AP (Sec. 3.2 last paragraph; App. E): W_q and z at N bits.
 * Layout (the paper fixes none): each row is a little-endian bit stream, code i
 * of the row in bits [i*N,(i+1)*N), stored as bytes, least significant first.
 *   Wpacked [O, I*N/8] bytes, zpacked [O, 4*ceil(G*N/32)] bytes (tail bits 0).
 * zbar = clamp(round(z), 0, 2^N-1) as in the Block-AP calls.  d->tokens is ignored.
 */
eqat_status eqat_pack(const eqat_desc *d, const void *W, const float *s, const float *z,
                      uint8_t *Wpacked, uint8_t *zpacked, void *stream);

/* Test aid: expand the packed streams to int32 codes [O,I] and zero points [O,G]
 * (either output may be NULL). */
eqat_status eqat_unpack(const eqat_desc *d, const uint8_t *Wpacked, const uint8_t *zpacked,
                        int32_t *codes, int32_t *zcodes, void *stream);

/*
 * E2E-QP forward (Sec. 3.3): What = (w_q - z) * s from the packed codes, Y = X * What^T.
 * With bf16 activations the packed arrays are read as they are, by one kernel and without the workspace: up to 16 tokens
 * (any group that is 32, 64 or a multiple of 128, else while T * I * 2 <= 64 KiB) and for some dozens by a memory-bound
 * matrix-vector kernel (the decode-time case of the paper's App. "Speedup with BitBLAS"), beyond by a GEMM made for few
 * output tiles, where it is the faster one (3-bit codes of three or more token tiles in two rounds of workgroups are
 * re-laid first); otherwise the codes are re-laid and the tiled MFMA GEMM runs.  eqat_fwd_route tells which.
 */
eqat_status eqat_qlinear_fwd(const eqat_desc *d, const void *X, const uint8_t *Wpacked, const float *s,
                             const uint8_t *zpacked, void *Y, void *ws, size_t ws_bytes, void *stream);

/*
 * E2E-QP backward (Sec. 3.3): dX = dY * What and
 *   ds[o,j] = sum over group of (dY^T X)[o,i] * (w_q[o,i] - z[o,j]).
 * dX or ds may be NULL (skipped); as in eqat_fq_linear_bwd, ds does not depend on which is asked for, dX may in the order of its sums (so, too, in the
 * calls below).  d->w_dtype is ignored.
 */
eqat_status eqat_qlinear_bwd(const eqat_desc *d, const void *X, const uint8_t *Wpacked, const float *s,
                             const uint8_t *zpacked, const void *dY, void *dX, float *ds,
                             void *ws, size_t ws_bytes, void *stream);

/*
 * The E2E-QP pair for a training step that runs forward and backward on unchanged (Wpacked, s, zpacked): the forward
 * leaves the codes in the library's working layout and the (s, z) pairs in the workspace, the backward uses them.
 * Both take a workspace of EQAT_OP_Q_BWD size; the forward never takes the
 * kernel for up to 16 tokens.
 * Precondition of _bwd_kept (not checked): `ws` untouched since eqat_qlinear_fwd_keep ran on the same descriptor (any
 * token count), Wpacked, s and zpacked.  Results are bitwise those of eqat_qlinear_fwd (more than 16 tokens) /
 * eqat_qlinear_bwd.
 */
eqat_status eqat_qlinear_fwd_keep(const eqat_desc *d, const void *X, const uint8_t *Wpacked, const float *s,
                                  const uint8_t *zpacked, void *Y, void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_qlinear_bwd_kept(const eqat_desc *d, const void *X, const uint8_t *Wpacked, const float *s,
                                  const uint8_t *zpacked, const void *dY, void *dX, float *ds,
                                  void *ws, size_t ws_bytes, void *stream);

/*
 * E2E-QP on a layer prepared once (Sec. 3.3: W_q is frozen in this phase and only s, or s and z, train).  The codes are
 * brought into the layout the GEMM kernels read and the packed zero points become floats, one time; a call then runs its
 * GEMMs behind one small launch that pairs the current step sizes with the zero points (O*G pairs: s changes every step;
 * the forward of a short batch makes the pairs itself).
 *   eqat_prepared_bytes    size of the prepared layer for this descriptor (tokens ignored; act_dtype matters:
 *                          with fp32 activations the prepared layer holds the dense stream); 0 for a bad descriptor.
 *   eqat_qlinear_prepare   Wpacked, zpacked (as eqat_pack wrote them) -> prepared (device, 256-byte aligned, owned by
 *                          the caller, at least eqat_prepared_bytes; too small gives EQAT_ERR_WORKSPACE).  Enqueues one
 *                          kernel (and, with fp32 activations, one device-to-device copy).
 *   eqat_qlinear_fwd_prepared / _bwd_prepared
 *                          Y, and dX / ds / dz, exactly (bitwise) as eqat_qlinear_fwd / eqat_qlinear_bwd, or, with a
 *                          float array z [O,G] given, as eqat_qlinear_fwd_z / eqat_qlinear_bwd_z.  z NULL: the zero
 *                          points the layer was prepared with.  dz = -s * group-sum (dY^T X) may be asked for either way.
 *                          Workspace of EQAT_OP_QP_FWD / EQAT_OP_QP_BWD size (the pairs; no room for codes).
 *                          The kernel for up to 16 tokens is not taken (there the results agree to
 *                          rounding).  The prepared layer is only read, except for
 *                          a few counters inside it that a launch uses and leaves at zero: calls on the same prepared
 *                          layer must not overlap in time (different streams need their own copy).
 *   eqat_qlinear_fwd_prepared_keep / eqat_qlinear_bwd_prepared_kept
 *                          The same two calls for a training step that runs both on unchanged (s, z): the forward takes
 *                          a workspace of EQAT_OP_QP_BWD size and leaves the pairs in it; the backward, given the same
 *                          workspace untouched and the same s and z, skips the pairing launch.  Results are bitwise
 *                          those of the plain pair.  With tokens = 0 the _keep call still writes the pairs.
 */
size_t eqat_prepared_bytes(const eqat_desc *d);
eqat_status eqat_qlinear_prepare(const eqat_desc *d, const uint8_t *Wpacked, const uint8_t *zpacked, void *prepared,
                                 size_t prepared_bytes, void *stream);
eqat_status eqat_qlinear_fwd_prepared(const eqat_desc *d, const void *X, const void *prepared, const float *s,
                                      const float *z, void *Y, void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_qlinear_bwd_prepared(const eqat_desc *d, const void *X, const void *prepared, const float *s,
                                      const float *z, const void *dY, void *dX, float *ds, float *dz,
                                      void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_qlinear_fwd_prepared_keep(const eqat_desc *d, const void *X, const void *prepared, const float *s,
                                      const float *z, void *Y, void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_qlinear_bwd_prepared_kept(const eqat_desc *d, const void *X, const void *prepared, const float *s,
                                      const float *z, const void *dY, void *dX, float *ds, float *dz,
                                      void *ws, size_t ws_bytes, void *stream);

/*
 * Test aid: the integer state the GEMM kernels work from, in plain arrays.  `kind` (eqat_state_kind) says what `state` is.
 *   codes   int32 [O,I]   W_int of Eq.(1) (Block-AP) or the frozen w_q (E2E-QP), or NULL
 *   clamped uint8 [O,I]   1 where Eq.(1) clamped the weight, i.e. where Eq.(5) zeroes dW; EQAT_STATE_FQ_KEPT only
 *                         (EQAT_ERR_NULL if asked of another kind), or NULL
 *   zbar    float [O,G]   the zero point Eq.(2) uses: clamp(round(z), 0, 2^N-1), or the unpacked N-bit zero point; or NULL
 * bf16 activations only (the fp32 path keeps no such state): EQAT_ERR_DTYPE otherwise.  d->tokens is ignored.
 */
eqat_status eqat_unpack_state(const eqat_desc *d, int kind, const void *state, int32_t *codes, uint8_t *clamped,
                              float *zbar, void *stream);

/*
 * E2E-QP with trained zero points (Sec. 3.3 and the ablation on the trainable parameters of E2E-QP: training z
 * promotes it from N bits to a floating-point tensor).  There is no Eq.(1) in this phase, so z enters Eq.(2) as it
 * is, WITHOUT rounding:  What = (w_q - z) * s,  Y = X * What^T.
 *   z [O,G] fp32 (device), any finite value.  Everything else as eqat_qlinear_fwd; workspace of EQAT_OP_Q_FWD.
 */
eqat_status eqat_qlinear_fwd_z(const eqat_desc *d, const void *X, const uint8_t *Wpacked, const float *s,
                               const float *z, void *Y, void *ws, size_t ws_bytes, void *stream);

/*
 * Backward of the above:  dX = dY * What,
 *   ds[o,j] = sum over group of (dY^T X)[o,i] * (w_q[o,i] - z[o,j]),
 *   dz[o,j] = -s[o,j] * sum over group of (dY^T X)[o,i]            (derivative of Eq.(2) with respect to z).
 * dX, ds, dz may each be NULL (skipped).  Workspace of EQAT_OP_Q_BWD.  d->w_dtype is ignored.
 */
eqat_status eqat_qlinear_bwd_z(const eqat_desc *d, const void *X, const uint8_t *Wpacked, const float *s,
                               const float *z, const void *dY, void *dX, float *ds, float *dz,
                               void *ws, size_t ws_bytes, void *stream);

/*
 * Block-AP step glue.  Sec. 3.2 trains the quantized block against the output of its full-precision counterpart with
 * a reconstruction loss; Sec. 4.1 ("Training") gives one learning rate for the quantization parameters and another
 * for the weights.  The paper names neither the form of the loss nor the optimizer; taken here: the mean squared
 * error over all elements, and AdamW (bias-corrected Adam with decoupled weight decay).
 *
 * eqat_recon_loss:   loss[0] = (1/n) sum (Y - Yref)^2,   dY = 2 (Y - Yref) / n   (dY may be NULL; it must not overlap Y or Yref).
 *   Y, Yref, dY: n elements of `dtype` (eqat_dtype), device, 16-byte aligned; loss: one float, device.
 *   ws: eqat_recon_loss_workspace_bytes() bytes, 256-byte aligned.  The sum is taken in a fixed order in binary32.
 *   n < 1 gives EQAT_ERR_SHAPE.
 */
size_t eqat_recon_loss_workspace_bytes(void);
eqat_status eqat_recon_loss(int64_t n, int32_t dtype, const void *Y, const void *Yref, float *loss, void *dY,
                            void *ws, size_t ws_bytes, void *stream);

/*
 * eqat_recon_loss for callers that cannot allocate device memory or pass a workspace: code under HIP graph capture,
 * tight serving or training loops, harnesses that forbid hipMalloc.  Same kernels, same results (bitwise) as
 * eqat_recon_loss; the workgroup partials live in an 8 KiB array inside the library's device image (one copy per GPU,
 * held until the process ends) instead of `ws`.  The call allocates and frees nothing.
 *   Limit: none on n; the array holds the 2048 partials that are the most a launch ever uses (a library built with a
 *   larger eqat_recon_loss_workspace_bytes() returns EQAT_ERR_WORKSPACE here).
 *   The address of the array is looked up on the first call on each device (hipGetSymbolAddress; failure gives
 *   EQAT_ERR_DEVICE): make that first call outside stream capture.
 *   All calls on one GPU share the array: calls that may run at the same time on one GPU (different streams) race on
 *   it and must be ordered by the caller.  Nothing needs clearing between calls.
 */
eqat_status eqat_recon_loss_static(int64_t n, int32_t dtype, const void *Y, const void *Yref, float *loss, void *dY,
                                   void *stream);

/*
 * eqat_block_ap_update: one AdamW step, in place, on the three trained tensors of a linear in ONE launch, taking the
 * gradients as eqat_fq_linear_bwd wrote them (dW in W's dtype, ds and dz fp32).  Per element, in binary32:
 *   p <- p - lr wd p;  m <- b1 m + (1-b1) g;  v <- b2 v + (1-b2) g^2;
 *   p <- p - lr (m / (1 - b1^step)) / (sqrt(v / (1 - b2^step)) + eps)          (then s <- max(s, 1e-10), see below)
 * with lr = lr_w, wd = weight_decay_w for W and lr_q, weight_decay_q for s and z.  Moments are fp32 arrays of the
 * parameter's shape, zero before the first step, owned by the caller.  A NULL parameter pointer (W, s or z) skips that
 * tensor together with its gradient and moments (E2E-QP trains s alone).  d->tokens and d->act_dtype are ignored.
 * A bf16 W is rounded to nearest even after the update; steps smaller than half an ulp are lost, so W should be kept
 * in fp32 while it is trained.  Constants outside 0 <= beta < 1, eps >= 0, step >= 1 give EQAT_ERR_HYPER.
 * The updated step sizes are held at or above 1e-10, the floor of their min/max initialisation (Eq.(1) divides by s, and
 * nothing else keeps an optimizer step from crossing zero): s <- max(s, 1e-10).
 */
typedef struct eqat_adamw {
    float lr_w;             /* learning rate of the weights (Sec. 4.1: 2e-5 at 2 bit, 1e-5 at 3 and 4 bit)   */
    float lr_q;             /* learning rate of step sizes and zero points (Sec. 4.1: 1e-4)                  */
    float beta1, beta2, eps;
    float weight_decay_w, weight_decay_q;
    int32_t step;           /* number of this update, counted from 1                                         */
} eqat_adamw;
eqat_status eqat_block_ap_update(const eqat_desc *d, const eqat_adamw *h, void *W, float *s, float *z,
                                 const void *dW, const float *ds, const float *dz, float *mW, float *vW,
                                 float *ms, float *vs, float *mz, float *vz, void *stream);

/*
 * Test aid (host only, nothing is launched): how the forward (gemm = 0), dX (gemm = 1) or dW (gemm = 2: tile rows are
 * in-features, tile columns out-features, K runs over the tokens) GEMM of this descriptor (bf16 activations, tokens >= 1)
 * divides its output tiles and their K range among its workgroups, as the kernel itself works it out.  item[12] = { tile row, tile column, first and past-the-last K-tile pair of this piece,
 * number of workgroups that contribute to the tile, index of the first of them within its XCD (workgroup = index * 8 +
 * XCD, XCD = block % 8), 1 if the tile is split among a group of workgroups (else pieces come from runs), index of the
 * tile's counter, workgroups in the launch, K-tile pairs per tile, tile rows, tile columns }; *exists = 0 past the last
 * item j of workgroup `block`.  EQAT_ERR_SHAPE for block outside the launch, gemm not 0, 1 or 2, j < 0.  Lets a test check,
 * without a GPU, that every K-tile pair of every tile is computed exactly once for any shape.
 * This is the launch of the tile kernels, given all the workspace it asks for.  A forward or dX may take another kernel altogether
 * (eqat_fwd_route, eqat_dx_route), one of few output tiles may run in the kernel that eqat_shared_item is about, and dX and dW of one call
 * may share a launch (eqat_dx_route).
 */
eqat_status eqat_plan_item(const eqat_desc *d, int gemm, int block, int j, int32_t *item, int32_t *exists);

/*
 * Test aid (host only, nothing is launched): the same for a forward (gemm = 0) or dX (gemm = 1) with at most 256 output tiles of
 * 128 x 128, whose tiles are shared by one to four workgroups, a stretch of the K-tile pairs each (two groups of waves of a
 * workgroup take the tiles of a pair).  *exists = 0 where another kernel computes it (dX: asked for alone), and past the last workgroup; else
 * item[10] = { tile row, tile column, first and past-the-last K-tile pair of workgroup `block`, which part of the tile this is, parts
 * of the tile, workgroups in the launch, K-tile pairs per tile, tile rows, tile columns }.  The parts of a tile are counted in at the
 * counter with the number of the tile.
 */
eqat_status eqat_shared_item(const eqat_desc *d, int gemm, int block, int32_t *item, int32_t *exists);

/*
 * Test aid (host only, nothing is launched): the bytes [*first, *end) of a workspace of `ws_bytes` bytes, for a call of kind `op`
 * (eqat_op), within which its forward (gemm = 0), dX (1) or dW (2) launch on a GPU of `cus` compute units (8 or more) writes the
 * accumulator parts of tiles that several workgroups share; *end = *first where it writes none.  EQAT_ERR_WORKSPACE for a
 * size that the call itself refuses.  bf16 activations, tokens >= 1.
 */
eqat_status eqat_plan_scratch(const eqat_desc *d, int op, int gemm, int cus, size_t ws_bytes, size_t *first, size_t *end);

/*
 * Test aid (host only, nothing is launched): the kernel that a forward of this descriptor (bf16 activations, tokens >= 1)
 * takes, from the packed arrays as they are (source 1: eqat_qlinear_fwd, 2: eqat_qlinear_fwd_z) or from codes in the working
 * layout (0: every other forward).  route[3] = { 0 tiled GEMM (which one: eqat_shared_item); 1 GEMM for few tiles; 2 matrix-vector with streamed
 * tokens; 3 matrix-vector, any group; 4 matrix-vector, 5 the same segment by segment, 6 the same in pairs of lookups;
 * 7 a re-layout of the codes, then 1,  tokens,  rows that a workgroup computes (0 for the tiled GEMM) }.  Lets a test
 * assert that its sizes reach the kernel it is about.
 */
eqat_status eqat_fwd_route(const eqat_desc *d, int source, int32_t *route);
/* Test aid (host only): what computes dX in a call with the workspace of eqat_workspace_bytes.  route[2] = { asked for alone: the token tile of the
 * kernel for few output tiles, 0: another kernel;  asked for with dW, ds or dz (block_ap: eqat_fq_linear_bwd, else the E2E-QP calls): -1 a launch of
 * its own, as alone; else a launch that it shares with dW: 0, 1 256 x 256 tiles (1: contraction of no whole K-tile pairs), else such a token tile }. */
eqat_status eqat_dx_route(const eqat_desc *d, int block_ap, int32_t *route);

/*
 * The key-value cache of a served model, in 4 bits.  (Not part of the paper's method: it is what a decoder reads beside the packed weights at every token.)
 *
 *   In groups of `group` neighbouring elements of a key or a value (of one token and head), sixteen steps from the least element to the greatest:
 *     m = f16(min x),  s = f16(max((max x - min x) / 15, 2^-24)),  c = clamp(round((x - m) / s), 0, 15),  x^ = m + s c
 *   in binary32 (the quotients correctly rounded, round() half to even), f16 the nearest binary16 number.  A group with an element that is not finite, or beyond
 *   binary16 (65504), stands as NaN; one that spans less than about 2^-16 is held in steps of 2^-24.
 *
 *   Pool       eqat_kv_pool_bytes(desc) bytes of device memory, 256-byte aligned, owned by the caller; of any size (offsets are 64 bits; fewer than 2^31 records of
 *              32 tokens and a head), of any contents at first.
 *              It is a number of pages of `page_tokens` tokens; how a page is laid out is the library's own.  Bytes per token and head: head_dim + 8 head_dim / group.
 *   Sequences  An eqat_kv_batch says, in device arrays, where the sequences of a call stand: sequence b holds lens[b] tokens, its position p on page
 *              table[b * table_stride + p / page_tokens] (at p % page_tokens), and its newest starts[b+1] - starts[b] tokens are the rows starts[b] .. starts[b+1] - 1 of
 *              the call's tensors: lens counts them in.  Either number may be 0, and there may be more new tokens than held ones (the first of them, which stand
 *              before the beginning, are not there).  The host gives bounds only (tokens, max_new, max_len), so that a captured graph serves lengths, pages and
 *              numbers of new tokens that change between its replays.  What lies beyond the bounds, or on a page outside the pool, is taken as not there: not
 *              written, read as zeros, not attended to; the tokens within keep their positions (a step replayed past the end writes nothing).  Of a sequence with
 *              more new tokens than max_new the first max_new rows are taken; the others, and rows from starts[sequences] on, are left as they are.  Nothing
 *              outside the tensors and the pool is touched whatever stands in the arrays.
 *   Tensors    [tokens, heads, head_dim] with any strides (in elements, of a token and of a head; elements of a head are contiguous), such as slices of the rows of
 *              a stacked q|k|v projection.  Pointers and strides in bytes are multiples of 16.
 *   Types      desc.act_dtype (bf16 or fp32) for every tensor; lse is fp32.
 */
typedef struct eqat_kv_desc {
    int64_t pages;          /* of the pool, below 2^31                                          */
    int32_t heads;          /* of keys and values                                               */
    int32_t head_dim;       /* 64, 128 or 256                                                   */
    int32_t group;          /* 32, 64, 128 or 256, at most head_dim, or -1: head_dim            */
    int32_t page_tokens;    /* a multiple of 32                                                 */
    int32_t act_dtype;      /* eqat_dtype                                                       */
} eqat_kv_desc;

typedef struct eqat_kv_batch {
    const int32_t *table;   /* [sequences, table_stride] pages, device                          */
    const int32_t *lens;    /* [sequences] tokens held, the newest included, device             */
    const int32_t *starts;  /* [sequences + 1] first rows, not decreasing, starts[0] = 0, device */
    int64_t tokens;         /* rows of the call's tensors: starts[sequences] or more            */
    int32_t sequences, table_stride;
    int32_t max_new;        /* no sequence has more newest tokens                               */
    int32_t max_len;        /* none holds more tokens                                           */
} eqat_kv_batch;

typedef struct eqat_kv_attn {
    int32_t q_heads;        /* a multiple of desc.heads: query head h reads head h / (q_heads / heads) */
    int32_t causal;         /* not 0: a query sees no position after its own; 0: those after it too    */
    int32_t window;         /* > 0: of the positions up to its own it sees only the last `window`      */
    float scale;            /* of the scores, up to 2^100; 0: 1 / sqrt(head_dim)                       */
} eqat_kv_attn;

size_t eqat_kv_pool_bytes(const eqat_kv_desc *d);                       /* 0 for a bad descriptor */

/* The newest tokens of every sequence into the cache.  Strides of K and V in elements: { token, head }. */
eqat_status eqat_kv_write(const eqat_kv_desc *d, const eqat_kv_batch *b, const void *K, const int64_t *k_strides, const void *V,
                          const int64_t *v_strides, void *pool, void *stream);

/* The newest tokens of every sequence (all of them where starts[b+1] - starts[b] = lens[b]) as values.  K or V may be NULL (skipped). */
eqat_status eqat_kv_read(const eqat_kv_desc *d, const eqat_kv_batch *b, void *K, const int64_t *k_strides, void *V, const int64_t *v_strides,
                         const void *pool, void *stream);

/*
 * Softmax attention of the newest tokens' queries over what their sequences hold (write first, then attend):
 *   out[t, h] = sum over j of softmax_j(scale q[t, h] . k^_j) v^_j,   lse[t, h] = ln(sum over j of exp(scale q . k^_j)),
 * j over the positions that the query, at position lens[b] - (new tokens) + (its place among them), sees.  A query that sees none gives zeros and lse -inf.
 * NaN or infinities at positions that a query does not see do not reach it.  Scores, softmax and sums are binary32.  With fp32 tensors the results are as near as
 * binary32 arithmetic; with bf16 the products of p and a value's step are rounded to 11 bits (or to 2^-36 of their largest, where that is more).  Where max_new x q_heads / heads
 * is more than 64, it may be p (or to 2^-36 of the largest), queries with the scale, keys and values that are rounded to 11 bits instead, keys and values to 2^-24 where
 * that is more (below 2^-13; the cache has no finer steps).
 *   Q, out: [tokens, q_heads, head_dim];  lse: [tokens, q_heads] contiguous, or NULL.
 *   ws: eqat_kv_workspace_bytes bytes (independent of the batch but for max_new and max_len), 256-byte aligned, ZEROED ONCE by the caller before its first use.  Every call
 *   leaves the counters in it at zero; calls that share a workspace must not overlap in time.
 * EQAT_ERR_HYPER for a scale that is negative, NaN or more than 2^100, or a negative window.  Queries of any size serve, as long as scale q and the scores are binary32
 * numbers.
 */
size_t eqat_kv_workspace_bytes(const eqat_kv_desc *d, const eqat_kv_batch *b, int q_heads);
eqat_status eqat_kv_attention(const eqat_kv_desc *d, const eqat_kv_batch *b, const eqat_kv_attn *a, const void *Q, const int64_t *q_strides,
                              void *out, const int64_t *out_strides, float *lse, const void *pool, void *ws, size_t ws_bytes, void *stream);

/*
 * What a decoder layer computes around its quantized linears: the norm in front of them, the rotary positions of queries and keys, the gate of the feed-forward.  (Not part of the
 * paper's method: what stands between the linears of the blocks that it trains and serves.)
 *
 * Root-mean-square norm with the residual's addition.
 *   S = X + R, rounded to the activations' type (R NULL: S = X);   Y = w S / sqrt(mean S^2 + eps), the mean over the row's `width` elements of S as it stands (w NULL: ones)
 *   codes, scales   Y in 8 bits instead of, or beside, Y: of `group` neighbouring elements scale = max(max |Y| / 448, 2^-126), codes = e4m3(Y / scale) (the finite-only 8-bit
 *                   float with 4 exponent bits, largest 448), from Y before it is rounded; to nearest, ties to even (max / 448 and the
 *                   quotient are binary32, each rounded once).
 *   Backward, of S (what the forward left in S, or its X without R), the gradients dY of Y and dS of S (along the residual; NULL: none):
 *                   dX = dS + rstd (w dY - S rstd^2 mean(w dY S)),  which is the gradient of X and of R;   dw = sum over the rows of dY S rstd,   rstd = 1 / sqrt(mean S^2 + eps).
 *   All tensors are contiguous: X, R, S, Y, dY, dS, dX [tokens, width] in act_dtype, w [width] in w_dtype, codes [tokens, width] bytes, scales [tokens, width / group] and dw [width]
 *   fp32, of any size (offsets are 64 bits).  S may be X or R itself, and so may Y (not the one that S is), dX may be dY, dS or S (a row is read before it is written); no other overlap.
 *   Sums, means and products are binary32: a row whose squares pass binary32 gives zeros, a NaN or infinity stays in its row (and in dw).
 *   With eps = 0 (allowed) a row of zeros gives NaN, as the formula does, and one whose mean square is below 2^-126 (elements around 2^-63 and less) loses bits of it.
 *   width: a multiple of 8, up to 32768 (a multiple of `group` where codes are asked for); group 32, 64, 128, 256 or 512, or -1: one scale a row.
 *   tokens >= 0 of any number below 2^31; none leaves dw at zero.  eps >= 0, finite (EQAT_ERR_HYPER otherwise).
 *   ws: eqat_norm_workspace_bytes(d) bytes, 256-byte aligned, wanted for dw only; contents undefined before and after; calls that share one must not overlap in time.
 * S, Y, (codes and scales together), dX and dw may each be NULL (skipped).  Same inputs give bitwise the same outputs.
 */
typedef struct eqat_norm_desc {
    int64_t tokens;
    int32_t width;
    int32_t group;          /* of a scale; ignored without codes                                */
    int32_t act_dtype;      /* eqat_dtype                                                       */
    int32_t w_dtype;        /* eqat_dtype of w                                                  */
    float eps;
} eqat_norm_desc;

eqat_status eqat_norm_fwd(const eqat_norm_desc *d, const void *X, const void *R, const void *w, void *S, void *Y, uint8_t *codes, float *scales, void *stream);
size_t eqat_norm_workspace_bytes(const eqat_norm_desc *d);                /* 0 for a bad descriptor or no tokens */
eqat_status eqat_norm_bwd(const eqat_norm_desc *d, const void *S, const void *w, const void *dY, const void *dS, void *dX, float *dw, void *ws, size_t ws_bytes, void *stream);

/*
 * Rotary positions.  The first `part` elements of every head are part / 2 pairs, (i, i + part / 2) or, interleaved, (2 i, 2 i + 1); pair i of a token at position p becomes
 *   (a, b) -> amplitude (a cos t - b sin t, b cos t + a sin t),   t = p frequencies[i],
 * the other elements stay.  The frequencies are the caller's (device, fp32, part / 2 of them): base^(-2 i / part), or any scaling of them for long contexts.  The angle is held in
 * binary64, so that far positions keep it; cosine and sine are good to binary32.  `inverse` turns back by the same angles with the same amplitude: the transpose, which is
 * the backward pass (gradients of the turned tensors in, of the tensors out).
 *   positions   int32 [tokens], device, any values.
 *   Q, K        [tokens, heads, head_dim] in act_dtype, strides { token, head } in elements; pointers and strides in bytes are multiples of 16, elements of a head contiguous.
 *               Either may be NULL (with its output).  An output may be its input (same pointer and strides); no other overlap.
 *   head_dim    a multiple of 8 up to 1024; part even, 2 .. head_dim.  tokens x heads below 2^31; tensors of any size.
 * EQAT_ERR_HYPER for an amplitude that is not finite.
 */
typedef struct eqat_rotary_desc {
    const float *frequencies;   /* [part / 2], device                                            */
    int32_t head_dim, part;
    int32_t interleaved;        /* not 0: pairs are neighbours                                   */
    int32_t act_dtype;          /* eqat_dtype                                                    */
    float amplitude;
} eqat_rotary_desc;

eqat_status eqat_rotary(const eqat_rotary_desc *d, int64_t tokens, const int32_t *positions, const void *Q, const int64_t *q_strides, int q_heads, void *q_out,
                        const int64_t *q_out_strides, const void *K, const int64_t *k_strides, int k_heads, void *k_out, const int64_t *k_out_strides, int inverse, void *stream);

/*
 * A served model's step into the 4-bit cache, in one launch: the queries of the newest tokens turned into q_out, their keys turned and, rounded to act_dtype, written into the cache
 * with the values; the positions are those that `b` gives.  Bitwise what eqat_rotary (with those positions) and eqat_kv_write do one after the other.  K and V are only read.  Rows
 * of q_out behind the last sequence, and those of a sequence beyond b->max_new, are left as they are; queries of tokens that are not there (beyond the bounds, on no page) are
 * turned by their position all the same.  head_dim and act_dtype of both descriptors have to agree (EQAT_ERR_SHAPE, EQAT_ERR_DTYPE).  q_out may be Q itself, with its strides.
 */
eqat_status eqat_kv_rotary_write(const eqat_kv_desc *d, const eqat_kv_batch *b, const eqat_rotary_desc *r, const void *Q, const int64_t *q_strides, int q_heads, void *q_out,
                                 const int64_t *q_out_strides, const void *K, const int64_t *k_strides, const void *V, const int64_t *v_strides, void *pool, void *stream);

/*
 * Gated feed-forward:  H = act(G) U,  G = X Wg^T and U = X Wu^T two projections stacked in one layer of 2 F output rows, the F rows of Wg first.
 *   kind   EQAT_GATE_SILU  act(x) = x / (1 + exp(-x));   EQAT_GATE_GELU  act(x) = x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))) / 2
 *
 * eqat_gate_fwd / _bwd: element by element, for projections of any kind (Y = [G | U] as eqat_fq_linear_fwd leaves it on stacked weights).
 *   Y, dY [tokens, 2 F], H, dH [tokens, F] in `dtype`, contiguous; F a multiple of 8, tokens x F below 2^34.  dY = [dH U act'(G) | dH act(G)].  In the backward pass H, or dY, may be NULL (skipped); dY
 *   may be Y itself, H may be dH itself; no other overlap.
 *
 * eqat_gated_fwd / _bwd: both projections from the packed layer, the activation and the product in one kernel (G and U are not rounded and not stored):
 *   d          the stacked layer: out_features = 2 F, F a multiple of 8; tokens, in_features, bits, group, act_dtype as for eqat_qlinear_fwd (w_dtype is ignored; out_features x in_features below 2^30).
 *   forward    X -> H [tokens, F].
 *   backward   X, dH -> dY = [dH U act'(G) | dH act(G)] [tokens, 2 F], and H again (either may be NULL): both projections are made anew, so that a training step keeps X
 *              alone between its passes (H bitwise that of the forward where both take the same kernel: more than 64 tokens, or fp32); dY is what eqat_qlinear_bwd of the layer takes (dX, ds), H the input of the next linear in its own backward pass.
 *   _prepared  the same on a layer prepared by eqat_qlinear_prepare, which is only read; s the current step sizes, the zero points those that it was prepared with.
 *   No tensor may overlap another.
 *   ws         eqat_gated_workspace_bytes(d) bytes, 256-byte aligned, contents undefined before and after.  That of more tokens serves fewer, too.
 *              Calls that share one must not overlap in time.
 * With fp32 activations all of it is binary32.  With bf16 activations the weights that the layer stands for, q s - z s, are rounded to bf16 before the products, as in every other call with bf16
 * activations; sums, activation and gradient are binary32, and each result is rounded once.
 * EQAT_ERR_HYPER for an unknown kind.
 */
typedef enum { EQAT_GATE_SILU = 0, EQAT_GATE_GELU = 1 } eqat_gate_kind;

eqat_status eqat_gate_fwd(int64_t tokens, int64_t F, int32_t dtype, int kind, const void *Y, void *H, void *stream);
eqat_status eqat_gate_bwd(int64_t tokens, int64_t F, int32_t dtype, int kind, const void *Y, const void *dH, void *dY, void *H, void *stream);
size_t eqat_gated_workspace_bytes(const eqat_desc *d);                 /* 0 for a bad descriptor */
eqat_status eqat_gated_fwd(const eqat_desc *d, int kind, const void *X, const uint8_t *Wpacked, const float *s, const uint8_t *zpacked, void *H, void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_gated_bwd(const eqat_desc *d, int kind, const void *X, const uint8_t *Wpacked, const float *s, const uint8_t *zpacked, const void *dH, void *dY, void *H,
                           void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_gated_fwd_prepared(const eqat_desc *d, int kind, const void *X, const void *prepared, const float *s, void *H, void *ws, size_t ws_bytes, void *stream);
eqat_status eqat_gated_bwd_prepared(const eqat_desc *d, int kind, const void *X, const void *prepared, const float *s, const void *dH, void *dY, void *H,
                                    void *ws, size_t ws_bytes, void *stream);

/*
 * Optional per-kernel timing (measurement aid, not part of the paper's method).
 * Between eqat_profile_start() and eqat_profile_stop() every kernel launch of the
 * library is bracketed by a pair of HIP events recorded on the caller's stream.
 * eqat_profile_stop() waits for those events and writes, per kernel class k in
 * [0, eqat_profile_kernels()), the summed elapsed milliseconds and the number of
 * launches into host arrays of length n; it then switches timing off.  Event
 * objects are created on first use and kept until the process ends.  The calls
 * may come from several threads; a session is process-wide (one start, one stop).
 */
int eqat_profile_kernels(void);
const char *eqat_profile_kernel_name(int k);
eqat_status eqat_profile_start(void);
eqat_status eqat_profile_stop(double *total_ms, int64_t *launches, int n);

#ifdef __cplusplus
}
#endif
#endif /* EQAT_H_ */
