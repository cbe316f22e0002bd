/*
 * dcnv4.h -- C ABI of the MI355X (gfx950) DCNv4 spatial-aggregation library.
 *
 * The operator (paper Sec. 3.1, Eq. 1-2, with the softmax over the taps removed as
 * "Enhancing dynamic property" prescribes; thread/channel organisation after
 * Sec. 3.2 "Eliminating redundant workload / memory instructions"):
 *
 *   y[n,oh,ow,g*Cg+c] = sum_{k} m[n,oh,ow,g,k] * bilinear(x[n,:,:,g*Cg+c], hy_k, wx_k)
 *   hy_k = oh*stride_h - pad_h + i*dil_h + offset_scale * offset[n,oh,ow,g,k,1]
 *   wx_k = ow*stride_w - pad_w + j*dil_w + offset_scale * offset[n,oh,ow,g,k,0]
 *   k = j*kernel_h + i   (j: window column, slow; i: window row, fast)
 *
 * Whole-number coordinates are pixel centres; the four neighbours are floor and
 * floor+1; a neighbour outside the image reads zero.  m is used as given
 * (unbounded, not normalised).
 *
 * Memory: every tensor pointer is a DEVICE pointer owned by the caller, dense and
 * contiguous, 16-byte aligned, all of one element type `dtype`:
 *   x, grad_x            [N, H,  W,  G*Cg]     channel-last
 *   offset, grad_offset  [N, Ho, Wo, G, 9, 2]
 *   mask, grad_mask      [N, Ho, Wo, G, 9]
 *   y, grad_y            [N, Ho, Wo, G*Cg]
 *   offset_mask, grad_offset_mask  [N, Ho, Wo, G, 32]   (the *_merged entry points: per (pixel, group)
 *                        the 18 offsets, then the 9 mask values, then 5 unused entries)
 * with (Ho, Wo) as returned by dcnv4_output_hw().  The library allocates nothing and
 * keeps nothing between calls except the test switches below; it enqueues its kernels
 * on `stream` (a hipStream_t, NULL = the default stream) and returns without
 * synchronising.  Outputs must not alias inputs.  (The module entry points further down
 * need memory for the tensors between their layers: dcnv4_module_forward takes it from the
 * caller, dcnv4_module_forward_static from a 32 MiB device array that is part of the library.)
 *
 * Supported: square windows of 3x3 (every entry point and kernel), 1x1 and 5x5 (dcnv4_forward in
 * F32 and F16, dcnv4_backward in F32, through the direct kernels; 5x5 forward needs Cg >= 16; K = 1 or
 * 25 replaces 9 in the layouts above); stride, dilation >= 1; pad >= 0; Cg in {8, 16, 32, 64};
 * dtype F32 or F16.  F16 is fp16 storage with fp32 positions and accumulation and one
 * round-to-nearest at the store; where the forward runs out of its ring of input rows
 * in LDS (fp16, Cg 16, maps of several hundred pixels) the four products m * corner
 * weight of a tap are rounded to fp16 before they multiply the (fp16) inputs; products
 * and sums stay fp32.  The fp16 backward exists for Cg 8, 16 and 32.  Byte
 * offsets inside one image are 32-bit: one image of x and of y, and the farthest
 * clamped sampling position (about twice the image extent), must stay below 2 GiB;
 * larger images are refused with DCNV4_ERR_UNSUPPORTED.
 *
 * Errors: every call validates its arguments on the host first and returns a
 * nonzero DCNV4_ERR_* without launching or writing anything; nothing throws or
 * aborts.  DCNV4_ERR_LAUNCH reports a HIP launch failure.
 */
#ifndef DCNV4_H
#define DCNV4_H

#ifdef __cplusplus
extern "C" {
#endif

enum { DCNV4_F32 = 0, DCNV4_F16 = 1 };

enum {
    DCNV4_OK = 0,
    DCNV4_ERR_NULL = 1,        /* a required pointer is NULL */
    DCNV4_ERR_SHAPE = 2,       /* a size is non-positive, the window does not fit, or a workspace is too small */
    DCNV4_ERR_UNSUPPORTED = 3, /* kernel size, Cg, dtype or tensor size outside the supported set */
    DCNV4_ERR_ALIGN = 4,       /* a tensor pointer is not 16-byte aligned */
    DCNV4_ERR_LAUNCH = 5,      /* the HIP runtime refused the launch */
    DCNV4_ERR_TOO_LARGE = 6    /* dcnv4_module_forward_static: the call needs more than the built-in workspace */
};

/* Output extent of the sliding window: Ho = (H + 2*pad_h - dil_h*(kernel_h-1) - 1)/stride_h + 1,
 * likewise Wo (Sec. 3.1: the operator slides like a regular convolution).
 * Host pointers H_out/W_out; returns DCNV4_ERR_SHAPE if the window does not fit. */
int dcnv4_output_hw(int H, int W, int kernel_h, int kernel_w, int stride_h, int stride_w,
                    int pad_h, int pad_w, int dil_h, int dil_w, int *H_out, int *W_out);

/* Forward aggregation, Eq. 1-2 (gather the 4 neighbours of each of the 9 taps for a run of
 * channels, interpolate, modulate by m, reduce over the taps).  Overwrites y. */
int dcnv4_forward(const void *x, const void *offset, const void *mask, void *y,
                  int N, int H, int W, int G, int Cg,
                  int kernel_h, int kernel_w, int stride_h, int stride_w,
                  int pad_h, int pad_w, int dil_h, int dil_w,
                  float offset_scale, int dtype, void *stream);

/* The same with offsets and mask values in ONE buffer [N,Ho,Wo,G,32].  Sec. 3.2 "Micro design" merges
 * the two linear layers that produce offsets and mask values into one; this is the tensor such a
 * layer hands over when its 27 outputs per group are padded to 32 (this library's choice: records
 * of 64 bytes in fp16, 128 in fp32, never straddling more than two cache lines).  Entries 0..17 of
 * a (pixel, group) are its offsets (tap-major, width then height), 18..26 its mask values, 27..31
 * are ignored.  Runs through the LDS-staged kernels only; a shape none of them takes is refused
 * with DCNV4_ERR_UNSUPPORTED. */
int dcnv4_forward_merged(const void *x, const void *offset_mask, void *y,
                         int N, int H, int W, int G, int Cg,
                         int kernel_h, int kernel_w, int stride_h, int stride_w,
                         int pad_h, int pad_w, int dil_h, int dil_w,
                         float offset_scale, int dtype, void *stream);

/* Backward of Eq. 1 by the chain rule (the paper gives no backward):
 *   grad_mask_k  = sum_c gy[c] * S_k[c]
 *   grad_offset  = offset_scale * m_k * sum_c gy[c] * dS_k[c]/d(wx, hy)   (right-hand derivative
 *                  at whole-number coordinates)
 *   grad_x      += m_k * corner weight * gy[c]   at the in-image neighbours
 * Overwrites all three outputs; grad_x is zero-filled on `stream` first.  grad_offset/grad_mask are
 * fp32 sums, rounded once in F16.  In the LDS-staged path grad_x is summed per tile in 32-bit fixed
 * point with 22 fractional bits (every term m * weight * gy[c] rounded to a multiple of 2^-22, the
 * sum itself exact and independent of the order); terms of magnitude 64 or more, and whatever would
 * take a tile's sum for one pixel beyond 512, are added straight to memory in fp32 instead.  The
 * tile sums (a pixel is touched by the few tiles that reach it) go to memory through fp32 atomics,
 * packed fp16 atomics in F16.  With Cg 32 or 64 (fp32) the group's channels are processed in slices
 * and grad_offset/grad_mask are summed with fp32 atomics, so their last bits can differ between
 * runs, like grad_x's. */
int dcnv4_backward(const void *x, const void *offset, const void *mask, const void *grad_y,
                   void *grad_x, void *grad_offset, void *grad_mask,
                   int N, int H, int W, int G, int Cg,
                   int kernel_h, int kernel_w, int stride_h, int stride_w,
                   int pad_h, int pad_w, int dil_h, int dil_w,
                   float offset_scale, int dtype, void *stream);

/* dcnv4_backward for the merged buffer: grad_offset_mask has the layout of
 * offset_mask (gradients of the 18 offsets, of the 9 mask values, 5 zeros), all of it written whatever
 * was there.  Same restrictions as dcnv4_forward_merged. */
int dcnv4_backward_merged(const void *x, const void *offset_mask, const void *grad_y,
                          void *grad_x, void *grad_offset_mask,
                          int N, int H, int W, int G, int Cg,
                          int kernel_h, int kernel_w, int stride_h, int stride_w,
                          int pad_h, int pad_w, int dil_h, int dil_w,
                          float offset_scale, int dtype, void *stream);

/* The DCNv3 form of Eq. 1 (Sec. 3.1: there the K modulation scalars of a sampling location are
 * softmax-normalised; DCNv4 removes exactly this): `mask_logits` [N,Ho,Wo,G,9] holds logits, and
 * m = softmax over the 9 taps is formed inside the kernels, in registers, before the aggregation
 * (expf of the shifted logits in fp32).  Everything else as in dcnv4_forward.  Runs through the
 * LDS-staged kernels only (ring of rows or input rectangle); a shape they do not take is refused with
 * DCNV4_ERR_UNSUPPORTED. */
int dcnv4_forward_softmax(const void *x, const void *offset, const void *mask_logits, void *y,
                          int N, int H, int W, int G, int Cg,
                          int kernel_h, int kernel_w, int stride_h, int stride_w,
                          int pad_h, int pad_w, int dil_h, int dil_w,
                          float offset_scale, int dtype, void *stream);

/* Backward of dcnv4_forward_softmax: grad_x and grad_offset as in dcnv4_backward with the normalised
 * m; grad_mask_logits[k] = m_k * (g_k - sum_j m_j * g_j), g being the gradient w.r.t. m. */
int dcnv4_backward_softmax(const void *x, const void *offset, const void *mask_logits, const void *grad_y,
                           void *grad_x, void *grad_offset, void *grad_mask_logits,
                           int N, int H, int W, int G, int Cg,
                           int kernel_h, int kernel_w, int stride_h, int stride_w,
                           int pad_h, int pad_w, int dil_h, int dil_w,
                           float offset_scale, int dtype, void *stream);

/* A linear layer over the channel axis -- the 1x1 point-wise convolution that Sec. 3.1 puts before and
 * after the operator, and the layer of Sec. 3.2 "Micro design" that predicts offsets and modulation
 * scalars:  y[p][o] = sum_k x[p][k] * w[o][k] + b[o].
 * Device pointers, dense row-major: x [P][K], w [Nout][K], b [Nout] or NULL (no bias), y [P][Nout];
 * x, w and y 16-byte aligned.  On the matrix cores with fp32 accumulation; y is rounded once in F16.
 * Needs K * element size a multiple of 32 bytes, Nout a multiple of 32, and every tensor below 2 GiB
 * (else DCNV4_ERR_UNSUPPORTED).  Allocates nothing; enqueues on `stream`. */
int dcnv4_linear(const void *x, const void *w, const void *b, void *y,
                 long long P, int K, int Nout, int dtype, void *stream);

/* Its backward pass, from grad_y [P][Nout]:
 *     grad_x[p] = sum_o grad_y[p][o] * w[o],   grad_w[o] = sum_p grad_y[p][o] * x[p],   grad_b[o] = sum_p grad_y[p][o]
 * Each of the three may be NULL where not wanted (not all); x is read for grad_w alone, w for grad_x alone.  Sums are fp32 in a fixed order, rounded once in
 * F16.  F32: operands as three bf16 numbers, fp32's accuracy for numbers above 2^-100; finite and below 3.3e38.
 * Needs K and Nout multiples of 8, at most 2^24 rows, K and Nout at most 2^20 (else DCNV4_ERR_UNSUPPORTED): more layers than dcnv4_linear takes, which needs
 * Nout a multiple of 32 and whole 32 bytes of K (fp16 2728 -> 1024 or 936 -> 352 and fp32 384 -> 1000 have this gradient here and no forward layer).
 * `workspace`: at least dcnv4_linear_backward_workspace_bytes() bytes. */
int dcnv4_linear_backward(const void *x, const void *w, const void *grad_y, void *grad_x, void *grad_w, void *grad_b, void *workspace,
                          long long workspace_bytes, long long P, int K, int Nout, int dtype, void *stream);

/* Bytes of workspace it needs; -1 for arguments that it refuses.  Host-only helper. */
long long dcnv4_linear_backward_workspace_bytes(long long P, int K, int Nout, int dtype);

/* The gated layer of a block's feed-forward part, both projections, the activation and the product in one kernel:
 *     a = x w[0]^T + b[0],   u = x w[1]^T + b[1],   h = act(a) * u
 * act: DCNV4_SILU (a / (1 + exp(-a))) or DCNV4_GELU (a times the normal distribution function).  x [P][K], w [2][F][K], b [2][F] or NULL, h [P][F].
 * Nothing but h is stored, with one rounding.  F32 as in dcnv4_linear_backward.  Needs K and F multiples of 8, at most 2^24 rows,
 * K at most 2^20, F at most 2^19, and w below 2 GiB (F32: below 1.33) (else DCNV4_ERR_UNSUPPORTED).
 * `workspace`: at least dcnv4_gated_linear_workspace_bytes(..., backward = 0) bytes, NULL where that is 0 (F16). */
enum { DCNV4_SILU = 0, DCNV4_GELU = 1 };
int dcnv4_gated_linear(const void *x, const void *w, const void *b, void *h, void *workspace, long long workspace_bytes, long long P, int K, int F,
                       int activation, int dtype, void *stream);

/* Its backward pass, from grad_h [P][F]; a and u are made again.  With da = grad_h * u * act'(a) and du = grad_h * act(a):
 *     grad_x[p] = sum_f da[p][f] * w[0][f] + du[p][f] * w[1][f],   grad_w = (sum_p da[p][f] * x[p], sum_p du[p][f] * x[p]),   grad_b = sums over the rows
 * Each of the three may be NULL where not wanted (not all).  In F16 da and du are rounded to fp16, times one power of two that puts the largest finite
 * |grad_h| of the tensor into [2, 4), for grad_x and grad_w: they keep all of fp16's bits down to 2^-15 of that, lose them one by one below and are zero from
 * 2^-27 on (2^-26 where that lies at 2), so a row whose grad_h is that much smaller than another's gets no more of grad_x; and u * act'(a) and act(a) have to be less than 16000
 * (else infinities).  F32 has neither limit.  grad_b is made from fp32 numbers alone.  Sums are fp32 in a fixed order.
 * `workspace`: at least dcnv4_gated_linear_workspace_bytes(..., backward = 1) bytes. */
int dcnv4_gated_linear_backward(const void *x, const void *w, const void *b, const void *grad_h, void *grad_x, void *grad_w, void *grad_b, void *workspace,
                                long long workspace_bytes, long long P, int K, int F, int activation, int dtype, void *stream);

/* Bytes of workspace the two need; -1 for arguments that they refuse.  Host-only helper. */
long long dcnv4_gated_linear_workspace_bytes(long long P, int K, int F, int dtype, int backward);

/* The 3x3 depthwise convolution of the separable structure that computes offsets and scalars in the
 * module (Sec. 3.2 "Micro design"), zero padding, stride 1, channel-last:
 *     y[n,h,w,c] = b[c] + sum_{i,j in 0..2} w[i][j][c] * x[n, h+i-1, w+j-1, c]      (x = 0 outside the map)
 * Device pointers, 16-byte aligned: x, y [N,H,W,C]; w [3][3][C] (i: height tap, j: width tap); b [C] or
 * NULL.  fp32 accumulation, one rounding at the store.  Needs C * element size a multiple of 16 bytes and
 * the tensor below 2 GiB (else DCNV4_ERR_UNSUPPORTED). */
int dcnv4_depthwise3x3(const void *x, const void *w, const void *b, void *y,
                       int N, int H, int W, int C, int dtype, void *stream);

/* Forward of the DCNv4 module (Sec. 3.2 "Micro design"; the two variants of the module-level
 * benchmark of the appendix):
 *     value = x W_in^T + b_in          (w_in == w_out == NULL: the "lightweight" variant, value = x)
 *     x'    = depthwise3x3(x; w_dw, b_dw)   (w_dw == NULL: x' = x -- the paper notes the convolution can go
 *                                      where latency matters)
 *     om    = x' W_om^T + b_om         ONE layer for offsets and scalars, in the merged layout above:
 *                                      w_om [G*32][C], b_om [G*32]; row g*32 + e produces entry e of
 *                                      group g (0..17 offsets, 18..26 scalars, 27..31 ignored)
 *     y_op  = dcnv4_forward_merged(value, om)
 *     y     = y_op W_out^T + b_out     (left out in the lightweight variant: y = y_op)
 * x, y [N,H,W,C], C = G*Cg; w_in, w_out [C][C]; w_dw [3][3][C]; biases may be NULL.  The window must be
 * 3x3 and keep the map's size (stride 1, pad = dilation), C * element size a multiple of 32 bytes.
 * `workspace`: device memory of at least dcnv4_module_workspace_bytes() bytes, 16-byte aligned, owned by
 * the caller; it holds om, value, y_op and x' during the call and may be reused afterwards.  Without the
 * depthwise convolution the value projection and the merged layer run as one kernel that reads x once.
 * Tensors between the layers are stored in `dtype`.  On an error y is untouched (the workspace may
 * have been written). */
int dcnv4_module_forward(const void *x, const void *w_in, const void *b_in,
                         const void *w_dw, const void *b_dw,
                         const void *w_om, const void *b_om,
                         const void *w_out, const void *b_out,
                         void *workspace, long long workspace_bytes, void *y,
                         int N, int H, int W, int G, int Cg,
                         int kernel_h, int kernel_w, int stride_h, int stride_w,
                         int pad_h, int pad_w, int dil_h, int dil_w,
                         float offset_scale, int dtype, void *stream);

/* Bytes of workspace dcnv4_module_forward needs (lightweight != 0: without the two projections;
 * depthwise != 0: with the depthwise convolution); -1 for a bad argument.  Host-only helper. */
long long dcnv4_module_workspace_bytes(int N, int H, int W, int G, int Cg, int dtype, int lightweight,
                                       int depthwise);

/* dcnv4_module_forward for callers that cannot allocate device memory or hand over a workspace -- code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc: the same kernels, with
 * the workspace in a buffer built into the library (a static device array of
 * dcnv4_module_static_workspace_limit() = 32 MiB bytes; every GPU the library runs on holds its own copy
 * until the process ends).  No allocation of any kind happens in the call.  A call that needs more than the
 * limit (dcnv4_module_workspace_bytes() tells) returns DCNV4_ERR_TOO_LARGE and does nothing; at 32 MiB
 * that is e.g. one 200x320x128 fp16 map, or 16 maps of 56x56x128, with both projections.
 * All calls on one GPU share that GPU's buffer: calls that overlap in time on one GPU (different streams,
 * different host threads) race on it; on one stream they are ordered and safe.  Nothing in the buffer
 * has to start at zero (every tensor in it is written in full before it is read).  The first call on a
 * device looks the buffer's address up (hipGetSymbolAddress): make one call before capturing a graph. */
int dcnv4_module_forward_static(const void *x, const void *w_in, const void *b_in,
                                const void *w_dw, const void *b_dw,
                                const void *w_om, const void *b_om,
                                const void *w_out, const void *b_out, void *y,
                                int N, int H, int W, int G, int Cg,
                                int kernel_h, int kernel_w, int stride_h, int stride_w,
                                int pad_h, int pad_w, int dil_h, int dil_w,
                                float offset_scale, int dtype, void *stream);

/* Size in bytes of the built-in workspace of dcnv4_module_forward_static.  Host-only helper. */
long long dcnv4_module_static_workspace_limit(void);

/* Operators of a training step around the module, on rows: x [P][C], C channels (or features) of P pixels.  As everywhere:
 * DEVICE pointers, dense, 16-byte aligned, tensors of element type `dtype`, arithmetic and statistics in fp32, one rounding
 * to nearest at each store (what else the cross entropy rounds is said there), outputs must not alias inputs, nothing is allocated,
 * nothing is kept between calls.  A workspace is the caller's and needs no initial values; two calls, or two captured graphs, that may run at
 * the same time need one each. */

/* Layer norm over the channels of each row (biased variance, as normalisation layers have it):
 *     y = (x - mean) * rstd * gamma + beta,   rstd = 1 / sqrt(var + eps)
 * gamma, beta [C] or NULL (ones, zeros).  mean, rstd: fp32 [P] for the backward pass, or NULL.  Any C from 1 to 16384 (else
 * DCNV4_ERR_UNSUPPORTED), any P; eps >= 0. */
int dcnv4_layer_norm(const void *x, const void *gamma, const void *beta, void *y, float *mean, float *rstd,
                     long long P, int C, float eps, int dtype, void *stream);

/* Its backward pass, from the forward's mean and rstd.  With xhat = (x - mean) * rstd and g = grad_y * gamma:
 *     grad_x     = rstd * (g - avg(g) - xhat * avg(g * xhat))
 *     grad_gamma = sum over the rows of grad_y * xhat,   grad_beta = sum of grad_y      (fp32 sums in a fixed order)
 * grad_gamma, grad_beta [C]: either or both NULL where not wanted (both: no workspace is needed).  `workspace`: at least
 * dcnv4_layer_norm_workspace_bytes(P, C) bytes. */
int dcnv4_layer_norm_backward(const void *x, const void *gamma, const float *mean, const float *rstd, const void *grad_y,
                              void *grad_x, void *grad_gamma, void *grad_beta, void *workspace, long long workspace_bytes,
                              long long P, int C, int dtype, void *stream);

/* Bytes of workspace the backward passes of the two norms need; -1 for a bad argument.  Host-only helper. */
long long dcnv4_layer_norm_workspace_bytes(long long P, int C);

/* Dropout of n elements, its mask never stored:  y[i] = residual[i] + (dropped(i) ? 0 : x[i] / (1 - p'))
 * residual: [n] or NULL (zeros).  0 <= p <= 1; p' is p to the nearest multiple of 2^-16.  Element i is dropped where its 16
 * random bits are below p' * 65536: number i % 8 (low half of a word first) of the four words that Philox 4x32 with ten
 * rounds makes of the key `seed` and the counter (i / 8, offset), low words first.  So the same (seed, offset) drops the same
 * elements, in the backward pass as in the forward one, whatever the type, and every call of a training run takes an offset of
 * its own.  offset_on_device: NULL, or the device address (8-byte aligned) of one 64-bit number that is added to
 * `offset` as the kernel runs: for captured graphs, whose arguments stay what they were.  A dropped element gives zero whatever x holds. */
int dcnv4_dropout(const void *x, const void *residual, void *y, long long n, float p, unsigned long long seed,
                  unsigned long long offset, const void *offset_on_device, int dtype, void *stream);

/* grad_x of dcnv4_dropout with the same p, seed and offset (that of the residual is grad_y itself). */
int dcnv4_dropout_backward(const void *grad_y, void *grad_x, long long n, float p, unsigned long long seed,
                           unsigned long long offset, const void *offset_on_device, int dtype, void *stream);

/* The end of a residual branch and the norm in front of the next one, in one pass:
 *     z = residual + dropout(x)  (element i = row * C + channel),   y = layer norm of z as stored
 * x, residual, z, y [P][C]; the rest as in dcnv4_layer_norm and dcnv4_dropout. */
int dcnv4_dropout_add_layer_norm(const void *x, const void *residual, const void *gamma, const void *beta, void *z, void *y,
                                 float *mean, float *rstd, long long P, int C, float p, unsigned long long seed,
                                 unsigned long long offset, const void *offset_on_device, float eps, int dtype, void *stream);

/* Its backward pass.  grad_y: the gradient of y; grad_z: that of z from what else reads it, or NULL.
 *     grad_residual = grad_z + the norm's grad_x at z,   grad_x = dropout's gradient of that sum (before its rounding) */
int dcnv4_dropout_add_layer_norm_backward(const void *z, const void *gamma, const float *mean, const float *rstd,
                                          const void *grad_y, const void *grad_z, void *grad_x, void *grad_residual,
                                          void *grad_gamma, void *grad_beta, void *workspace, long long workspace_bytes,
                                          long long P, int C, float p, unsigned long long seed, unsigned long long offset,
                                          const void *offset_on_device, int dtype, void *stream);

/* The end of a residual block with its norms, in one pass:
 *     b = first norm of x (DCNV4_FIRST_NORM; else b = x),   z = residual + gate * scale * b,   y = second norm of z as stored (DCNV4_SECOND_NORM)
 * The norms as in dcnv4_layer_norm with gamma1, beta1 and gamma2, beta2 [C], each NULL for ones or zeros, and one eps.  `norms`: which there are, or 0.
 * scale [C] (of `dtype`) or NULL (ones).  gate: fp32, one for each of `gates` images of P / gates rows, or NULL with gates = 0 (ones); a gate of 0 leaves
 * z = residual, whatever x holds.  x, residual, z, y [P][C]; y NULL without a second norm.  mean1, rstd1, mean2, rstd2: fp32 [P] for the
 * backward pass, or NULL.  C from 1 to 8192; with gates, P below 2^31 and a multiple of gates, gates up to 2^20. */
enum { DCNV4_FIRST_NORM = 1, DCNV4_SECOND_NORM = 2 };
int dcnv4_norm_scale_add_norm(const void *x, const void *residual, const void *gamma1, const void *beta1, const void *scale, const float *gate,
                              const void *gamma2, const void *beta2, void *z, void *y, float *mean1, float *rstd1, float *mean2, float *rstd2,
                              long long P, int C, int gates, int norms, float eps, int dtype, void *stream);

/* Its backward pass.  grad_y: the gradient of y; grad_z: that of z from what else reads it (NULL for none, with a second norm).  With gz the sum of grad_z
 * and the second norm's grad_x at z (before its rounding), and h = gz * gate * scale:
 *     grad_residual = gz (without a second norm that is grad_z itself, and nothing is written: NULL)
 *     grad_x = the first norm's gradient for h (or h),    grad_scale [C] = sum over the rows of gz * gate * b,
 *     grad_gate [gates] = sum over the image's rows and channels of gz * scale * b (fp32),   grad_gamma1, ... [C] as in dcnv4_layer_norm_backward
 * Any of grad_scale, grad_gate and the norms' four may be NULL where not wanted (all: no workspace is needed).  Rows with a gate of 0 have
 * grad_x 0 and count for nothing, whatever x holds, but in grad_gate.  Sums are fp32 in a fixed order.  z is read with a second norm only.
 * `workspace`: at least dcnv4_norm_scale_add_norm_workspace_bytes(P, C, gates) bytes. */
int dcnv4_norm_scale_add_norm_backward(const void *x, const void *z, const void *gamma1, const void *beta1, const void *scale, const float *gate,
                                       const void *gamma2, const float *mean1, const float *rstd1, const float *mean2, const float *rstd2,
                                       const void *grad_y, const void *grad_z, void *grad_x, void *grad_residual, void *grad_scale, float *grad_gate,
                                       void *grad_gamma1, void *grad_beta1, void *grad_gamma2, void *grad_beta2, void *workspace,
                                       long long workspace_bytes, long long P, int C, int gates, int norms, int dtype, void *stream);

/* Bytes of workspace it needs; -1 for a bad argument.  Host-only helper. */
long long dcnv4_norm_scale_add_norm_workspace_bytes(long long P, int C, int gates);

/* Softmax cross entropy out of the last linear layer (a classifier's, or each pixel's), without its logits being stored:
 *     logit[p][v] = sum_k x[p][k] * w[v][k] + b[v],   lse[p] = log sum_v exp(logit[p][v]),   loss[p] = lse[p] - logit[p][target[p]]
 * x [P][K], w [V][K], b [V] or NULL; target: 64-bit class numbers [P]; loss, lse: fp32 [P].  A row whose target is ignore_index
 * has loss 0; one whose target is neither that nor a class has loss NaN.  Logits and sums are fp32 (F32: products of operands
 * held as three bf16 numbers, fp32's accuracy for numbers above 2^-100; x and w must be finite and below 3.3e38; F16 follows fp16's infinities).  b may
 * hold -infinity: that class has probability 0.
 * Needs K * element size a multiple of 32 bytes, and at most 2^20 rows, 2^20 features and 2^22 classes (else DCNV4_ERR_UNSUPPORTED).
 * `workspace`: at least dcnv4_linear_cross_entropy_workspace_bytes(..., backward = 0) bytes. */
int dcnv4_linear_cross_entropy(const void *x, const void *w, const void *b, const long long *target, float *loss, float *lse,
                               void *workspace, long long workspace_bytes, long long P, int K, int V,
                               long long ignore_index, int dtype, void *stream);

/* Its backward pass, from the forward's lse and grad_loss fp32 [P].  With d = exp(logit - lse) - (v == target), a piece of the classes
 * at a time:
 *     grad_x[p] = grad_loss[p] * sum_v d[p][v] * w[v],   grad_w[v] = sum_p grad_loss[p] * d[p][v] * x[p],   grad_b[v] = sum_p grad_loss[p] * d[p][v]
 * In F16 d is rounded to fp16 (of 2^15 * d) for grad_x and grad_w; grad_w's other operand, x * grad_loss / the largest |grad_loss|, is x itself
 * where grad_loss is the same in all rows and is rounded to fp16 otherwise, to 2^-11 of it and 2^-17 of x = 1 for rows of down to 2^-32 of the
 * largest (each power of two below doubles the latter).  Sums are fp32, grad_b is made from fp32 numbers alone.
 * A row that is ignored, or whose grad_loss is 0, counts for nothing and has grad_x 0, whatever x holds there (w being finite); one with
 * loss NaN has grad_x NaN and makes grad_w NaN.  grad_b may be NULL.  Sums are made in a fixed order.
 * `workspace`: at least dcnv4_linear_cross_entropy_workspace_bytes(..., backward = 1) bytes. */
int dcnv4_linear_cross_entropy_backward(const void *x, const void *w, const void *b, const long long *target,
                                        const float *lse, const float *grad_loss, void *grad_x, void *grad_w, void *grad_b,
                                        void *workspace, long long workspace_bytes, long long P, int K, int V,
                                        long long ignore_index, int dtype, void *stream);

/* Bytes of workspace the two need; -1 for arguments that they refuse.  Host-only helper. */
long long dcnv4_linear_cross_entropy_workspace_bytes(long long P, int K, int V, int dtype, int backward);

/* One tensor of dcnv4_adamw: device pointers to n elements each, in HOST memory itself. */
typedef struct {
    long long n;
    float *param;             /* fp32, updated */
    const void *grad;         /* of the call's dtype */
    void *m, *v;              /* states, updated: fp32; or 8 bits (e4m3) of m and of sqrt(v) */
    float *scales;            /* states of 8 bits: [(n + 255) / 256][2], of m and of sqrt(v), 8-byte aligned; else ignored */
    void *copy;               /* F16: param rounded to fp16 after the step (what the forward pass reads), or NULL */
    double lr, weight_decay;
} dcnv4_adamw_tensor;

/* A step of AdamW (decoupled weight decay) over `count` tensors, t = step + the number at step_on_device:
 *     g = grad * f0,   m = beta1 * m + (1 - beta1) * g,   v = beta2 * v + (1 - beta2) * g^2
 *     param = param * (1 - lr * f1 * weight_decay) - lr * f1 / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 * tensors: host memory, read during the call only.  Each n from 1 to 2^34; no two buffers may share memory.  `dtype`: that of the gradients (and copies).
 * step_on_device: NULL, or the device address of one 64-bit number (8-byte aligned; t is 1 where the sum is less).  factors_on_device:
 * NULL (f0 = f1 = 1), or the device address of two fp32 numbers f0, f1 (8-byte aligned): a loss scale's inverse times what clips gradients, and a schedule's
 * factor.  Where f0 is infinite or NaN the step changes nothing (a loss scale that was too large).  Both are for captured graphs, whose
 * arguments stay what they were.  state_bits: 32, or 8: m and r = sqrt(v) are stored as e4m3 (fp8, largest number 448, zeros to start with), times a scale
 * of its own for each 256 elements of the tensor: their largest magnitude / 448 (zeros for blocks of m below 2^-100, and for blocks of r below 2^-75, as v in fp32 is
 * zero below 2^-150).  m * 448 / that magnitude is rounded to nearest; r so scaled to one of its two neighbours, up with the probability that keeps its mean
 * (random bits of dcnv4_dropout's generator with key `seed` and counter (i / 8 + number of the tensor * 2^40, t), 16 for element i as there), and in
 * other blocks never from above zero to zero.  With 8 bits g must be finite where f0
 * is, and less than 2^63: a block of elements shares what is not.
 * 0 <= beta < 1, eps > 0 (a normal fp32 number), step >= 1 (0 with step_on_device). */
int dcnv4_adamw(const dcnv4_adamw_tensor *tensors, int count, double beta1, double beta2, double eps, long long step,
                const void *step_on_device, const void *factors_on_device, unsigned long long seed, int state_bits, int dtype, void *stream);

/* Bytes the ideal memory-access model of Sec. 3.2 ("2HWC + 27HWG", every value touched
 * once) assigns to one forward call: x + offset + mask + y.  Host-only helper. */
long long dcnv4_forward_algorithmic_bytes(int N, int H, int W, int G, int Cg,
                                          int H_out, int W_out, int dtype);

/* Same model for one backward call: reads x, offset, mask, grad_y; writes grad_x,
 * grad_offset, grad_mask (the zero-fill of grad_x is not counted). */
long long dcnv4_backward_algorithmic_bytes(int N, int H, int W, int G, int Cg,
                                           int H_out, int W_out, int dtype);

/* The two models with the merged buffer: 32 instead of 27 values per (pixel, group). */
long long dcnv4_forward_merged_algorithmic_bytes(int N, int H, int W, int G, int Cg,
                                                 int H_out, int W_out, int dtype);
long long dcnv4_backward_merged_algorithmic_bytes(int N, int H, int W, int G, int Cg,
                                                  int H_out, int W_out, int dtype);

/* TEST AND BENCHMARK SWITCHES, not an application interface: they force a kernel or a tile shape so
 * that every path can be checked on every shape (process-wide, not thread-safe).  An application
 * never calls this; the library's own choice is the value 0 of every switch.
 *   "reset"       (any value) puts every switch back to 0
 *   "fwd_path"    1 = direct global gather, 2 = input rectangle staged in LDS, 3 = ring of input rows
 *                 in LDS (fp16, Cg 16); 0 = the first of these that takes the call: ring (fp16, Cg 16, maps of
 *                 512 pixels or more up to 80 wide, where the (image, group) pairs fill the chip), strips
 *                 (below), rectangle where a useful tile fits, ring on any map that it fits, direct
 *   "fwd_strip"   out of a rolling window of input rows, in strips of columns: the forward (with fwd_path 0) of
 *                 every type and group width, and the backward's grad_offset/grad_mask pass (with bwd_path 0) of
 *                 whole groups of up to 64 bytes.  0 = where the library's own estimate is that they are the
 *                 faster, 1 = wherever they apply (in the backward also where the direct kernel would be taken,
 *                 so that grad_x goes through its fixed-point sums), 2 = never.  Where strips take a call,
 *                 "fwd_threads", "fwd_single" and "wg_per_cu" have no effect on it
 *   "bwd_path"    1 = one kernel with global atomics for grad_x (fp32), 2 = two LDS-staged kernels
 *                 (gathers out of rectangles for grad_offset/grad_mask; fixed-point accumulation of grad_x in
 *                 LDS), 0 = staged, by strips or rectangles, where a useful rectangle fits, else the first
 *   "fwd_single"  LDS rectangle buffers of the staged gather kernels: 1 = always two (the next tile
 *                 streams in during the current one), 2 = always one (bigger rectangle, refilled
 *                 between tiles), 0 = whichever the tile chooser estimates to be cheaper
 *   "wg_per_cu"   persistent workgroups per compute unit of the rectangle kernels (1..32, as far as
 *                 LDS allows)
 *   "module_rows" 1 = dcnv4_module_forward keeps the tensors between its layers channel-last (default: the
 *                 full module keeps them plane-major, one (image, group) after the other)
 *   "linear_tile" tile of the linear layers, output channels x pixels: 1 = 128x128, 2 = 64x64, 3 = 256x256,
 *                 4 = 128x256 (fp32), 5 = the kernel that reads x once (fp16, K of up to 256 bytes); 0 = the one
 *                 with the lowest estimated time.  In place of a tile that a type or K does not have: 128x128
 *   "loss_tile"   tile of the cross entropy's products, classes x pixels: 1 = 64x64, 2 = 128x128, 3 = 256x256 (fp32: 256x128)
 *   "loss_splits" workgroups that share a sum of its gradients (1..64)
 *   "loss_piece"  classes of a piece (rounded up to a multiple of 256); these three change the size of its workspace
 *   "layer_tile"  tile of the gated layer's and the layers' gradients' products, as "loss_tile"; 4 = 256x128 by half the waves (the gated
 *                 layer in fp16; elsewhere no preference)
 *   "layer_splits" workgroups that share a sum of those gradients (1, 2, 3, 8 or 64); both change the size of their workspaces
 *   "gom_coop"    1 = the fp32 grad_offset/grad_mask pass moves its values through per-wave LDS slices
 *                 even for whole groups (default: each lane reads and writes its own pixel's values)
 *   "gx_threads"  workgroup size of the staged grad_x kernel (256, 512 or 768)
 *   "gx_own"      grad_x kernel: 1 = all tiles of an (image, channel run) go to one workgroup, which stores
 *                 its sums, 2 = tiles one by one, whose sums are added atomically (default: the faster by estimate)
 *   "halo"        displacement in pixels (rows, for the ring) that the staged window allows for;
 *                 samples beyond it are still exact, they take the path through global memory
 *   "lds_kb"      LDS budget per workgroup of the staged kernels (8..160)
 *   "fwd_threads" workgroup size of the staged forward (64, 128, 256, 512, 640 or 768 for the
 *                 rectangle kernel; 256 = four waves instead of eight for the ring)
 *   "fwd_cpt"     channels per thread in the direct forward kernel (8 or 16)
 *   "bwd_cpt"     channels per thread in the direct backward kernel (1, 2, 4, 8 or 16)
 *   "xcd_remap"   1 = hand consecutive tiles to one XCD (default), 0 = plain block order
 * Returns DCNV4_ERR_UNSUPPORTED for an unknown key or value. */
int dcnv4_set_option(const char *key, int value);

/* Name of the kernel that the most recent dcnv4_forward (backward = 0) or dcnv4_backward
 * (backward = 1) call launched, as it appears in a profiler's kernel trace; two kernels with " + " between
 * them, and "(owned)" before a grad_x kernel whose workgroups have whole planes to themselves, "(owned,
 * uncleared)" where no other kernel has cleared grad_x for it.  Static storage;
 * NULL before the first such call. */
const char *dcnv4_last_kernel_name(int backward);

const char *dcnv4_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* DCNV4_H */
