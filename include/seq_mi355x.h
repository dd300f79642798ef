/*
 * seq_mi355x.h -- C ABI of the sequence operators of the MI355X (gfx950) library: what a
 * language model of short convolutions and state spaces runs between its projections.
 *
 *   seq_conv   short causal convolution of every channel of a sequence, with SiLU
 *   seq_scan   selective state space scan
 *   seq_rec    gated linear recurrence of every channel
 *   seq_norm   root-mean-square norm with the residual's addition
 *   seq_lnorm  layer norm with the residual's addition
 *   seq_mv4    products of a few rows with weights of 4 bits and scales for groups of channels
 *   seq_adamw  AdamW step over many tensors, its states in 32 bits or in 8
 *
 * A sequence is the blocked activation tensor of conv_mi355x.h with H = 1 and W = L, and its
 * projections are that library's 1x1 convolutions (all three passes); these operators read and
 * write the same tensors in place.  The conventions are those of conv_mi355x.h: device
 * pointers, 16-byte aligned (index arrays 4-byte), owned by the caller; calls only enqueue on
 * `stream`; outputs are overwritten; a handle owns a host-side plan only and may be used from
 * one host thread at a time; every function returns a conv_status_t; no allocation, no
 * fallback.  Everything a pass has to know beyond its pointers (sizes, types, strides) is in the
 * descriptor that its handle was created from.
 *
 * Sequence tensors: X[N][Cb][L][v], v = 16 bytes / element size channels side by side, channel
 * c in block c / v at slot c % v; slots beyond C hold zeros on input and are written as zero.
 * A seq_view_t gives the distances between sequences, blocks and positions, so that a tensor may
 * be a slice of blocks of a larger one, or have a position's channels side by side
 * ([N][L][Cb][v]).  A view of three zeros is the dense X[N][Cb][L][v].
 * "fp32 vector": Cp entries, Cp = C rounded up to v, entries beyond C zero.
 *
 * Lengths.  `lengths` (int32, N entries, device, or NULL) says how many positions of each
 * sequence there are, 0 ... L (values outside are clamped).  What lies beyond is never used,
 * whatever it holds, and outputs are written as zero there, gradients too.
 *
 * States.  What a sequence carries from one call to the next lies in one of `slots` slots of a
 * state tensor: that of sequence n in slot slots[n] (int32, N entries, device), or n where the
 * array is NULL.  Slots of one call have to differ.  A sequence whose slot is outside
 * [0, slots) has none: it starts from zeros and stores nothing (seq_*_step: writes zeros).
 *
 * Sums, states, parameters and their gradients are fp32; what is stored in bf16 is rounded to
 * it once, to nearest even.  Every sum has a fixed order: results are the same on every run.
 */
#ifndef SEQ_MI355X_H
#define SEQ_MI355X_H

#include "conv_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SEQ_F32 = CONV_F32,
    SEQ_BF16 = CONV_BF16,
    SEQ_I8 = 2 /* activations of seq_mv4 only: 8 bits and a scale a row */
} seq_dtype_t;

/* Distances in elements between sequences, channel blocks and positions: multiples of v, not
 * negative, 2^40 at most and 2^58 over all of a dimension; those of an output may not let two
 * elements share a place. */
typedef struct {
    int64_t n, c, l;
} seq_view_t;

typedef struct {
    int32_t vlen, Cb, Cp;   /* v, channel blocks, C rounded up to v (seq_mv4: of x)         */
    int32_t reserved;
    size_t workspace_bytes; /* max over the passes; may be 0                                */
    size_t state_bytes;     /* one slot of the state (seq_conv, seq_scan, seq_rec); m, and v, of seq_adamw */
    size_t wt_bytes;        /* packed weights (seq_mv4)                                     */
    size_t scale_bytes;     /* their scales (seq_mv4); those of both states of seq_adamw    */
} seq_info_t;

typedef struct seq_plan *seq_handle_t;

/* Free the host-side plan.  CONV_EINVAL for NULL. */
conv_status_t seq_destroy(seq_handle_t h);
/* Sizes of a plan.  CONV_EINVAL for a NULL argument. */
conv_status_t seq_query(seq_handle_t h, seq_info_t *info);
/* What each pass launches, in readable form (at most buflen bytes, NUL-terminated). */
conv_status_t seq_describe(seq_handle_t h, char *buf, size_t buflen);

/* ------------------------------------------------------------------ short convolution
 *   s[n,c,l] = bias[c] + sum_{j < W} w[j][c] * x[n,c,l - W + 1 + j],   y = silu ? s * sigmoid(s) : s
 * with x at negative positions from the state (the last W - 1 inputs, oldest first), zero where
 * there is none.  w: fp32 [W][Cp]; bias: fp32 vector or NULL; state: [slots][Cb][W-1][v] of the
 * tensors' type.
 * Errors of create: CONV_EINVAL for a NULL pointer, an extent < 1, slots < 0, an unknown type, a
 * view that is not as stated; CONV_EUNSUPPORTED beyond N, C <= 2^20, L <= 2^30, 2^31 positions
 * and 2^39 elements a tensor, problems of more than 2^32 work-items, and for W outside 2 ... 8. */
typedef struct {
    int32_t N, C, L, W;
    int32_t silu, slots, dtype;
    int32_t reserved;
    seq_view_t x, y, dy, dx;
} seq_conv_desc_t;
conv_status_t seq_conv_create(const seq_conv_desc_t *desc, seq_handle_t *out);
/* state_in, state_out: NULL or a state tensor (CONV_EINVAL for a plan without slots); the two
 * may be the same. */
conv_status_t seq_conv_fwd(seq_handle_t h, const void *x, const float *w, const float *bias,
                           const void *state_in, void *y, void *state_out, const int32_t *slots,
                           const int32_t *lengths, void *stream);
/* One new position of each sequence, the state moved on in place: a plan of L = 1 with slots. */
conv_status_t seq_conv_step(seq_handle_t h, const void *x, const float *w, const float *bias,
                            void *state, void *y, const int32_t *slots, void *stream);
/* Gradients of seq_conv_fwd without states: dx, dw (fp32 [W][Cp]), dbias (fp32 vector or NULL).
 * ws: workspace_bytes of scratch; CONV_EWORKSPACE if ws_bytes is less. */
conv_status_t seq_conv_bwd(seq_handle_t h, const void *x, const float *w, const float *bias,
                           const void *dy, void *dx, float *dw, float *dbias,
                           const int32_t *lengths, void *ws, size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------ selective scan
 * For every channel c, in group g = c / (C/G), and state s < S:
 *   d        = softplus ? log(1 + exp(dt + dt_bias)) : dt + dt_bias
 *   h[s][l]  = exp(d * A[s][c]) * h[s][l-1] + d * B[g*S+s][l] * x[l]
 *   y[l]     = sum_s C[g*S+s][l] * h[s][l] + D[c] * x[l],   times z * sigmoid(z) where there is a z
 * A: fp32 [S][Cp]; D, dt_bias: fp32 vectors or NULL (zero); B and C: sequence tensors of G*S
 * channels; z: sequence tensor or NULL; state: fp32 [slots][S][Cp].
 * Errors of create: as seq_conv_create; CONV_EINVAL where G does not divide C, CONV_EUNSUPPORTED
 * where G > 1 and C/G is no multiple of v, for S > 64 or G*S > 2^16, and for blocks or positions of
 * a view more than 2^24 elements apart. */
typedef struct {
    int32_t N, C, L, S, G;
    int32_t softplus, slots, dtype;
    seq_view_t x, dt, B, C_, z, y;
    seq_view_t dy, dx, ddt, dB, dC, dz;
} seq_scan_desc_t;
conv_status_t seq_scan_create(const seq_scan_desc_t *desc, seq_handle_t *out);
/* ws: workspace_bytes of scratch; CONV_EWORKSPACE if ws_bytes is less than the pass needs. */
conv_status_t seq_scan_fwd(seq_handle_t h, const void *x, const void *dt, const float *A,
                           const void *B, const void *C, const float *D, const void *z,
                           const float *dt_bias, const float *state_in, void *y, float *state_out,
                           const int32_t *slots, const int32_t *lengths, void *ws, size_t ws_bytes,
                           void *stream);
/* One new position of each sequence, the state moved on in place: a plan of L = 1 with slots. */
conv_status_t seq_scan_step(seq_handle_t h, const void *x, const void *dt, const float *A,
                            const void *B, const void *C, const float *D, const void *z,
                            const float *dt_bias, float *state, void *y, const int32_t *slots,
                            void *stream);
/* Gradients of seq_scan_fwd without states.  dx, ddt, dB, dC: sequence tensors; dz: one where
 * there is a z; dA: fp32 [S][Cp]; dD, ddt_bias: fp32 vectors or NULL.  The decays exp(d A) of up to
 * 64 positions are multiplied together: where d A > 0 their product has to stay below 2^128.
 * The scratch holds the states in fp32 at every eighth position: for sequences of 64 positions and
 * more some 11 bytes an element of x at 16 states, 53 at 64 (seq_query has the size). */
conv_status_t seq_scan_bwd(seq_handle_t h, const void *x, const void *dt, const float *A,
                           const void *B, const void *C, const float *D, const void *z,
                           const float *dt_bias, const void *dy, void *dx, void *ddt, float *dA,
                           void *dB, void *dC, float *dD, void *dz, float *ddt_bias,
                           const int32_t *lengths, void *ws, size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------ gated linear recurrence
 * For every channel c:
 *   s    = sigmoid(f + f_bias),  g = sigmoid(i + i_bias),  a = exp(A[c] * s)
 *   h[l] = a * h[l-1] + sqrt(1 - a^2) * g * x[l]
 *   y[l] = h[l],   times z * sigmoid(z) where there is a z
 * A: fp32 vector; numbers above zero count as zero, and so does 1 - a^2 below 2^-126.
 * f_bias, i_bias: fp32 vectors or NULL (zero);
 * z: sequence tensor or NULL; state: fp32 [slots][Cp].
 * Errors of create: as seq_conv_create; CONV_EUNSUPPORTED for positions of a view more than 2^20
 * elements apart and, where x has its blocks nearer to each other than its positions, for blocks
 * of a view more than 2^24. */
typedef struct {
    int32_t N, C, L;
    int32_t slots, dtype;
    int32_t reserved;
    seq_view_t x, f, i, z, y;
    seq_view_t dy, dx, df, di, dz;
} seq_rec_desc_t;
conv_status_t seq_rec_create(const seq_rec_desc_t *desc, seq_handle_t *out);
/* ws: workspace_bytes of scratch; CONV_EWORKSPACE if ws_bytes is less than the pass needs. */
conv_status_t seq_rec_fwd(seq_handle_t h, const void *x, const void *f, const void *i,
                          const float *A, const void *z, const float *f_bias, const float *i_bias,
                          const float *state_in, void *y, float *state_out, const int32_t *slots,
                          const int32_t *lengths, void *ws, size_t ws_bytes, void *stream);
/* One new position of each sequence, the state moved on in place: a plan of L = 1 with slots. */
conv_status_t seq_rec_step(seq_handle_t h, const void *x, const void *f, const void *i,
                           const float *A, const void *z, const float *f_bias, const float *i_bias,
                           float *state, void *y, const int32_t *slots, void *stream);
/* Gradients of seq_rec_fwd without states.  dx, df, di: sequence tensors; dz: one where there is a
 * z; dA, df_bias, di_bias: fp32 vectors, the last two or NULL.  Where 1 - a^2 is zero, the square
 * root's slope is left out of dA and df; dA of an A above zero is zero. */
conv_status_t seq_rec_bwd(seq_handle_t h, const void *x, const void *f, const void *i,
                          const float *A, const void *z, const float *f_bias, const float *i_bias,
                          const void *dy, void *dx, void *df, void *di, float *dA, void *dz,
                          float *df_bias, float *di_bias, const int32_t *lengths, void *ws,
                          size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------ norm
 *   r = x + res (rounded to the tensors' type; without a residual r = x),
 *   y[c] = r[c] * w[c] / sqrt(mean_c r^2 + eps)          of every position on its own
 * w: fp32 vector; res: sequence tensor or NULL; r: sequence tensor, may be x or res itself (their
 * view then has to be the same), or NULL if it is not needed.
 * Errors of create: as seq_conv_create; CONV_EINVAL for an eps that is negative or no number. */
typedef struct {
    int32_t N, C, L;
    int32_t dtype;
    float eps;
    int32_t reserved;
    seq_view_t x, res, r, y, q, dy, dr, dx;
} seq_norm_desc_t;
conv_status_t seq_norm_create(const seq_norm_desc_t *desc, seq_handle_t *out);
conv_status_t seq_norm_fwd(seq_handle_t h, const void *x, const void *res, const float *w, void *r,
                           void *y, void *stream);
/* The same with y in 8 bits: q = y / scale (by its reciprocal) rounded to nearest even, scale[n][l] = max_c |y| / 127
 * (fp32, [N][L]); a position of zeros has scale and q zero.  q: int8, a sequence tensor of
 * v = 16 whatever the others are (its view is in bytes). */
conv_status_t seq_norm_fwd_q8(seq_handle_t h, const void *x, const void *res, const float *w,
                              void *r, int8_t *q, float *scale, void *stream);
/* Gradients: r is what seq_norm_fwd stored (x without a residual); dr the gradient that reaches r
 * from elsewhere, or NULL; dx the gradient of x and of res; dw: fp32 vector. */
conv_status_t seq_norm_bwd(seq_handle_t h, const void *r, const float *w, const void *dy,
                           const void *dr, void *dx, float *dw, void *ws, size_t ws_bytes,
                           void *stream);

/* ------------------------------------------------------------------ layer norm
 *   r = x + res (rounded to the tensors' type; without a residual r = x),
 *   y[c] = (r[c] - mean r) * w[c] / sqrt(mean_c (r - mean r)^2 + eps) + b[c]    of every position on its own
 * w: fp32 vector; b: fp32 vector or NULL (zero); res, r and the errors of create: as seq_norm. */
typedef seq_norm_desc_t seq_lnorm_desc_t;
conv_status_t seq_lnorm_create(const seq_lnorm_desc_t *desc, seq_handle_t *out);
conv_status_t seq_lnorm_fwd(seq_handle_t h, const void *x, const void *res, const float *w,
                            const float *b, void *r, void *y, const int32_t *lengths, void *stream);
/* The same with y in 8 bits, as seq_norm_fwd_q8. */
conv_status_t seq_lnorm_fwd_q8(seq_handle_t h, const void *x, const void *res, const float *w,
                               const float *b, void *r, int8_t *q, float *scale,
                               const int32_t *lengths, void *stream);
/* Gradients: r, dr and dx as seq_norm_bwd; dw: fp32 vector; db: one, or NULL. */
conv_status_t seq_lnorm_bwd(seq_handle_t h, const void *r, const float *w, const void *dy,
                            const void *dr, void *dx, float *dw, float *db, const int32_t *lengths,
                            void *ws, size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------ products with 4-bit weights
 *   y[m,k] = xscale[m] * sum_c x[m,c] * q[k,c] * scale[c / group][k] + bias[k],   q = -8 ... 7
 * x: [M][Cx], Cx = C rounded up to v (SEQ_I8: 16, as seq_norm_fwd_q8 leaves one position of M
 * sequences), entries beyond C zero; xscale: fp32, M entries, SEQ_I8 only; y: [M][Ky], fp32 for
 * SEQ_F32, else bf16, Ky = K rounded up to its v, entries beyond K written as zero;
 * bias: fp32, K entries, or NULL; scale: fp32 [ceil(C/group)][Kp], Kp = K rounded up to 16.
 * Packed weights [Cw/128][Kp][4][4][8 x 4 bits], Cw = C rounded up to 128: word i of the 16
 * bytes j of row k holds channels 128 b + 32 i + 8 j ... + 7, the first in the lowest bits, in
 * two's complement; rows and channels beyond K and C hold zeros.
 * Errors of create: CONV_EINVAL for extents < 1, an unknown type, a group that is not 32, 64 or
 * 128; CONV_EUNSUPPORTED beyond M <= 65536, C, K <= 2^24, K*C <= 2^39, K*M <= 2^31.
 * fp32 activations are taken as three bf16 numbers each: their products are exact to fp32 down to
 * 2^-109, and numbers from 3.39e38 on count as infinite. */
typedef struct {
    int32_t M, C, K, group;
    int32_t dtype; /* of x */
    int32_t reserved;
} seq_mv4_desc_t;
conv_status_t seq_mv4_create(const seq_mv4_desc_t *desc, seq_handle_t *out);
conv_status_t seq_mv4(seq_handle_t h, const void *x, const float *xscale, const void *wt,
                      const float *scale, const float *bias, void *y, void *stream);
/* Weights laid out once: q = w / scale rounded to nearest even and clamped, scale = max |w| of the
 * group / 7 (0 for a group of zeros; NaN, and q zero, for one that holds a NaN or an infinity).
 * w: fp32 [K][C], logical. */
conv_status_t seq_mv4_quant(seq_handle_t h, const float *w, void *wt, float *scale, void *stream);
/* And back: w[k][c] = q * scale. */
conv_status_t seq_mv4_unquant(seq_handle_t h, const void *wt, const float *scale, float *w,
                              void *stream);

/* ------------------------------------------------------------------ AdamW
 * Of every number p of every tensor, with its gradient g, at step t = 1, 2, ...:
 *   m = beta1 m + (1 - beta1) factor g,   v = beta2 v + (1 - beta2) (factor g)^2
 *   p = p - rate decay p - rate (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * p: dense fp32; g: dense, of the plan's type; copy: dense bf16, gets p rounded to it.  m and v are
 * two dense arrays for all tensors: a tensor's numbers begin a whole number of 256 after those of
 * the one before; what lies between is written as zero.  Zeros are a fresh state.
 * bits = 32: m and v in fp32.  bits = 8: of m its signed square root, of v its fourth root, in int8
 * and uint8 times a scale for each 256 numbers: scales [2][numbers / 256], m's first.  The scale is
 * the largest's times 1/127 (m) and 1/255 (v), factor and product rounded to fp32; a root over it is
 * rounded to the nearest whole number, halves to even, of v never down to zero.  p moves by m and v
 * before that rounding.  An m or v that is not finite (v from scaled gradients of 1.85e19 on, whose
 * square fp32 does not hold) makes those of its 256 numbers NaN.
 * The step's rate, t and factor are doubles in host memory (now), or, so that a recorded step may
 * run with new ones, fp32 in device memory (now_device); the other is NULL.
 * sizes: numbers of each tensor, >= 0; decays: decay of each.  Both are copied.
 * Errors of create: CONV_EINVAL for a NULL pointer, count < 1, a size < 0, an unknown type, bits
 * other than 8 and 32, betas outside [0, 1), an eps or decay that is negative or not finite;
 * CONV_EUNSUPPORTED beyond 2^20 tensors and 2^35 numbers. */
typedef struct {
    const int64_t *sizes;
    const double *decays;
    double beta1, beta2, eps;
    int32_t count, bits;
    int32_t dtype; /* of g */
    int32_t reserved;
} seq_adamw_desc_t;
conv_status_t seq_adamw_create(const seq_adamw_desc_t *desc, seq_handle_t *out);
/* p, g, copy: arrays of device pointers in host memory, one a tensor, read before the call returns.
 * A tensor whose g is NULL stays as it is, its state too.  copy: NULL, or NULL for some.
 * Tensors may not overlap.  scales: bits = 8 only. */
conv_status_t seq_adamw(seq_handle_t h, void *const *p, const void *const *g, void *const *copy,
                        void *m, void *v, float *scales, const double *now,
                        const float *now_device, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SEQ_MI355X_H */
