/*
 * ea_block.h -- C ABI of the operators inside a residual block of a language model, between those of ea_lm.h
 * at its two ends: layer norm, a gated linear recurrence along each sequence, and dropout from a counter, each with its
 * gradient.
 *
 * Calls, streams, workspaces, graphs, devices and errors are as in ea_lm.h: every call is asynchronous on the stream
 * given to the init call, except the *_sync_status and *_selftest_* calls; the library allocates no device memory; a
 * handle belongs to one device and to one host thread at a time; a call that is refused has done nothing, and
 * ea_last_error(NULL) says why.
 *
 * Tensors are rows of `dim` consecutive elements, outer x inner of them: row (i, j) lies at i * outer stride +
 * j * inner stride elements from the address.  Strides of what is read may be any that stay inside the caller's memory
 * (0 for one row in the place of many); rows that are written may not overlap, so the smaller of their strides is at least
 * dim and the larger at least the extent of the rows along the smaller.  Every address is aligned to its element.  What is
 * written overlaps nothing that the call reads or writes, but where a call says that one tensor may be another.
 * The layer norm's backward call writes to its handle's workspace: graphs that hold such calls of one handle are replayed
 * one after another.
 */
#ifndef EA_BLOCK_H
#define EA_BLOCK_H

#include "ea_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------- layer norm */

typedef struct ea_layernorm_config {
    int64_t dim;      /* 1 .. 2^20 */
    int64_t max_rows; /* most rows of one call, 0 .. 2^30 */
    float eps;        /* >= 1e-30, finite */
} ea_layernorm_config;

typedef struct ea_layernorm ea_layernorm;

typedef struct ea_layernorm_call {
    int64_t outer, inner;         /* rows, each >= 0 */
    int64_t x_outer, x_inner;     /* strides of x */
    int64_t y_outer, y_inner;     /* of y or dy */
    int64_t dx_outer, dx_inner;
    int64_t add_outer, add_inner;
    int32_t x_type;               /* of x, dx and add: EA_T_F32, EA_T_BF16 or EA_T_F16 */
    int32_t y_type;               /* of y or dy: x_type, or with EA_T_F32 there any of the three */
    int32_t weight_type;          /* of w and b: any of the three */
    int32_t grad_type;            /* of dw and db: any of the three */
} ea_layernorm_call;

int ea_layernorm_workspace_bytes(const ea_layernorm_config *cfg, size_t *bytes);
int ea_layernorm_init(const ea_layernorm_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_layernorm **out);

/* y = (x - mean) * rstd * w + b for every row, mean its mean, rstd = 1 / sqrt(variance + eps) with the variance about that
 * mean; in binary32, rounded once to y's type (of a row whose sum or squares pass binary32's range, y is not to be used).
 * w, b: dim values, or NULL for ones and zeros.  stats: NULL, or two binary32 values per row (mean, rstd; row (i, j) at
 * 2 (i * inner + j)) for the backward call, aligned to 8 bytes.  y may be x, with the same strides and type. */
int ea_layernorm_forward(ea_layernorm *h, const ea_layernorm_call *c, const void *x, const void *w, const void *b, void *y, float *stats);

/* With t = (x - mean) * rstd and q = dy * w, per row
 *   dx = add + rstd * (q - mean of q - t * mean of q t),    and over all rows    dw = sum of dy t,  db = sum of dy,
 * with accumulate = 1 added to what dw and db hold.  add: NULL, or rows that are added (the gradient that passes the block
 * by).  dx, dw, db: each may be NULL.  In binary32, sums in an order that depends on the call's sizes, types and alignment
 * alone (the same bits on every run), rounded once to the type at hand.  dx may be dy, x or add, with the same strides and
 * type.  stats: of the forward call. */
int ea_layernorm_backward(ea_layernorm *h, const ea_layernorm_call *c, const void *dy, const void *x, const float *stats, const void *w,
                          const void *add, void *dx, void *dw, void *db, int32_t accumulate);
int ea_layernorm_destroy(ea_layernorm *h);

/* ------------------------------------------------------------------------------- gated linear recurrence */

typedef struct ea_scan_config {
    int64_t dim; /* 1 .. 2^20 */
} ea_scan_config;

typedef struct ea_scan ea_scan;

/* batch sequences of length rows: row t of sequence i at i * batch stride + t * row stride. */
typedef struct ea_scan_call {
    int64_t batch, length;      /* 0 .. 2^24 and 0 .. 2^30, batch * dim < 2^31 */
    int64_t z_batch, z_row;
    int64_t v_batch, v_row;
    int64_t h_batch, h_row;
    int64_t dh_batch, dh_row;
    int64_t dz_batch, dz_row;
    int64_t dv_batch, dv_row;
    int32_t type;               /* of all of these: EA_T_F32, EA_T_BF16 or EA_T_F16 */
    int32_t length_type;        /* of lengths, where they are given: EA_T_I32 or EA_T_I64 */
} ea_scan_call;

int ea_scan_workspace_bytes(const ea_scan_config *cfg, size_t *bytes);
int ea_scan_init(const ea_scan_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_scan **out);

/* In every sequence and column, with f_t = 1 / (1 + exp(-z_t)),
 *   h_t = f_t h_{t-1} + (1 - f_t) v_t,    h_{-1} = initial,
 * the states carried in binary32 and each rounded once to h's type.  f and 1 - f each are within (4 + 0.7 |z|) 2^-23 of
 * themselves (exp's argument is a rounded product, whose absolute error grows with |z|) and 2^-126.  Each is rounded by itself,
 * and each of the terms that make up a state is off, relative to itself, by what f is and a rounding for every row that it is
 * carried through, 2^-21 at most where z >= 0 (2^-25 was measured where gates nearly hold): over very many rows of such gates f and
 * 1 - f do not keep a state between its inputs as a mean would.  A state that is not finite leaves the later ones of its column
 * not finite.
 * initial: batch x dim binary32 values, or NULL for zeros.  final: NULL, or batch x dim binary32 values that receive every
 * sequence's last state; it may be initial.
 * lengths: NULL, or one length per sequence on the device: rows from there on are not read, their h is 0, and the state after
 * the last row before them is the final one (the initial one for a length of 0).  A length outside [0, length] counts as
 * the nearest of the two, and ea_scan_sync_status reports it.  h may be z or v, with the same strides. */
int ea_scan_forward(ea_scan *s, const ea_scan_call *c, const void *z, const void *v, const float *initial, const void *lengths, void *h,
                    float *final);

/* With g_t = dh_t + f_{t+1} g_{t+1}, f_{t+1} g_{t+1} = d_final behind the last row, and h as the forward call stored it,
 *   dv_t = (1 - f_t) g_t,    dz_t = f_t (1 - f_t) g_t (h_{t-1} - v_t),    d_initial = f_0 g_0,
 * in binary32, g carried and each result rounded once.  initial, lengths: of the forward call.  d_final, d_initial: NULL, or
 * batch x dim binary32 values.  dz and dv of rows behind a sequence's length are 0.  d_initial may be d_final; dz may be z and
 * dv may be v or dh (or dz may be dh), with the same strides. */
int ea_scan_backward(ea_scan *s, const ea_scan_call *c, const void *dh, const void *z, const void *v, const void *h, const float *initial,
                     const void *lengths, const float *d_final, void *dz, void *dv, float *d_initial);

/* Synchronize the stream; EA_E_CUDA for a CUDA error, EA_E_DEVICE_CHECK if a length since the last such call lay outside
 * [0, length], EA_E_TIMEOUT if a wait between the CTAs of a cluster ran out (after two seconds; what the call wrote is then
 * not to be used). */
int ea_scan_sync_status(ea_scan *s);
int ea_scan_destroy(ea_scan *s);

/* The exchange between the CTAs of a cluster by itself, with this limit (in cycles of the SM) of its waits: EA_OK with
 * *timed_out = 0 where all of them take part (silent = -1), and with 1 where CTA `silent` (0 .. 3) stops halfway: the others'
 * waits run out, and the kernel ends. */
int ea_scan_selftest_exchange(int64_t limit_cycles, int32_t silent, void *stream, int32_t *timed_out);

/* ------------------------------------------------------------------------------- dropout */

typedef struct ea_dropout_config {
    double p;      /* probability that an element is dropped, in [0, 1]; taken as the nearest multiple of 2^-16 (ties to even) */
    uint64_t seed; /* Philox key */
} ea_dropout_config;

typedef struct ea_dropout ea_dropout;

typedef struct ea_dropout_call {
    int64_t outer, inner, dim;    /* each >= 0, outer * inner * dim <= 2^40 */
    int64_t x_outer, x_inner;
    int64_t add_outer, add_inner;
    int64_t y_outer, y_inner;
    int32_t x_type;               /* EA_T_F32, EA_T_BF16 or EA_T_F16 */
    int32_t y_type;               /* of y and add: x_type, or EA_T_F32, or with EA_T_F32 in x_type any */
} ea_dropout_call;

int ea_dropout_workspace_bytes(const ea_dropout_config *cfg, size_t *bytes);
int ea_dropout_init(const ea_dropout_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_dropout **out);

/* y = add + (x / (1 - p) where the element is kept, 0 where it is dropped), in binary32, rounded once to y's type; add may be
 * NULL.  Element e, counted through the rows (e = (i * inner + j) * dim + column), is dropped where half word e mod 8 (the low
 * half of a word first) of Philox4x32-10 at the counter (e / 8 low, e / 8 high, counter low, counter high) under the key seed is
 * below 2^16 p.  The mask depends on seed, counter and e alone: the same call with dy for x and no add is the gradient.
 * device_counter: NULL, or one 64-bit value on the device that is read in the place of counter, so that a replayed graph
 * can draw other masks.  y may be x or add, with the same strides and type. */
int ea_dropout_apply(ea_dropout *h, const ea_dropout_call *c, const void *x, const void *add, uint64_t counter,
                     const uint64_t *device_counter, void *y);
int ea_dropout_destroy(ea_dropout *h);

#ifdef __cplusplus
}
#endif

#endif /* EA_BLOCK_H */
