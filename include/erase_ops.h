/*
 * erase_ops.h -- C ABI of the operators of a transformer block around its
 * matrix products and its attention: rotary positions, layer norm, dropout,
 * each with its backward pass.  The transformer step of erase_tf.h runs them
 * inside its blocks on request (erase_tf_init_options); here they stand alone,
 * like the embedding-bag stage of erase.h.
 *
 * The conventions of erase.h hold: erase_status results, caller-owned device
 * memory on the current device, arguments checked on the host before anything
 * is enqueued, no device allocation, nothing thrown.  Every call enqueues on
 * `stream` (a HIP stream handle of the current device, NULL for the default
 * stream) and returns without waiting; it may be captured into a HIP graph
 * (kernel launches only) and keeps nothing between calls, so that calls on
 * several streams or host threads at once are independent as long as their
 * buffers are.  Types are erase_dtype (fp32 or bf16) for activations and their
 * gradients, fp32 for weights, statistics and weight gradients; arithmetic and
 * sums are fp32, each output is rounded once (to nearest, ties to even).
 * Pointers are aligned to their element; nothing else is asked of addresses
 * and pitches (rows that start on 16 bytes are the fastest).  Pitches and
 * strides count elements.  ERASE_ERR_INVALID_ARG for null, misaligned or
 * contradictory pointers, unknown enumerators and numbers out of range,
 * ERASE_ERR_SHAPE for sizes and pitches, ERASE_ERR_WORKSPACE for scratch,
 * ERASE_ERR_HIP when a launch fails.  A tensor of no elements may be NULL.
 * Outputs may not overlap inputs or each other except where a call says so.
 */
#ifndef ERASE_OPS_H_
#define ERASE_OPS_H_

#include "erase.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * Rotary positions.  The first rot_dim columns of every head hold rot_dim / 2
 * pairs (x1, x2); at position p pair i turns by the angle p f_i,
 *   y1 = a (x1 cos(p f_i) - x2 sin(p f_i)),  y2 = a (x2 cos(p f_i) + x1 sin(p f_i)),
 * and the other columns pass unchanged.  f_i and the amplitude a come from the
 * scaling (factor s, unscaled frequencies g_i = base^(-2 i / rot_dim)):
 *   NONE      f_i = g_i
 *   LINEAR    f_i = g_i / s                       (positions interpolated)
 *   NTK       f_i from the base base * s^(rot_dim / (rot_dim - 2))
 *   BY_PARTS  f_i = g_i (c_i + (1 - c_i) / s), a = 0.1 ln(s) + 1, with
 *             c_i = min(1, max(0, (L g_i / (2 pi) - slow) / (fast - slow))):
 *             pairs that turn often within the original length L keep their
 *             frequency, slow ones are interpolated (Peng et al. 2023, "YaRN").
 * a = 1 but for BY_PARTS. */
typedef enum { ERASE_ROPE_HALF = 0, ERASE_ROPE_INTERLEAVED = 1 } erase_rope_layout;
typedef enum {
  ERASE_ROPE_NONE = 0,
  ERASE_ROPE_LINEAR = 1,
  ERASE_ROPE_NTK = 2,
  ERASE_ROPE_BY_PARTS = 3
} erase_rope_scaling;

typedef struct {
  int32_t rot_dim;         /* even, 2..1024 */
  int32_t scaling;         /* erase_rope_scaling */
  double base;             /* >= 1, finite */
  double factor;           /* s >= 1, finite; not read for NONE */
  double original_length;  /* BY_PARTS: L > 0, finite */
  double fast, slow;       /* BY_PARTS: fast > slow >= 0, finite (32 and 1 in the paper) */
} erase_rope_spec;

/* The frequencies f_i (host, [rot_dim / 2]) and the amplitude a (host, [1]).
 * Host only; no HIP call. */
ERASE_API erase_status erase_rope_frequencies(const erase_rope_spec* spec, double* freq, double* amplitude);

/* The device table of a spec: per pair the turns of one position as a 64-bit
 * fraction of a full turn, f_i / (2 pi) modulo 1 in units of 2^-64, then the
 * amplitude.  The product position * fraction modulo 2^64 is the angle modulo
 * a turn.  The table puts it off by at most |position| 2^-63 turns (BY_PARTS with
 * fast and slow close together: times fast / (fast - slow)), and the kernel drops
 * what is below 2^-32 turns (1.5e-9 radians).  So every int32 position is as
 * accurate as a near one; position 2^40 is off by up to 7.5e-7 radians (an fp32
 * angle by 0.03 at 2^20 already).  erase_rope_table() fills `table` (8-byte aligned
 * device memory of erase_rope_table_bytes()) on `stream`; afterwards a table is
 * only read and serves any number of calls.  A caller orders another stream that
 * uses it after this one: no call waits for it. */
ERASE_API erase_status erase_rope_table_bytes(const erase_rope_spec* spec, size_t* bytes);
ERASE_API erase_status erase_rope_table(const erase_rope_spec* spec, void* table, void* stream);

/* Shape of one call: q and k are [batch][seq][heads][head_dim], heads' columns
 * contiguous, everything else by strides (batch row, position, head), so that
 * slices of a packed projection are taken where they are.  k_heads may be
 * smaller than q_heads (shared key heads) or 0 (no k: its pointers are not
 * read). */
typedef struct {
  int32_t dtype;            /* erase_dtype */
  int32_t layout;           /* erase_rope_layout: pairs (i, i + rot_dim / 2) or (2 i, 2 i + 1) */
  int32_t batch, seq;       /* >= 0, batch * seq < 2^31 */
  int32_t q_heads, k_heads; /* q_heads 1..4096, k_heads 0..4096 */
  int32_t head_dim;         /* rot_dim..1024 */
  int32_t rot_dim;          /* of the table: even, 2..head_dim */
  int64_t q_stride[3], k_stride[3];    /* >= 0 (0: read again, a broadcast) */
  int64_t qo_stride[3], ko_stride[3];  /* elements of an output may not coincide: sorted by size, each
                                          stride covers the extent of the ones before */
  int64_t pos_stride;       /* >= 0, of a row of `positions`; 0: one row for every batch row */
  int64_t start;            /* position of t = 0 when `positions` is NULL; |start| <= 2^40 */
} erase_rope_config;

/* q_out = rotated q, k_out = rotated k, one launch.  positions: device int32
 * [batch][seq] (unit stride along seq), any value including negative ones, or
 * NULL for start + t.  q_out may be q and k_out may be k, with the same
 * strides.  erase_rope_backward() turns by the negative angle: the gradients
 * at q and k from those at q_out and k_out (the transposed map, amplitude
 * included). */
ERASE_API erase_status erase_rope(const erase_rope_config* cfg, const void* q, const void* k, void* q_out, void* k_out,
                                  const int32_t* positions, const void* table, void* stream);
ERASE_API erase_status erase_rope_backward(const erase_rope_config* cfg, const void* dq_out, const void* dk_out, void* dq,
                                           void* dk, const int32_t* positions, const void* table, void* stream);

/* ------------------------------------------------------------------------
 * Layer norm over the columns of each row:
 *   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), h = (x - m) r, y = h w + b.
 * The variance is taken of the centred row (no difference of large sums), and
 * what the mean's own rounding leaves there is taken off the row and the variance,
 * so that rows of one value centre to zero.  (Sums are fp32: a row whose sum passes
 * 3.4e38 has no finite mean.) */
typedef struct {
  int64_t rows;   /* 0..2^31-1 */
  int32_t cols;   /* 1..16384 */
  int32_t dtype;  /* erase_dtype of x, y and their gradients */
  float eps;      /* >= 0, finite */
  int64_t x_ld, y_ld;           /* row pitches, >= cols */
  int64_t dy_ld, dx_ld, res_ld; /* of the backward pass */
} erase_norm_config;

/* w, b fp32 [cols], either may be NULL (ones, zeros); mean, rstd fp32 [rows],
 * either may be NULL (not wanted).  y may be x with the same pitch. */
ERASE_API erase_status erase_layer_norm(const erase_norm_config* cfg, const void* x, const float* w, const float* b,
                                        void* y, float* mean, float* rstd, void* stream);

/* Gradients from dy (at y) and the forward's x, mean and rstd:
 *   g = dy w,  dx = r (g - mean(g) - h mean(g h)) + res,
 *   dw = sum over rows of dy h,  db = sum over rows of dy.
 * res (the gradient that reaches x by another path, such as a residual's) may
 * be NULL, and so may dx, dw and db where they are not wanted; no rows give
 * dw = db = 0.  dx may be dy or res, with the same pitch.  dw and db are summed
 * in fp32 in an order that depends on the type, the sizes and whether dx is dy:
 * equal calls give equal bits.  scratch: erase_layer_norm_backward_scratch_bytes()
 * bytes of device memory (16-byte aligned, any contents), its own for every call
 * in flight; not read where neither dw nor db is wanted. */
ERASE_API erase_status erase_layer_norm_backward_scratch_bytes(const erase_norm_config* cfg, size_t* bytes);
ERASE_API erase_status erase_layer_norm_backward(const erase_norm_config* cfg, const void* x, const void* dy,
                                                 const float* w, const float* mean, const float* rstd, const void* res,
                                                 void* dx, float* dw, float* db, void* scratch, size_t scratch_bytes,
                                                 void* stream);

/* ------------------------------------------------------------------------
 * Dropout from a counter-based generator: the mask is a function of (seed,
 * offset, row, column) and is never stored; the backward pass computes it
 * again.  The random bits are Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011,
 * "Parallel random numbers: as easy as 1, 2, 3") with key (seed low, seed
 * high) and counter (column / 8, row, offset low, offset high); its four words
 * are eight 16-bit halves, low halves first, and column c takes half c mod 8:
 *   T = round(65536 p),  kept = half >= T,  y = res + (kept ? x * 65536 / (65536 - T) : 0).
 * So p is taken in steps of 2^-16 and the scale matches the step exactly; with
 * T = 65536 nothing is kept.  A dropped element contributes 0 whatever it is
 * (also NaN or infinity).  Calls with the same seed must differ in offset to
 * have independent masks. */
typedef struct {
  int64_t rows;     /* 0..2^31-1 */
  int64_t cols;     /* 0..2^31-1 */
  int32_t dtype;    /* erase_dtype */
  double p;         /* probability of dropping, 0..1 */
  uint64_t seed;
  uint64_t offset;
  int64_t x_ld, res_ld, y_ld; /* row pitches, >= cols (res_ld is not read without res) */
} erase_dropout_config;

/* res may be NULL (zeros).  step: device uint64 [1] or NULL; its value when the
 * launch runs is added to offset (modulo 2^64), so that a captured graph draws
 * new masks when the program advances the counter between replays.  y may be x
 * or res, with the same pitch. */
ERASE_API erase_status erase_dropout(const erase_dropout_config* cfg, const void* x, const void* res, void* y,
                                     const uint64_t* step, void* stream);

/* The gradient at x: dx = kept ? dy * 65536 / (65536 - T) : 0, for the seed,
 * offset and step of the forward call (x_ld: dy's pitch, y_ld: dx's; the
 * gradient at res is dy itself).  dx may be dy with the same pitch. */
ERASE_API erase_status erase_dropout_backward(const erase_dropout_config* cfg, const void* dy, void* dx,
                                              const uint64_t* step, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ERASE_OPS_H_ */
