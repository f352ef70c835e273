/*
 * als_serve.h -- answering with a trained factor model on an AMD Instinct MI355X (gfx950).
 *
 * What als.h leaves in X and Theta answers requests through three operators:
 *
 *     als_quantize   rows of a factor as 8-bit integers with one scale a row
 *     als_score      the scores of users against items, from 8-bit rows of both
 *     als_sample     one item a user, drawn from a row of scores
 *
 * The conventions are those of als.h: device pointers owned by the caller, no device memory allocated
 * or freed, argument checks before the call returns, all work queued on `stream` (a hipStream_t, NULL =
 * the null stream) without a host synchronisation, status codes and als_strerror of als.h, no C++
 * exception across the interface.  Strides are in elements.  A context serves one device and must not be
 * used from two host threads at once; calls queued on different streams of one context must not
 * overlap in time (they share the workspace).  Every call may be captured into a HIP graph.
 */
#ifndef ALS_SERVE_H
#define ALS_SERVE_H

#include "als.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of dense arguments. */
enum { ALS_F32 = 0, ALS_F16 = 1, ALS_BF16 = 2 };

/* Largest row length of als_quantize and als_score: sums of 128^2 f stay below 2^31. */
#define ALS_SERVE_F_MAX 131071
/* Most columns of als_sample: sums of 2^40 n stay below 2^62. */
#define ALS_SERVE_N_MAX 4194304

/* Columns of the longest row that als_sample draws from without the workspace.  (als_score does without it where both
   sides' rows lie at addresses and strides that are multiples of 16, strides below 2^22; als_quantize always.) */
#define ALS_SERVE_HELD_MAX 65536

typedef struct als_serve_ctx als_serve_ctx;

/* Bytes of device workspace a context on `device` needs; 0 if the device cannot be queried or is not a
   gfx950 device. */
size_t als_serve_workspace_bytes(int device);

/* Create a context on `device` using the caller's device workspace (at least
   als_serve_workspace_bytes(device) bytes, 256-byte aligned, kept alive until als_serve_destroy). */
int als_serve_init(als_serve_ctx** ctx, int device, void* workspace, size_t workspace_bytes);

/* Release the context (not the workspace).  Does not synchronise. */
int als_serve_destroy(als_serve_ctx* ctx);

/* HIP error code of the most recent ALS_ERR_HIP on this context (0 if none). */
int als_serve_last_hip_error(const als_serve_ctx* ctx);

/*
 * Rows of x as 8-bit integers with one scale each:
 *   a = max_k |x_uk|,   q_uk = rint(127 x_uk / a),   scale_u = a (1 / 127)     (so x_uk ~ scale_u q_uk)
 * 127 x and its quotient by a are each rounded to fp32, the quotient then to the nearest integer, ties to
 * even (127 x as if fp32 had no largest value); 1 / 127 and its product with a are rounded to fp32.  The result
 * is the same on every run.  A row of zeros gets scale 0 and zeros.  A row with an infinity or a NaN gets scale
 * NaN and zeros, so that its scores are NaN.
 *   x      : `of` rows of f values of type dtype, row stride ldx >= f
 *   users  : int32[rows], the rows of x to take (repeats allowed), or NULL: rows 0 .. rows - 1 (rows <= of).
 *            An entry outside [0, of) gives a row of scale NaN and zeros.
 *   q      : rows x f, row stride ldq >= f; columns f .. ldq - 1 are written as zeros up to the next
 *            multiple of 16 (or ldq, if that is less), in the last row too.  A stride that is a multiple of 16 is
 *            the fastest for als_score.
 *   scale  : fp32[rows]
 * q and scale must not overlap x, users or each other (ALS_ERR_ALIAS).  f in [1, ALS_SERVE_F_MAX].
 */
int als_quantize(als_serve_ctx* ctx, const void* x, int32_t dtype, int64_t of, int64_t ldx,
                 const int32_t* users, int64_t rows, int32_t f, int8_t* q, int64_t ldq, float* scale,
                 void* stream);

/*
 * als_quantize into rows of which only the first `width` columns are the caller's to write, f <= width <= ldq and
 * width no more than f's next multiple of 16: columns f .. width - 1 are written as zeros, what lies past them (columns
 * of other matrices, the end of the memory) is left alone.
 */
int als_quantize_into(als_serve_ctx* ctx, const void* x, int32_t dtype, int64_t of, int64_t ldx,
                      const int32_t* users, int64_t rows, int32_t f, int8_t* q, int64_t ldq, int32_t width,
                      float* scale, void* stream);

/*
 * Scores of m users against n items (or any product of 8-bit rows with a scale for each row of either):
 *   out[i][j] = ((float) sum_k xq_ik tq_jk) xs_i ts_j
 * The sum is exact (32-bit integers); it is rounded to fp32, multiplied by xs_i, then by ts_j, each product
 * rounded to fp32, and the result rounded to the output's type.  The result is the same on every run.
 *   xq, tq : int8, m x f and n x f, row strides ldx, ldt >= f, any alignment; what lies between f and the stride
 *            is not used
 *   xs, ts : fp32[m], fp32[n]
 *   out    : m x n of type dtype, row stride ldo >= n; must not overlap an input (ALS_ERR_ALIAS)
 */
int als_score(als_serve_ctx* ctx, const int8_t* xq, int64_t ldx, const float* xs, int64_t m,
              const int8_t* tq, int64_t ldt, const float* ts, int64_t n, int32_t f, void* out,
              int32_t dtype, int64_t ldo, void* stream);

/* What a row asks of als_sample: an array with one value for each row, or, where the pointer is NULL, one
   value for all rows. */
typedef struct {
    const float* temperature;   /* T > 0; any other value (0, NaN) asks for the best column */
    const int32_t* top_k;       /* columns kept by rank; <= 0: all */
    const float* top_p;         /* share of the weight kept; >= 1 or NaN: all, <= 0: the best column */
    const float* min_p;         /* least weight kept, relative to the best column's; <= 0 or NaN: all */
    float temperature_all;
    int32_t top_k_all;
    float top_p_all;
    float min_p_all;
} als_sample_limits;

/*
 * One column a row, drawn from its scores z by a given uniform number:
 *   1. Allowed columns: z above -inf and not NaN, and not among the columns of the row's CSR row.  A row without any
 *      gets index -1 and log -inf.
 *   2. Order: z descending, among equals the lower column first (-0 equals 0).  The first top_k stay.
 *   3. Weights: whole numbers w = floor(2^40 exp((z - max z) / T)), in fp32 up to the rounding down: the
 *      difference, its product with 1 / T (rounded once) and the exponential.  A difference past fp32's
 *      range weighs nothing, whatever T.  A score of +inf weighs 2^40, and then finite ones nothing.
 *      Sums of weights are exact, so no result depends on an order of summation.
 *   4. top_p: with W the sum of the weights so far, a column stays while the weight before it in the
 *      order is below floor(W floor(2^24 top_p) / 2^24), at least one column.
 *   5. min_p: columns whose exponential is below min_p go.
 *   6. With W' the sum of what is left and t = floor(W' floor(2^24 u) / 2^24), the result is the first column,
 *      by column number, at which the running sum of the weights exceeds t.
 *   index : int32[rows], the column drawn
 *   log   : fp32[rows] or NULL, the natural logarithm of w / W' without the rounding down of w
 * z     : rows x n of type dtype, row stride ldz >= n; n in [0, ALS_SERVE_N_MAX]
 * u     : fp32[rows] in [0, 1) (clamped to it; NaN counts as 0)
 * rated_ptr, rated_idx : a CSR with `of` rows (int64[of + 1], int32) of columns to leave out, in any order (one
 *         outside [0, n) is skipped), or both NULL.  Row r leaves out CSR row users[r] (int32[rows]), or r if
 *         users is NULL (then of >= rows).  An entry of users outside [0, of) gives index -1 and log NaN.
 * index and log must not overlap an input or each other (ALS_ERR_ALIAS; rated_idx is the caller's to look at, as its
 * length is on the device).
 */
int als_sample(als_serve_ctx* ctx, const void* z, int32_t dtype, int64_t rows, int64_t n, int64_t ldz,
               const als_sample_limits* limits, const float* u, const int64_t* rated_ptr,
               const int32_t* rated_idx, const int32_t* users, int64_t of, int32_t* index, float* log,
               void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ALS_SERVE_H */
