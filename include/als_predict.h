/*
 * als_predict.h -- how probable items are under a trained factor model, on an AMD Instinct MI355X (gfx950).
 *
 * als_serve.h answers from 8-bit rows; here are predictions at the factors' own precision, and what they say of given
 * items:
 *
 *     als_predict         predictions of users for items, with the model's offsets, an activation and a residual
 *     als_log_prob        the log probabilities of given items in rows of scores, with the rows' entropy and best items
 *     als_log_prob_grad   their gradient with respect to the scores, or to the items' offsets
 *
 * A row of scores stands for the distribution that als_sample draws from without top-k, top-p and min-p: p = softmax(z / T)
 * over the allowed columns.  The conventions are those of als_serve.h (device pointers owned by the caller, no device
 * memory allocated or freed, checks before the call returns, work queued on `stream` without a host synchronisation,
 * status codes and als_strerror of als.h, no C++ exception across the interface, strides in elements, one host thread at a
 * time; calls on one context's different streams must not overlap in time, as they share the workspace).  Every
 * call may be captured into a HIP graph.  Results are the same on every run: sums are taken in a fixed order.
 */
#ifndef ALS_PREDICT_H
#define ALS_PREDICT_H

#include "als_serve.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest row length of als_predict. */
#define ALS_PREDICT_F_MAX 1048576
/* Most columns of als_log_prob and als_log_prob_grad. */
#define ALS_PREDICT_N_MAX 4194304
/* Most alternatives of als_log_prob. */
#define ALS_PREDICT_TOP_MAX 128

typedef struct als_predict_ctx als_predict_ctx;

/* Bytes of device workspace a context on `device` needs; 0 if the device cannot be queried or is not a
   gfx950 device. */
size_t als_predict_workspace_bytes(int device);

/* Create a context on `device` using the caller's device workspace (at least
   als_predict_workspace_bytes(device) bytes, 256-byte aligned, kept alive until als_predict_destroy). */
int als_predict_init(als_predict_ctx** ctx, int device, void* workspace, size_t workspace_bytes);

/* Release the context (not the workspace).  Does not synchronise. */
int als_predict_destroy(als_predict_ctx* ctx);

/* HIP error code of the most recent ALS_ERR_HIP on this context (0 if none). */
int als_predict_last_hip_error(const als_predict_ctx* ctx);

/* Activations; y is the product with its offsets.  Where y is -inf, GELU and SILU are -0, their limit.  A NaN stays.
   Exponentials below 2^-126 are 0: so are SIGMOID and SILU where y is below -87.3, and GELU where y is below -13.2. */
enum {
    ALS_ACT_NONE = 0,
    ALS_ACT_CLIP = 1,       /* min(max(y, low), high), low <= high (infinities allowed) */
    ALS_ACT_RELU = 2,       /* max(y, 0) */
    ALS_ACT_GELU = 3,       /* y (1 + erf(y / sqrt 2)) / 2 */
    ALS_ACT_SILU = 4,       /* y / (1 + exp(-y)) */
    ALS_ACT_SIGMOID = 5,    /* 1 / (1 + exp(-y)) */
    ALS_ACT_TANH = 6
};

/*
 * Predictions of m users for n items (or any product of rows with rows, with what follows it):
 *   y_ij = sum_k x_uk theta_jk + user_offset_u + item_offset_j,   out_ij = act(y_ij) + residual_ij
 * with u = users[i], or i.  Sums are held in fp32.  Products of f16 and bf16 are exact; fp32 rows are taken
 * apart into three bf16 parts of 8 bits each, which hold them exactly (below 2^-110 parts are lost), and multiplied in
 * six products that leave out what lies 2^-23 and more below a product: fp32's own precision.  A row of fp32 with an
 * infinity gives NaN; elsewhere infinities and NaN go as IEEE arithmetic has them.  The result is
 * rounded once to the output's type.
 *   x, theta  : `of` x f and n x f, both of type dtype, row strides ldx, ldt >= f, any alignment of their elements
 *   users     : int32[m], the rows of x to take (repeats allowed), or NULL: rows 0 .. m - 1 (m <= of).
 *               An entry outside [0, of) gives a row of NaN.
 *   user_offset, item_offset : fp32[of], fp32[n], or NULL.  An offset of -inf leaves an item out of what als_sample
 *               and als_log_prob make of the row.
 *   residual  : m x n of the output's type, row stride ldr >= n, or NULL.  It may be `out` itself (the same
 *               pointer and stride).
 *   out       : m x n of type out_dtype, row stride ldo >= n; must not overlap an input but so (ALS_ERR_ALIAS)
 * f in [1, ALS_PREDICT_F_MAX].  Rows of 16-bit types at addresses and strides that are multiples of 16 bytes (and fp32 ones
 * at strides of multiples of 128) are the fastest; of such a 16-bit row the last 16 bytes that hold a value are read whole,
 * up to 14 bytes past it (within the same 16 bytes), and what lies there does not count.
 */
int als_predict(als_predict_ctx* ctx, const void* x, int64_t of, int64_t ldx, const int32_t* users, int64_t m,
                const void* theta, int64_t n, int64_t ldt, int32_t dtype, int32_t f, const float* user_offset,
                const float* item_offset, int32_t activation, float low, float high, const void* residual,
                int64_t ldr, void* out, int64_t ldo, int32_t out_dtype, void* stream);

/* Rows of scores and what a distribution over their columns depends on. */
typedef struct {
    const void* z;              /* rows x n of type dtype, row stride ldz >= n; n in [0, ALS_PREDICT_N_MAX] */
    int32_t dtype;
    int64_t rows, n, ldz;
    const float* temperature;   /* fp32[rows], or NULL: temperature_all.  T > 0; any other value (0, NaN) puts all */
    float temperature_all;      /* of the probability on the best column, the lowest among equals */
    const int64_t* rated_ptr;   /* a CSR with `of` rows (int64[of + 1], int32) of columns to leave out, in any order */
    const int32_t* rated_idx;   /* (one outside [0, n) is skipped), or both NULL.  Row r leaves out CSR row users[r] */
    const int32_t* users;       /* (int32[rows]), or r if users is NULL (then of >= rows).  An entry of users outside */
    int64_t of;                 /* [0, of) makes all of a row's results NaN (and its top_index -1). */
} als_scores;

/* The columns of each row that are asked about. */
typedef struct {
    const int64_t* ptr;         /* int64[rows + 1]: row r has entries ptr[r] .. ptr[r + 1] - 1, as far as they lie in */
                                /* [0, entries).  Or NULL: it has entries r each .. r each + each - 1. */
    const int32_t* idx;         /* int32[entries]: columns, repeats allowed, in any order */
    int64_t entries;            /* how many there are; without ptr, rows x each */
    int64_t each;
} als_given;

/*
 * Rows of scores as distributions:
 *   Allowed columns: z above -inf and not NaN, and not among the row's columns to leave out.  y = z / T,
 *   p_j = exp(y_j) / sum exp(y) over the allowed columns; equal best scores of +inf share the probability.
 *   A difference from the best score, or its quotient by T, that is past fp32's range counts as -inf.
 *   log       : fp32[entries], log p of each given column; -inf for one that is left out or lies outside [0, n).
 *               Elements that belong to no row's entries are left alone.
 *   stats     : fp32[rows][2] or NULL, the best allowed score M and log sum exp((z - M) / T), for als_log_prob_grad;
 *               (-inf, -inf) for a row without an allowed column, (M, 0) where T is not above 0
 *   entropy   : fp32[rows] or NULL, - sum p log p; 0 for a row without an allowed column
 *   top_index, top_log : int32 and fp32, rows x top, or NULL (top = 0): the first `top` allowed columns in the order of
 *               als_sample (z descending, among equals the lower column first) and their log p; -1 and -inf past the last
 *               allowed one.  top in [0, ALS_PREDICT_TOP_MAX].
 * Outputs must not overlap an input or each other (ALS_ERR_ALIAS; rated_idx is the caller's to look at).
 */
int als_log_prob(als_predict_ctx* ctx, const als_scores* scores, const als_given* given, float* log, float* stats,
                 float* entropy, int32_t top, int32_t* top_index, float* top_log, void* stream);

/*
 * The gradient of  sum_e grad_log_e log p(given_e) + sum_r grad_entropy_r entropy_r  with respect to the scores:
 *   grad_rj = (1 / T_r) (sum of grad_log over the row's entries of column j - p_j G_r - grad_entropy_r p_j (log p_j + H_r))
 * with G_r the sum of grad_log over the row's entries and H_r its entropy.  Entries whose log p is -inf weigh nothing;
 * columns that are left out get 0; so does a row without an allowed column, or with T not above 0.
 *   log, stats, entropy : what als_log_prob gave for these scores (entropy only with grad_entropy)
 *   grad_log     : fp32[entries]
 *   grad_entropy : fp32[rows] or NULL
 *   grad         : rows x n of the scores' type, row stride ldg >= n, or NULL.  It may be the scores' own memory (the same
 *                  pointer and stride).
 *   columns      : fp32[n] or NULL, the gradient summed over the rows before any rounding to the scores' type: the
 *                  gradient of an offset that is added to every row's column.  n zeros if rows is 0.
 * Outputs must not overlap an input but so, or each other (ALS_ERR_ALIAS).
 */
int als_log_prob_grad(als_predict_ctx* ctx, const als_scores* scores, const als_given* given, const float* log,
                      const float* stats, const float* entropy, const float* grad_log, const float* grad_entropy,
                      void* grad, int64_t ldg, float* columns, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ALS_PREDICT_H */
