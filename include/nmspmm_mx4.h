/*
 * nmspmm_mx4.h -- C ABI of the 4-bit operators of a decoding step, in the
 * same library (libnmspmm.so):
 *   nmspmm_mx4_*  few rows times an N:M sparse (or, with N = M, dense) weight
 *                 held in 4 bits with a scale for every 32 kept rows
 *   nmspmm_kv4_*  a paged key-value cache held in 4 bits: new tokens written
 *                 into it, read back, and attention of one new token over it
 *
 * Four bits: a code c of 0 to 15 is a sign (c >= 8: negative) and one of the
 * magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 (c & 7); a scale is a byte s that
 * stands for 2^(s - 127), 255 for NaN.  32 values share a scale (the OCP
 * microscaling format with E2M1 elements).
 * Values are brought to 4 bits by one rule: the scale is the smallest power of
 * two with which the group's largest magnitude is at most 7 (from 2^-125 to
 * 2^125: s from 2 to 252), every value goes to the nearest magnitude times it,
 * ties to the even code, 6 at most.  A group that holds an infinity or NaN
 * gets s = 255 and reads as NaN throughout.  Values of 4 bits come back as
 * they are from a second rounding.
 *
 * Entry points, strides, streams, workspaces and errors as in nmspmm_serve.h.
 */
#ifndef NMSPMM_MX4_H
#define NMSPMM_MX4_H

#include "nmspmm_serve.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- The product with a 4-bit weight ----------------------------------- */

/* A weight in 4 bits, laid out once: nmspmm_mx4_pack writes `packed`.  Shape
 * and pattern as in nmspmm.h; w = (k/M)*N compressed rows. */
typedef struct {
    const void *packed;     /* nmspmm_mx4_bytes bytes, 256-byte aligned */
    int32_t N, M, V;
    int64_t k, n;
} nmspmm_mx4_weight_t;

/* Bytes of a packed weight, or -1 for a bad shape.  Host only. */
NMSPMM_API int64_t nmspmm_mx4_bytes(int64_t k, int64_t n, int N, int M, int V);

/* Brings the values Bc (w x n, row-major, of bc_dtype, as nmspmm_compress
 * writes them) to 4 bits by the rule above: codes (w x n bytes, row-major, 0
 * to 15) and scales (ceil(w/32) x n bytes, row-major: row g is shared by the
 * compressed rows 32g to 32g+31 of its column).  w == 0 or n == 0 returns
 * NMSPMM_OK without a launch.  Errors: NMSPMM_ERR_INVALID_ARG (negative size,
 * bad type, null pointer with non-empty data), NMSPMM_ERR_UNSUPPORTED
 * (misaligned pointer, sizes beyond int64, w or n of 2^31 - 255 or more),
 * NMSPMM_ERR_HIP. */
NMSPMM_API nmspmm_status_t nmspmm_mx4_quantize(const void *Bc, nmspmm_dtype_t bc_dtype, int64_t w, int64_t n,
                                    uint8_t *codes, uint8_t *scales, hipStream_t stream);

/* Lays a weight out for nmspmm_mx4_run.  codes and scales as
 * nmspmm_mx4_quantize writes them (or from elsewhere: any scale byte, but a
 * value that fp32 does not hold, of the bytes 253 and 254, may count as an
 * infinity; of a code the low four bits count), idx (w x q bytes) as in
 * nmspmm.h, read only.
 * weight->packed is written.  An offset >= M is clamped to M-1, as nmspmm_run
 * does; with N = M the offsets are 0 to M-1 and idx is not read (it may be
 * NULL).  Errors: as for nmspmm_half_pack. */
NMSPMM_API nmspmm_status_t nmspmm_mx4_pack(const uint8_t *codes, const uint8_t *scales, const uint8_t *idx,
                                const nmspmm_mx4_weight_t *weight, hipStream_t stream);

/* Bytes of workspace with which nmspmm_mx4_run splits k for a product of m
 * rows: 0 where it does not, -1 for a bad shape.  Host only. */
NMSPMM_API int64_t nmspmm_mx4_workspace_bytes(int64_t m, const nmspmm_mx4_weight_t *weight);

/* The sparse product of nmspmm.h (Eq. 1) with a 4-bit weight:
 *   C[i][j] = act(alpha * (A * B)[i][j] + bias[j]) * mul[i][j] + residual[i][j]
 *   A        m x k of a_dtype (NMSPMM_BF16 or NMSPMM_F16), row stride lda,
 *            columns contiguous
 *   C        m x n of c_dtype (a_dtype or NMSPMM_F32), row stride ldc
 *   bias, act, mul, residual   as in nmspmm_half_run
 * Products of A's values and the weight's are exact in fp32; sums, epilogue
 * and (where k is split) partial sums are fp32; C is rounded once (ties to
 * even).  The order of summation is fixed by shape, alignment and workspace.  Only kept
 * rows of B enter a sum.  Made for the 1 to 16 rows of decoding: from 17 rows
 * on nmspmm_half_run on a 16-bit weight is about as fast or faster (4096 x 11008
 * at 8:32: 7.9 and 11.8 us for 16 rows, 11.5 and 10.2 for 17, 34 and 28 for 256).
 * A's rows start on 16 bytes, or a product of more than one row takes up to three
 * times as long, of more than 16 up to six.  m == 0 or n == 0 returns NMSPMM_OK
 * without a launch; with k == 0 the sum is zero.  Errors: as for nmspmm_half_run. */
NMSPMM_API nmspmm_status_t nmspmm_mx4_run(const void *A, int64_t lda, nmspmm_dtype_t a_dtype,
                               const nmspmm_mx4_weight_t *weight, void *C, int64_t ldc, nmspmm_dtype_t c_dtype,
                               int64_t m, float alpha, const float *bias, nmspmm_half_act_t act, const void *mul,
                               int64_t ld_mul, const void *residual, int64_t ld_residual, void *workspace,
                               size_t workspace_bytes, hipStream_t stream);

/* Name of the kernel that nmspmm_mx4_run launches for m rows that start on 16
 * bytes, with a workspace or without ("none": no launch, "invalid": bad
 * shape), for reports.  Valid until the thread's next call. */
NMSPMM_API const char *nmspmm_mx4_kernel_name(int64_t m, const nmspmm_mx4_weight_t *weight, int with_workspace);

/* ---- The paged cache in 4 bits ------------------------------------------ */

/* A cache of `pages` pages of page_size tokens, each token `heads` rows of
 * `dim` values for keys and for values, a row in groups of 32 dimensions (the
 * last may be shorter) that share a scale.  Page p lies at pages + p*page_stride
 * bytes and is nmspmm_kv4_page_bytes long; how the library lays rows out in it
 * is its own affair (nmspmm_kv4_append writes, nmspmm_kv4_read reads them).  A
 * page's memory needs no clearing.  Table and positions as in
 * nmspmm_kv_cache_t. */
typedef struct {
    void *pages;            /* 16-byte aligned */
    int64_t page_stride;    /* a multiple of 16, at least the page's bytes */
    int64_t page_count;
    const int32_t *table;
    int64_t table_stride;
    int64_t sequences;      /* rows of the table */
    int64_t table_pages;    /* entries of a row */
    int32_t page_size, heads, dim;
} nmspmm_kv4_cache_t;

/* Bytes of a page (a multiple of 16), or -1 for bad sizes (below 1, or dim
 * beyond 512).  Host only. */
NMSPMM_API int64_t nmspmm_kv4_page_bytes(int64_t page_size, int64_t heads, int64_t dim);

/* Writes the keys and values of `tokens` new tokens into the cache, as
 * nmspmm_kv_append_norm does, and brings them to 4 bits by the rule above.
 * Keys are normalised and turned in fp64, so that their codes are those of the
 * formula (except where it comes within 2^-45 or so of a border); queries as
 * there, in fp32.  The places of one call's tokens must differ: a place that
 * is named twice is left with a mixture.  Errors: as for
 * nmspmm_kv_append_norm, and NMSPMM_ERR_INVALID_ARG for a page_stride below
 * the page's bytes, NMSPMM_ERR_UNSUPPORTED for one that is no multiple of 16
 * or pages off 16 bytes. */
NMSPMM_API nmspmm_status_t nmspmm_kv4_append(const nmspmm_kv4_cache_t *cache, const void *k_new, const int64_t *k_stride,
                                  const void *v_new, const int64_t *v_stride, nmspmm_dtype_t dtype, int64_t tokens,
                                  const int32_t *seq, const int32_t *pos, const float *cos, const float *sin,
                                  int64_t positions, int rot, int interleaved, const float *q_norm,
                                  const float *k_norm, float eps, const void *q, const int64_t *q_stride,
                                  void *q_out, const int64_t *q_out_stride, int64_t q_heads, hipStream_t stream);

/* Reads the keys and values of `tokens` places back, as the values that their
 * codes stand for, rounded once to `dtype`: token t is position pos[t] of
 * sequence seq[t].
 *   k_out, v_out   tokens x heads x dim of `dtype`; element (t, h, d) at
 *                  t*stride[0] + h*stride[1] + d; either may be NULL: not read
 * A token whose sequence, position or page lies outside its array is skipped:
 * its rows of k_out and v_out are left as they were.  tokens == 0 returns
 * NMSPMM_OK without a launch.  Errors: as for nmspmm_kv4_append. */
NMSPMM_API nmspmm_status_t nmspmm_kv4_read(const nmspmm_kv4_cache_t *cache, int64_t tokens, const int32_t *seq,
                                const int32_t *pos, nmspmm_dtype_t dtype, void *k_out, const int64_t *k_stride,
                                void *v_out, const int64_t *v_stride, hipStream_t stream);

/* Bytes of workspace with which nmspmm_kv4_attend splits the sequences of
 * this cache: 0 where it does not, -1 for bad sizes.  Host only. */
NMSPMM_API int64_t nmspmm_kv4_attend_workspace_bytes(const nmspmm_kv4_cache_t *cache, int64_t q_heads,
                                          int64_t max_length, int64_t window);

/* Attention of one new token per sequence over the 4-bit cache: arguments,
 * results and what is left out as in nmspmm_kv_attend (an infinite query as an
 * infinity in the range there).  Scores, softmax and
 * sums are fp32; queries and weights of the softmax enter the products with
 * all their bits (in bf16 parts), the cache's values as they are. */
NMSPMM_API nmspmm_status_t nmspmm_kv4_attend(const nmspmm_kv4_cache_t *cache, const void *q, const int64_t *q_stride,
                                  nmspmm_dtype_t dtype, int64_t q_heads, const int32_t *lengths, int64_t max_length,
                                  int64_t window, float scale, void *out, const int64_t *out_stride, float *lse,
                                  void *workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* NMSPMM_MX4_H */
