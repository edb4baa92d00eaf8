/*
 * nmspmm_serve.h -- C ABI of the operators that a decoding step needs beside
 * the fp32 products of nmspmm.h, in the same library (libnmspmm.so):
 *   nmspmm_half_*  the N:M sparse product in bf16 or fp16 with its epilogue
 *   nmspmm_kv_*    a paged key-value cache: new tokens written into it, with
 *                  rotary positions, and attention of one new token over it
 *
 * As in nmspmm.h every entry point is extern "C", checks its arguments on the
 * host, returns a status code, never throws, enqueues its kernels on `stream`
 * (NULL = the legacy default stream) and returns without synchronizing.
 * Pointers are DEVICE pointers on the current HIP device unless said
 * otherwise.  Strides count elements.
 *
 * Workspaces: device memory aligned to 256 bytes, contents irrelevant, for
 * one call at a time.  With a workspace of at least the size that the
 * operator's *_workspace_bytes gives, the library allocates nothing.  Without
 * one (NULL or smaller) the call takes one of the library's cached buffers
 * of nmspmm_run (one per device and stream), or, while `stream` is being
 * captured into a graph or when none can be had, runs without splitting its
 * long axis.
 */
#ifndef NMSPMM_SERVE_H
#define NMSPMM_SERVE_H

#include "nmspmm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the operators below. */
typedef enum {
    NMSPMM_F32 = 0,
    NMSPMM_BF16 = 1,
    NMSPMM_F16 = 2
} nmspmm_dtype_t;

/* ---- The sparse product in 16 bits ------------------------------------- */

/* An N:M sparse weight in bf16 or fp16, laid out once for the product:
 * nmspmm_half_pack writes `packed`.  Shape and pattern as in nmspmm.h. */
typedef struct {
    const void *packed;     /* nmspmm_half_bytes bytes, 256-byte aligned */
    nmspmm_dtype_t dtype;   /* NMSPMM_BF16 or NMSPMM_F16 */
    int32_t N, M, V;
    int64_t k, n;
} nmspmm_half_weight_t;

/* Bytes of a packed weight, or -1 for a bad shape.  Host only. */
NMSPMM_API int64_t nmspmm_half_bytes(int64_t k, int64_t n, int N, int M, int V);

/* Lays a weight out for nmspmm_half_run.  Bc (w x n, row-major, of bc_dtype:
 * NMSPMM_F32, as nmspmm_compress and nmspmm_compress_device write it, or the
 * weight's own type) and idx (w x q bytes) as in nmspmm.h, read only.
 * weight->packed is written.  fp32 values are rounded to the nearest value of
 * weight->dtype (ties to even).  An offset >= M is clamped to M-1, as
 * nmspmm_run does.  Errors: NMSPMM_ERR_INVALID_ARG (bad shape or type, null
 * pointer with non-empty data), NMSPMM_ERR_UNSUPPORTED (misaligned pointer,
 * sizes beyond int64, n of 2^31 or more), NMSPMM_ERR_HIP. */
NMSPMM_API nmspmm_status_t nmspmm_half_pack(const void *Bc, nmspmm_dtype_t bc_dtype, const uint8_t *idx,
                                 const nmspmm_half_weight_t *weight, hipStream_t stream);

/* Activations of nmspmm_half_run's epilogue: nmspmm_act_t's three and SiLU. */
typedef enum {
    NMSPMM_HALF_ACT_NONE = 0,
    NMSPMM_HALF_ACT_RELU = 1,   /* max(0, y) */
    NMSPMM_HALF_ACT_GELU = 2,   /* y * Phi(y) */
    NMSPMM_HALF_ACT_SILU = 3    /* y / (1 + exp(-y)) */
} nmspmm_half_act_t;

/* Bytes of workspace with which nmspmm_half_run splits k for a product of m
 * rows, wherever A's rows start (rows on 16 bytes may need fewer): 0 where it
 * does not, -1 for a bad shape.  Host only. */
NMSPMM_API int64_t nmspmm_half_workspace_bytes(int64_t m, const nmspmm_half_weight_t *weight);

/* The sparse product of nmspmm.h (Eq. 1) with 16-bit operands:
 *   C[i][j] = act(alpha * (A * B)[i][j] + bias[j]) * mul[i][j] + residual[i][j]
 *   A        m x k of the weight's type, row stride lda, columns contiguous
 *   C        m x n of c_dtype (the weight's type or NMSPMM_F32), row stride
 *            ldc, overwritten
 *   bias     n fp32 values, or NULL: none
 *   mul, residual   m x n of c_dtype, row strides ld_mul and ld_residual, or
 *            NULL: no factor, no term.  Either may be C itself (same pointer
 *            and stride): every element is read by the thread that overwrites
 *            it.  No other overlap of C with an input is allowed.
 * Products of two 16-bit values are exact in fp32; sums, epilogue and (where
 * k is split) partial sums are fp32; C is rounded once (ties to even).  The
 * order of summation is fixed by shape, alignment and workspace: results do not vary
 * between runs.  Only kept rows of B enter a sum: an infinity or NaN in a
 * column of A that a column block does not keep leaves that block alone.
 * Where A starts on 16 bytes and k is odd, the 4-byte word of the last row's
 * last value is read whole: the two bytes after A's end, which are not used.
 * A weight of which some whole windows, 128 columns of A at most, come to a
 * multiple of 8 columns and to 64 kept rows at most (128 where V is no multiple of
 * 32) runs on the matrix instructions where V is a multiple of 16, k below 2^21
 * and lda too; any other, on a kernel of 3 to 6 TFLOP/s.
 * m == 0 or n == 0 returns NMSPMM_OK without a launch; with k == 0 the sum is
 * zero.  Errors: NMSPMM_ERR_INVALID_ARG (bad shape, type or activation, a row
 * stride below the row's length, null pointer with non-empty data),
 * NMSPMM_ERR_UNSUPPORTED (misaligned pointer, sizes beyond int64, n of 2^31 or
 * more), NMSPMM_ERR_HIP. */
NMSPMM_API nmspmm_status_t nmspmm_half_run(const void *A, int64_t lda, const nmspmm_half_weight_t *weight, void *C,
                                int64_t ldc, nmspmm_dtype_t c_dtype, int64_t m, float alpha, const float *bias,
                                nmspmm_half_act_t act, const void *mul, int64_t ld_mul, const void *residual,
                                int64_t ld_residual, void *workspace, size_t workspace_bytes,
                                hipStream_t stream);

/* Name of the kernel that nmspmm_half_run launches for m rows that start on 16
 * bytes (others may take another), with a workspace or without ("none": no launch, "invalid": bad shape), for reports.
 * Valid until the thread's next call. */
NMSPMM_API const char *nmspmm_half_kernel_name(int64_t m, const nmspmm_half_weight_t *weight, int with_workspace);

/* ---- The paged key-value cache ----------------------------------------- */

/* A cache of `pages` pages of page_size tokens, each token `heads` rows of
 * `dim` contiguous values for keys and for values.  Element (page, slot, head,
 * d) of k_pages lies at page*k_stride[0] + slot*k_stride[1] + head*k_stride[2]
 * + d, and likewise for v_pages; strides may be any that keep the rows apart.
 * Position p of sequence s lies in page table[s*table_stride + p/page_size],
 * slot p % page_size; an entry of the table that no call reaches may hold
 * anything. */
typedef struct {
    void *k_pages, *v_pages;
    int64_t k_stride[3], v_stride[3];
    int64_t pages;
    const int32_t *table;
    int64_t table_stride;
    int64_t sequences;      /* rows of the table */
    int64_t table_pages;    /* entries of a row */
    int32_t page_size, heads, dim;
    nmspmm_dtype_t dtype;
} nmspmm_kv_cache_t;

/* Writes the keys and values of `tokens` new tokens into the cache.  Token t
 * is position pos[t] of sequence seq[t].
 *   k_new, v_new   tokens x heads x dim of `dtype`; element (t, h, d) at
 *                  t*stride[0] + h*stride[1] + d
 *   cos, sin       positions x rot/2 fp32, row-major: the rotary angles.  The
 *                  first rot dimensions of every key (rot even, rot <= dim)
 *                  are turned, in fp32, in pairs (d, d + rot/2), or, where
 *                  `interleaved` is not 0, (2d, 2d + 1):
 *                    (a, b) -> (a cos - b sin, a sin + b cos).
 *                  NULL with rot = 0: keys are copied.
 *   q, q_out       tokens x q_heads x dim of `dtype`: queries, turned the same
 *                  way into q_out, which may be q itself (same pointer and
 *                  strides).  NULL with q_heads = 0: none.
 * A value is rounded once to the cache's type (ties to even).  A token whose
 * sequence, position, page or (with cos) row of angles lies outside its array,
 * a negative position above all, is skipped: neither its keys and values nor
 * its q_out are written.  Two tokens of one call with one place leave there, value
 * by value, one of the two.  tokens == 0 returns NMSPMM_OK without a launch.  Errors:
 * NMSPMM_ERR_INVALID_ARG (negative size, bad type, odd rot or rot > dim, null
 * pointer with non-empty data), NMSPMM_ERR_UNSUPPORTED (misaligned pointer,
 * dim > 512, more than 2^31 - 1 positions, 2^24 tokens or more, more than 2^24 -
 * 256 pairs of dimensions a token, keys, values and queries together),
 * NMSPMM_ERR_HIP. */
NMSPMM_API nmspmm_status_t nmspmm_kv_append(const nmspmm_kv_cache_t *cache, const void *k_new, const int64_t *k_stride,
                                 const void *v_new, const int64_t *v_stride, nmspmm_dtype_t dtype,
                                 int64_t tokens, const int32_t *seq, const int32_t *pos, const float *cos,
                                 const float *sin, int64_t positions, int rot, int interleaved, const void *q,
                                 const int64_t *q_stride, void *q_out, const int64_t *q_out_stride,
                                 int64_t q_heads, hipStream_t stream);

/* Bytes of workspace with which nmspmm_kv_attend splits the sequences of this
 * cache: 0 where it does not, -1 for bad sizes.  Host only. */
NMSPMM_API int64_t nmspmm_kv_attend_workspace_bytes(const nmspmm_kv_cache_t *cache, int64_t q_heads,
                                         int64_t max_length, int64_t window);

/* Attention of one new token per sequence over the cache.  Query head h of
 * sequence s reads the cache's head h / (q_heads / heads):
 *   out[s][h] = sum_p softmax_p(scale * <q[s][h], k[p]>) v[p],
 *   p from max(0, lengths[s] - window) (0 with window = 0) to lengths[s] - 1
 *   q, out   sequences x q_heads x dim of `dtype`; element (s, h, d) at
 *            s*stride[0] + h*stride[1] + d; out may not overlap q
 *   lengths  one per sequence; it counts the new token, whose key and value
 *            are in the cache.  A length <= 0 leaves no position: that row of
 *            out is zero and its lse minus infinity.
 *   max_length  an upper bound of the lengths, known to the host, which sets
 *            how the work is split; a length beyond it, beyond the table or
 *            beyond 2^31 - 4097 is taken as the smallest of these
 *   lse      sequences x q_heads fp32, the natural logarithm of the softmax's
 *            denominator (to join results over parts of a context), or NULL
 * A position whose page lies outside the cache is left out.  Positions outside
 * the range are not read into any sum: what their slots hold (NaN, say) does
 * not matter.  An infinity inside it makes the sums it enters infinite or NaN,
 * but a row whose scores are all minus infinity is zero and its lse minus
 * infinity, as if there were no position.  Scores, softmax and sums are fp32
 * (beside 16-bit values a weight enters in 16-bit parts that hold its bits); out is
 * rounded once.  The order of summation is fixed by shapes, lengths and workspace.  No sequences
 * or no query heads: NMSPMM_OK without a launch.  Errors:
 * NMSPMM_ERR_INVALID_ARG (negative size, bad type, q_heads no multiple of
 * heads, null pointer with non-empty data), NMSPMM_ERR_UNSUPPORTED
 * (misaligned pointer, dim > 512, sizes beyond 2^31 - 1, 2^24 query rows or
 * more), NMSPMM_ERR_HIP. */
NMSPMM_API nmspmm_status_t nmspmm_kv_attend(const nmspmm_kv_cache_t *cache, const void *q, const int64_t *q_stride,
                                 nmspmm_dtype_t dtype, int64_t q_heads, const int32_t *lengths,
                                 int64_t max_length, int64_t window, float scale, void *out,
                                 const int64_t *out_stride, float *lse, void *workspace, size_t workspace_bytes,
                                 hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* NMSPMM_SERVE_H */
