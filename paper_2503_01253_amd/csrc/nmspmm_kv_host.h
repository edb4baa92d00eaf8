// Host code shared by the units of the paged caches: checks of their
// arguments, and how an attention call is cut and joined.
#ifndef NMSPMM_KV_HOST_H
#define NMSPMM_KV_HOST_H

#include <algorithm>
#include <cstdint>

#include "nmspmm_kv.h"

namespace nmspmm {

inline bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t INT31 = 0x7fffffff;
constexpr int KV_MAX_DIM = 512;
constexpr int64_t KV_MAX_LENGTH = INT31 - 4096;     // the kernels step a few hundred positions past the last

inline nmspmm_status_t check_cache(const nmspmm_kv_cache_t *c)
{
    if (!c || c->pages < 0 || c->sequences < 0 || c->table_pages < 0 || c->page_size < 1 || c->heads < 1 ||
        c->dim < 1 || !dtype_ok(c->dtype))
        return NMSPMM_ERR_INVALID_ARG;
    if (c->dim > KV_MAX_DIM || c->sequences > INT31 || c->pages > INT31 || c->table_pages > INT31)
        return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

inline nmspmm_status_t check_cache_pointers(const nmspmm_kv_cache_t *c)
{
    if (c->pages > 0 && (!c->k_pages || !c->v_pages)) return NMSPMM_ERR_INVALID_ARG;
    if (c->sequences > 0 && c->table_pages > 0 && !c->table) return NMSPMM_ERR_INVALID_ARG;
    const int es = dtype_bytes(c->dtype);
    if (!aligned_to(c->k_pages, es) || !aligned_to(c->v_pages, es) || !aligned_to(c->table, 4))
        return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

inline Pages device_view(const nmspmm_kv_cache_t *c)
{
    Pages p;
    p.table = c->table;
    p.table_stride = c->table_stride;
    p.pages = c->pages;
    for (int i = 0; i < 3; ++i) {
        p.ks[i] = c->k_stride[i];
        p.vs[i] = c->v_stride[i];
    }
    p.size = fast_div((uint32_t)c->page_size);
    return p;
}

// Positions that the table can name, at most 2^31 - 1.
inline int64_t table_positions(const nmspmm_kv_cache_t *c) { return std::min(INT31, c->table_pages * c->page_size); }

// Whether rows of `dim` elements of `bytes` bytes at these strides all start
// on 16 bytes and hold whole 16-byte pieces.
inline bool rows_aligned(const void *p, const int64_t *stride, int count, int dim, int bytes)
{
    if (!aligned_to(p, 16) || dim * bytes % 16) return false;
    for (int i = 0; i < count; ++i)
        if (stride[i] * bytes % 16) return false;
    return true;
}

// How the work is cut: query heads a workgroup takes together, workgroups
// along a sequence and the positions of each.
struct AttendPlan {
    int GT, gtiles, splits, chunk;
    int64_t groups;             // workgroups
    int64_t rows;               // sequences x query heads
    int64_t ml_bytes, bytes;    // workspace
};

// nmspmm_kv.hip.  mfma: tiles of 16 query heads; split: sequences may be cut.
AttendPlan attend_plan(const nmspmm_kv_cache_t *c, int64_t q_heads, int64_t max_length, int64_t window, bool mfma,
                       bool split);

// The positions of a sequence that a call may attend to, at most.
inline int64_t attend_span(const nmspmm_kv_cache_t *c, int64_t max_length, int64_t window)
{
    const int64_t span = std::min({max_length, table_positions(c), KV_MAX_LENGTH});
    return window > 0 ? std::min(span, window) : span;
}

// The plan with tiles of GT heads and about `splits` chunks of whole 128 positions.
inline AttendPlan attend_cut(const nmspmm_kv_cache_t *c, int64_t q_heads, int64_t span, int GT, int64_t splits)
{
    AttendPlan a{};
    a.GT = GT;
    a.gtiles = (int)((q_heads / c->heads + GT - 1) / GT);
    a.chunk = (int)std::max<int64_t>(128, ((span + splits - 1) / splits + 127) / 128 * 128);
    a.splits = (int)std::max<int64_t>(1, (span + a.chunk - 1) / a.chunk);     // 1 where splits is
    a.groups = c->sequences * c->heads * a.gtiles * a.splits;
    a.rows = c->sequences * q_heads;
    if (a.splits > 1) {
        a.ml_bytes = (a.rows * a.splits * 8 + 255) / 256 * 256;
        a.bytes = a.ml_bytes + a.rows * a.splits * c->dim * 4;
    }
    return a;
}

nmspmm_status_t check_attend_sizes(const nmspmm_kv_cache_t *c, int64_t q_heads, int64_t max_length, int64_t window);
constexpr int JN_SPLITS = 2048;     // most chunks of a sequence
void launch_join(const AttendArgs &p, int64_t rows, hipStream_t stream);     // the parts of split sequences joined

}  // namespace nmspmm

#endif
