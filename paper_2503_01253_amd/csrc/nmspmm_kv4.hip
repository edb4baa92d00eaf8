// The paged cache in 4 bits: its checks, nmspmm_kv4_read and nmspmm_kv4_attend
// (nmspmm_kv_norm.hip writes it).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nmspmm_kv4.h"
#include "nmspmm_kv_host.h"
#include "nmspmm_workspace.h"

namespace nmspmm {

nmspmm_kv_cache_t kv4_sizes(const nmspmm_kv4_cache_t *c)
{
    nmspmm_kv_cache_t s{};
    s.pages = c->page_count;
    s.table = c->table;
    s.table_stride = c->table_stride;
    s.sequences = c->sequences;
    s.table_pages = c->table_pages;
    s.page_size = c->page_size;
    s.heads = c->heads;
    s.dim = c->dim;
    s.dtype = NMSPMM_BF16;
    return s;
}

nmspmm_status_t check_kv4(const nmspmm_kv4_cache_t *c)
{
    if (!c) return NMSPMM_ERR_INVALID_ARG;
    const nmspmm_kv_cache_t sizes = kv4_sizes(c);
    const nmspmm_status_t st = check_cache(&sizes);
    if (st != NMSPMM_OK) return st;
    const int64_t bytes = nmspmm_kv4_page_bytes(c->page_size, c->heads, c->dim);
    if (bytes < 0) return NMSPMM_ERR_UNSUPPORTED;
    if (c->page_stride < bytes && c->page_count > 1) return NMSPMM_ERR_INVALID_ARG;
    return c->page_stride % 16 ? NMSPMM_ERR_UNSUPPORTED : NMSPMM_OK;
}

nmspmm_status_t check_kv4_pointers(const nmspmm_kv4_cache_t *c)
{
    if (c->page_count > 0 && !c->pages) return NMSPMM_ERR_INVALID_ARG;
    if (c->sequences > 0 && c->table_pages > 0 && !c->table) return NMSPMM_ERR_INVALID_ARG;
    return aligned_to(c->pages, 16) && aligned_to(c->table, 4) ? NMSPMM_OK : NMSPMM_ERR_UNSUPPORTED;
}

Kv4Pages kv4_view(const nmspmm_kv4_cache_t *c)
{
    return {static_cast<unsigned char *>(c->pages), c->page_stride, kv4_layout(c->page_size, c->dim)};
}

namespace {

// ---- nmspmm_kv4_read -------------------------------------------------------

struct ReadArgs {
    Pages c;
    Kv4Pages f;
    void *k_out, *v_out;
    int64_t ks[2], vs[2];
    const int32_t *seq, *pos;
    int64_t tokens, sequences, table_positions;
    int32_t heads, dim, words, items;
};

constexpr int RD_NT = 256;

// A word of eight codes a thread: a row's words side by side, keys before
// values.  VEC: rows of the outputs in whole 16-byte pieces.
template <class T, bool VEC>
__global__ __launch_bounds__(RD_NT) void nm_kv4_read_kernel(ReadArgs p)
{
    const int64_t t = blockIdx.x;
    const int item = blockIdx.y * RD_NT + threadIdx.x;
    if (item >= p.items) return;
    const int64_t pos = p.pos[t], seq = p.seq[t];
    if (pos < 0 || pos >= p.table_positions || seq < 0 || seq >= p.sequences) return;
    const Place at = place_of(p.c, p.c.table + seq * p.c.table_stride, (int)pos);
    if (!at.held) return;
    const int row = item / p.words, D = item - row * p.words;
    const bool is_k = row < p.heads;
    const int head = is_k ? row : row - p.heads;
    void *out = is_k ? p.k_out : p.v_out;
    if (!out) return;
    const Kv4Layout &l = p.f.l;
    const unsigned char *b = p.f.block(at.page, head);
    const uint32_t w = *reinterpret_cast<const uint32_t *>(b + (is_k ? l.k_word(at.slot, D) : l.v_word(at.slot, D)));
    float x[8];
    mx4_values(w, b[is_k ? l.k_scale(at.slot, D / 4) : l.v_scale(at.slot, D / 4)], x);
    const int64_t dst = is_k ? t * p.ks[0] + head * p.ks[1] : t * p.vs[0] + head * p.vs[1];
    store_row<8, VEC>(static_cast<T *>(out) + dst + D * 8, p.dim - D * 8, x);
}

template <class T>
hipError_t launch_read(const ReadArgs &p, bool vec, hipStream_t stream)
{
    const dim3 grid((unsigned)p.tokens, (unsigned)((p.items + RD_NT - 1) / RD_NT));
    if (vec) hipLaunchKernelGGL((nm_kv4_read_kernel<T, true>), grid, dim3(RD_NT), 0, stream, p);
    else hipLaunchKernelGGL((nm_kv4_read_kernel<T, false>), grid, dim3(RD_NT), 0, stream, p);
    return hipGetLastError();
}

// ---- nmspmm_kv4_attend -----------------------------------------------------

constexpr int A4_NW = 4, A4_NT = 64 * A4_NW;

// The attention of GT query heads that share one cache head, over one chunk of
// a sequence, on the vector ALU, for any page size and up to 512 dimensions:
// LPT lanes hold a token's row, a word of eight codes each.  As the kernel of
// the 16-bit cache (nm_attend_kernel), every team of LPT lanes keeps its own
// running maximum, sum and sums of values, joined at the end.
template <int LPT, int GT>
__global__ __launch_bounds__(A4_NT) void nm_attend4_kernel(AttendArgs p, Kv4Pages f)
{
    constexpr int TPW = 64 / LPT, U = 4;
    __shared__ float s_acc[A4_NW][GT][LPT * 8];
    __shared__ float2 s_ml[A4_NW][GT];
    const AttendTask t = attend_task(p, blockIdx.x, GT);
    if (t.begin >= t.end && p.splits > 1) {      // nothing here: the maximum says so
        if (threadIdx.x < t.heads_in_tile) {
            const int64_t row = t.seq * ((int64_t)p.heads * p.group) + t.first_head + threadIdx.x;
            p.part_ml[row * p.splits + t.split] = make_float2(NEG_INF, 0.f);
        }
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int grp = lane / LPT, D = lane % LPT, d0 = D * 8;
    const bool mine = D < 4 * f.l.G;

    float q[GT][8], acc[GT][8], m[GT], l[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
        m[g] = NEG_INF;
        l[g] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            q[g][i] = acc[g][i] = 0.f;
            if (g < t.heads_in_tile && d0 + i < p.dim) {
                const int64_t at = t.seq * p.qs[0] + (t.first_head + g) * p.qs[1] + d0 + i;
                q[g][i] = p.io == NMSPMM_F32    ? static_cast<const float *>(p.q)[at]
                          : p.io == NMSPMM_BF16 ? to_f32(static_cast<const bf16_t *>(p.q)[at])
                                                : to_f32(static_cast<const f16_t *>(p.q)[at]);
                q[g][i] *= p.scale2;
            }
        }
    }
    const int32_t *row = p.c.table + t.seq * p.c.table_stride;
    for (int base = t.begin + wave * (TPW * U); base < t.end; base += A4_NW * TPW * U) {
        float k[U][8], v[U][8];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pos = base + u * TPW + grp;
            in[u] = pos < t.end;
            Place at{0, 0, false};
            if (in[u]) at = place_of(p.c, row, pos);
            in[u] = in[u] && at.held;
            uint32_t kw = 0, vw = 0, ks = 127, vs = 127;    // zeros
            if (in[u] && mine) {
                const unsigned char *b = f.block(at.page, t.head);
                kw = *reinterpret_cast<const uint32_t *>(b + f.l.k_word(at.slot, D));
                vw = *reinterpret_cast<const uint32_t *>(b + f.l.v_word(at.slot, D));
                ks = b[f.l.k_scale(at.slot, D / 4)];
                vs = b[f.l.v_scale(at.slot, D / 4)];
            }
            mx4_values(kw, ks, k[u]);
            mx4_values(vw, vs, v[u]);
        }
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            float s[U], top = m[g];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) x = fmaf(q[g][i], k[u][i], x);
                x = lanes_sum<LPT>(x);
                s[u] = in[u] ? x : NEG_INF;
                top = fmaxf(top, s[u]);
            }
            const float ref = softmax_ref(top), corr = exp2f(m[g] - ref);
            m[g] = top;
            l[g] *= corr;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[g][i] *= corr;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float w = exp2f(s[u] - ref);
                l[g] += w;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[g][i] = fmaf(w, v[u][i], acc[g][i]);
            }
        }
    }
    // join the wave's teams, then the waves
#pragma unroll
    for (int g = 0; g < GT; ++g) {
#pragma unroll
        for (int step = LPT; step < 64; step *= 2) {
            const float om = __shfl_xor(m[g], step), ol = __shfl_xor(l[g], step);
            const float top = fmaxf(m[g], om), ref = softmax_ref(top);
            const float here = exp2f(m[g] - ref), there = exp2f(om - ref);
            m[g] = top;
            l[g] = l[g] * here + ol * there;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[g][i] = acc[g][i] * here + __shfl_xor(acc[g][i], step) * there;
        }
        if (grp == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s_acc[wave][g][d0 + i] = acc[g][i];
            if (lane == 0) s_ml[wave][g] = make_float2(m[g], l[g]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < t.heads_in_tile * p.dim; i += A4_NT) {
        const int g = i / p.dim, d = i % p.dim;
        float top = NEG_INF, x = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < A4_NW; ++w) top = fmaxf(top, s_ml[w][g].x);
        const float ref = softmax_ref(top);
#pragma unroll
        for (int w = 0; w < A4_NW; ++w) {
            const float c = exp2f(s_ml[w][g].x - ref);
            x += c * s_acc[w][g][d];
            sum += c * s_ml[w][g].y;
        }
        attend_store(p, t, t.first_head + g, d, x, top, sum);
    }
}

template <int LPT>
void launch_attend4_heads(const AttendArgs &p, const Kv4Pages &f, int GT, unsigned groups, hipStream_t stream)
{
    const dim3 grid(groups), block(A4_NT);
    if (GT == 1) hipLaunchKernelGGL((nm_attend4_kernel<LPT, 1>), grid, block, 0, stream, p, f);
    else if (GT == 2) hipLaunchKernelGGL((nm_attend4_kernel<LPT, 2>), grid, block, 0, stream, p, f);
    else if (GT == 4) hipLaunchKernelGGL((nm_attend4_kernel<LPT, 4>), grid, block, 0, stream, p, f);
    else hipLaunchKernelGGL((nm_attend4_kernel<LPT, 8>), grid, block, 0, stream, p, f);
}

void launch_attend4(const AttendArgs &p, const Kv4Pages &f, int GT, unsigned groups, hipStream_t stream)
{
    if (p.dim <= 128) launch_attend4_heads<16>(p, f, GT, groups, stream);
    else if (p.dim <= 256) launch_attend4_heads<32>(p, f, GT, groups, stream);
    else launch_attend4_heads<64>(p, f, GT, groups, stream);
}

// Whether the matrix-core kernel takes the cache.
bool attend4_takes_mfma(const nmspmm_kv4_cache_t *c)
{
    return c->page_size % 4 == 0 && c->dim <= 256 && kv4_layout(c->page_size, c->dim).block < (int64_t)1 << 31;
}

// How the work is cut.  For the matrix-core kernel, of which a CU holds four
// workgroups with bf16 queries, pages of 16 and up to 128 dimensions (three to one in
// its other forms, which are cut alike): into what runs at once, where that leaves chunks of 256 to 2048
// positions (one sequence of 131071 on 8 heads 37.5 us, in twice as many chunks 43);
// else into quarters of the longest, 1024 to 2048 positions each, for batches whose
// lengths differ (48 sequences of 0 to 5000, in chunks of 1792, 1280 and 640: 42.3,
// 37.5 and 40 us; 128 of 8192, in chunks of 2048, 1408 and 1024: 218, 225 and 233).
AttendPlan attend4_plan(const nmspmm_kv4_cache_t *c, int64_t q_heads, int64_t max_length, int64_t window, bool split)
{
    const nmspmm_kv_cache_t sizes = kv4_sizes(c);
    if (!attend4_takes_mfma(c)) return attend_plan(&sizes, q_heads, max_length, window, false, split);
    const int64_t span = attend_span(&sizes, max_length, window);
    const int64_t base = c->sequences * c->heads * ((q_heads / c->heads + ATTEND_MFMA_HEADS - 1) / ATTEND_MFMA_HEADS);
    int64_t splits = 1;
    if (split && base > 0) {
        splits = 1024 / base;
        if (splits == 0 || span > 2048 * splits) {
            const int64_t most = std::max<int64_t>(1024, std::min<int64_t>(2048, (span / 4 + 127) / 128 * 128));
            // (up to 64 workgroups a CU, which bounds the workspace)
            splits = std::max<int64_t>(1, std::min<int64_t>({JN_SPLITS, (span + most - 1) / most, 16384 / base}));
        } else {
            splits = std::max<int64_t>(1, std::min(splits, span / 256));
        }
    }
    return attend_cut(&sizes, q_heads, span, ATTEND_MFMA_HEADS, splits);
}

nmspmm_status_t check_attend4_sizes(const nmspmm_kv4_cache_t *c, int64_t q_heads, int64_t max_length, int64_t window)
{
    const nmspmm_status_t st = check_kv4(c);
    if (st != NMSPMM_OK) return st;
    const nmspmm_kv_cache_t sizes = kv4_sizes(c);
    return check_attend_sizes(&sizes, q_heads, max_length, window);
}

}  // namespace
}  // namespace nmspmm

using namespace nmspmm;

extern "C" int64_t nmspmm_kv4_page_bytes(int64_t page_size, int64_t heads, int64_t dim)
{
    if (page_size < 1 || heads < 1 || dim < 1 || dim > KV_MAX_DIM || page_size > INT31 || heads > INT31) return -1;
    const int64_t block = kv4_layout(page_size, dim).block;
    return block > (((int64_t)1 << 62) / heads) ? -1 : block * heads;
}

extern "C" nmspmm_status_t nmspmm_kv4_read(const nmspmm_kv4_cache_t *cache, int64_t tokens, const int32_t *seq,
                                           const int32_t *pos, nmspmm_dtype_t dtype, void *k_out,
                                           const int64_t *k_stride, void *v_out, const int64_t *v_stride,
                                           hipStream_t stream)
{
    nmspmm_status_t st = check_kv4(cache);
    if (st != NMSPMM_OK) return st;
    if (!dtype_ok(dtype) || tokens < 0) return NMSPMM_ERR_INVALID_ARG;
    if (tokens == 0 || (!k_out && !v_out)) return NMSPMM_OK;
    st = check_kv4_pointers(cache);
    if (st != NMSPMM_OK) return st;
    if (!seq || !pos || (k_out && !k_stride) || (v_out && !v_stride)) return NMSPMM_ERR_INVALID_ARG;
    const int es = dtype_bytes(dtype);
    if (!aligned_to(k_out, es) || !aligned_to(v_out, es) || !aligned_to(seq, 4) || !aligned_to(pos, 4))
        return NMSPMM_ERR_UNSUPPORTED;
    const int words = (cache->dim + 7) / 8;
    // a launch takes fewer than 2^32 threads along x and 2^16 workgroups along y
    if (tokens >= (int64_t)1 << 24 || 2 * (int64_t)cache->heads * words > (int64_t)65535 * RD_NT)
        return NMSPMM_ERR_UNSUPPORTED;
    const nmspmm_kv_cache_t sizes = kv4_sizes(cache);
    ReadArgs p{};
    p.c = device_view(&sizes);
    p.f = kv4_view(cache);
    p.k_out = k_out;
    p.v_out = v_out;
    for (int i = 0; i < 2; ++i) {
        p.ks[i] = k_out ? k_stride[i] : 0;
        p.vs[i] = v_out ? v_stride[i] : 0;
    }
    p.seq = seq;
    p.pos = pos;
    p.tokens = tokens;
    p.sequences = cache->sequences;
    p.table_positions = table_positions(&sizes);
    p.heads = cache->heads;
    p.dim = cache->dim;
    p.words = words;
    p.items = 2 * cache->heads * words;
    const bool vec = cache->dim % 8 == 0 && (!k_out || rows_aligned(k_out, k_stride, 2, cache->dim, es)) &&
                     (!v_out || rows_aligned(v_out, v_stride, 2, cache->dim, es));
    const hipError_t e = dtype == NMSPMM_F32    ? launch_read<float>(p, vec, stream)
                         : dtype == NMSPMM_BF16 ? launch_read<bf16_t>(p, vec, stream)
                                                : launch_read<f16_t>(p, vec, stream);
    return e == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" int64_t nmspmm_kv4_attend_workspace_bytes(const nmspmm_kv4_cache_t *cache, int64_t q_heads,
                                                     int64_t max_length, int64_t window)
{
    if (check_attend4_sizes(cache, q_heads, max_length, window) != NMSPMM_OK) return -1;
    if (q_heads == 0 || cache->sequences == 0) return 0;
    return attend4_plan(cache, q_heads, max_length, window, true).bytes;
}

extern "C" nmspmm_status_t nmspmm_kv4_attend(const nmspmm_kv4_cache_t *cache, const void *q, const int64_t *q_stride,
                                             nmspmm_dtype_t dtype, int64_t q_heads, const int32_t *lengths,
                                             int64_t max_length, int64_t window, float scale, void *out,
                                             const int64_t *out_stride, float *lse, void *workspace,
                                             size_t workspace_bytes, hipStream_t stream)
{
    nmspmm_status_t st = check_attend4_sizes(cache, q_heads, max_length, window);
    if (st != NMSPMM_OK) return st;
    if (!dtype_ok(dtype)) return NMSPMM_ERR_INVALID_ARG;
    if (q_heads == 0 || cache->sequences == 0) return NMSPMM_OK;
    st = check_kv4_pointers(cache);
    if (st != NMSPMM_OK) return st;
    if (!q || !q_stride || !out || !out_stride || !lengths) return NMSPMM_ERR_INVALID_ARG;
    const int es = dtype_bytes(dtype);
    if (!aligned_to(q, es) || !aligned_to(out, es) || !aligned_to(lengths, 4) || !aligned_to(lse, 4) ||
        !aligned_to(workspace, 256))
        return NMSPMM_ERR_UNSUPPORTED;
    const nmspmm_kv_cache_t sizes = kv4_sizes(cache);
    int cached = -1;
    const bool mfma = attend4_takes_mfma(cache);
    AttendPlan a = attend4_plan(cache, q_heads, max_length, window, true);
    if (a.bytes > 0 && (!workspace || (uint64_t)a.bytes > (uint64_t)workspace_bytes)) {
        workspace = capturing(stream) ? nullptr : ws_acquire(stream, (size_t)a.bytes, &cached);
        if (!workspace) a = attend4_plan(cache, q_heads, max_length, window, false);
    }
    AttendArgs p{};
    p.c = device_view(&sizes);
    p.q = q;
    p.out = out;
    p.lse = lse;
    p.part_ml = static_cast<float2 *>(workspace);
    p.part_acc = reinterpret_cast<float *>(static_cast<char *>(workspace) + a.ml_bytes);
    p.lengths = lengths;
    for (int i = 0; i < 2; ++i) {
        p.qs[i] = q_stride[i];
        p.os[i] = out_stride[i];
    }
    p.cap = (int)std::min({max_length, table_positions(&sizes), KV_MAX_LENGTH});
    p.window = (int)std::min(window, INT31);
    p.heads = cache->heads;
    p.group = (int)(q_heads / cache->heads);
    p.gtiles = a.gtiles;
    p.dim = cache->dim;
    p.splits = a.splits;
    p.chunk = a.chunk;
    p.scale2 = scale * 1.44269504089f;
    p.io = dtype;
    p.q_vec = rows_aligned(q, q_stride, 2, cache->dim, es);
    const Kv4Pages f = kv4_view(cache);
    if (mfma) launch_attend4_mfma(p, f, cache->page_size, (unsigned)a.groups, stream);
    else launch_attend4(p, f, a.GT, (unsigned)a.groups, stream);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        launch_join(p, a.rows, stream);
        e = hipGetLastError();
    }
    const hipError_t g = cached >= 0 ? ws_done(cached, stream) : hipSuccess;
    return e == hipSuccess && g == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}
