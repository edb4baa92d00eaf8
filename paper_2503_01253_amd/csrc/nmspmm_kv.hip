// The paged key-value cache behind nmspmm_kv_append and nmspmm_kv_attend.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nmspmm_kv.h"
#include "nmspmm_workspace.h"

namespace nmspmm {
namespace {

bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t INT31 = 0x7fffffff;
constexpr int KV_MAX_DIM = 512;
constexpr int64_t KV_MAX_LENGTH = INT31 - 4096;     // the kernels step a few hundred positions past the last

nmspmm_status_t check_cache(const nmspmm_kv_cache_t *c)
{
    if (!c || c->pages < 0 || c->sequences < 0 || c->table_pages < 0 || c->page_size < 1 || c->heads < 1 ||
        c->dim < 1 || !dtype_ok(c->dtype))
        return NMSPMM_ERR_INVALID_ARG;
    if (c->dim > KV_MAX_DIM || c->sequences > INT31 || c->pages > INT31 || c->table_pages > INT31)
        return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

nmspmm_status_t check_cache_pointers(const nmspmm_kv_cache_t *c)
{
    if (c->pages > 0 && (!c->k_pages || !c->v_pages)) return NMSPMM_ERR_INVALID_ARG;
    if (c->sequences > 0 && c->table_pages > 0 && !c->table) return NMSPMM_ERR_INVALID_ARG;
    const int es = dtype_bytes(c->dtype);
    if (!aligned_to(c->k_pages, es) || !aligned_to(c->v_pages, es) || !aligned_to(c->table, 4))
        return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

Pages device_view(const nmspmm_kv_cache_t *c)
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
int64_t table_positions(const nmspmm_kv_cache_t *c) { return std::min(INT31, c->table_pages * c->page_size); }

// Whether rows of `dim` elements of `bytes` bytes at these strides all start
// on 16 bytes and hold whole 16-byte pieces.
bool rows_aligned(const void *p, const int64_t *stride, int count, int dim, int bytes)
{
    if (!aligned_to(p, 16) || dim * bytes % 16) return false;
    for (int i = 0; i < count; ++i)
        if (stride[i] * bytes % 16) return false;
    return true;
}

// ---- nmspmm_kv_append ------------------------------------------------------

struct AppendArgs {
    Pages c;
    const void *k_new, *v_new, *q;
    void *k_pages, *v_pages, *q_out;
    int64_t kn[2], vn[2], qn[2], qo[2];
    const int32_t *seq, *pos;
    const float *cos, *sin;
    int64_t tokens, positions, sequences, table_positions;
    int32_t heads, q_heads, dim, rot, interleaved, items;
};

constexpr int AP_NT = 256;

// (a, b) turned by the angle of cos c and sin s.  Spelled with fused
// multiply-adds whose fp32 results are kept (fp16's rounding is not fused into
// them), so that every kernel rounds alike.
__device__ __forceinline__ void turn_pair(float &a, float &b, float c, float s)
{
    float x = fmaf(a, c, -(b * s)), y = fmaf(a, s, b * c);
#ifdef __HIP_DEVICE_COMPILE__
    asm("" : "+v"(x), "+v"(y));
#endif
    a = x;
    b = y;
}

// Every (token, row, dimension pair) by one thread: a row is a key, a value
// or a query head; a pair is two dimensions that turn together, or (beyond
// rot, and in values) two neighbours that are copied.  Elementwise, bound by
// memory and, for few tokens, by the chain pos -> table -> store.
template <class T, class C>
__global__ __launch_bounds__(AP_NT) void nm_append_kernel(AppendArgs p)
{
    const int64_t t = blockIdx.x;
    const int item = blockIdx.y * AP_NT + threadIdx.x;
    if (item >= p.items) return;
    const int64_t pos = p.pos[t], seq = p.seq[t];
    if (pos < 0 || pos >= p.table_positions || seq < 0 || seq >= p.sequences || (p.rot && pos >= p.positions)) return;
    const Place at = place_of(p.c, p.c.table + seq * p.c.table_stride, (int)pos);
    if (!at.held) return;
    const int pairs = (p.dim + 1) / 2;
    const int row = item / pairs, e = item % pairs;
    const bool is_k = row < p.heads, is_v = !is_k && row < 2 * p.heads;
    const int head = is_k ? row : is_v ? row - p.heads : row - 2 * p.heads;
    const int half = p.rot / 2;
    // the pair's dimensions; the second may lie past an odd row's end
    const bool turn = !is_v && e < half;
    const int d0 = turn && !p.interleaved ? e : 2 * e;
    const int d1 = turn && !p.interleaved ? e + half : 2 * e + 1;
    const T *src = is_k ? static_cast<const T *>(p.k_new) + t * p.kn[0] + head * p.kn[1]
                 : is_v ? static_cast<const T *>(p.v_new) + t * p.vn[0] + head * p.vn[1]
                        : static_cast<const T *>(p.q) + t * p.qn[0] + head * p.qn[1];
    float a = to_f32(src[d0]), b = d1 < p.dim ? to_f32(src[d1]) : 0.f;
    if (turn) {
        turn_pair(a, b, p.cos[pos * half + e], p.sin[pos * half + e]);
    }
    if (is_k || is_v) {
        C *dst = is_k ? static_cast<C *>(p.k_pages) + at.page * p.c.ks[0] + at.slot * p.c.ks[1] + head * p.c.ks[2]
                      : static_cast<C *>(p.v_pages) + at.page * p.c.vs[0] + at.slot * p.c.vs[1] + head * p.c.vs[2];
        dst[d0] = from_f32<C>(a);
        if (d1 < p.dim) dst[d1] = from_f32<C>(b);
    } else {
        T *dst = static_cast<T *>(p.q_out) + t * p.qo[0] + head * p.qo[1];
        dst[d0] = from_f32<T>(a);
        if (d1 < p.dim) dst[d1] = from_f32<T>(b);
    }
}

constexpr int AV_NT = 128;

// The same with eight pairs a thread, where every row holds whole 16-byte
// pieces of eight dimensions and rot/2 is a multiple of 8: 16-byte accesses.
// What does not depend on the position is asked for before anything is waited
// for (64 tokens of 48 rows of 128: 11.4 us with one pair a thread and the
// loads behind the checks).  4001 tokens of 48 fp32 rows take 37 us, 4.9 TB/s.
template <class T, class C>
__global__ __launch_bounds__(AV_NT) void nm_append_vec_kernel(AppendArgs p)
{
    const int64_t t = blockIdx.x;
    const int item = blockIdx.y * AV_NT + threadIdx.x;
    if (item >= p.items) return;
    const int64_t pos = p.pos[t], seq = p.seq[t];
    const int pieces = p.dim / 16, row = item / pieces, e = item - row * pieces;
    const bool is_k = row < p.heads, is_v = !is_k && row < 2 * p.heads;
    const int head = is_k ? row : is_v ? row - p.heads : row - 2 * p.heads;
    const int half = p.rot / 2;
    const bool turn = !is_v && e * 8 < half, apart = turn && !p.interleaved;
    const int d0 = apart ? e * 8 : e * 16, d1 = apart ? d0 + half : d0 + 8;
    const T *src = is_k ? static_cast<const T *>(p.k_new) + t * p.kn[0] + head * p.kn[1]
                 : is_v ? static_cast<const T *>(p.v_new) + t * p.vn[0] + head * p.vn[1]
                        : static_cast<const T *>(p.q) + t * p.qn[0] + head * p.qn[1];
    float a[8], b[8];
    load_row<8, true>(src + d0, 8, a);
    load_row<8, true>(src + d1, 8, b);
    if (pos < 0 || pos >= p.table_positions || seq < 0 || seq >= p.sequences || (p.rot && pos >= p.positions)) return;
    const Place at = place_of(p.c, p.c.table + seq * p.c.table_stride, (int)pos);
    if (turn) {
        float c[8], s[8];
        load_row<8, true>(p.cos + pos * half + e * 8, 8, c);
        load_row<8, true>(p.sin + pos * half + e * 8, 8, s);
        if (apart) {
#pragma unroll
            for (int i = 0; i < 8; ++i) turn_pair(a[i], b[i], c[i], s[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                turn_pair(a[2 * i], a[2 * i + 1], c[i], s[i]);
                turn_pair(b[2 * i], b[2 * i + 1], c[4 + i], s[4 + i]);
            }
        }
    }
    if (!at.held) return;
    if (is_k || is_v) {
        C *dst = is_k ? static_cast<C *>(p.k_pages) + at.page * p.c.ks[0] + at.slot * p.c.ks[1] + head * p.c.ks[2]
                      : static_cast<C *>(p.v_pages) + at.page * p.c.vs[0] + at.slot * p.c.vs[1] + head * p.c.vs[2];
        store_row<8, true>(dst + d0, 8, a);
        store_row<8, true>(dst + d1, 8, b);
    } else {
        T *dst = static_cast<T *>(p.q_out) + t * p.qo[0] + head * p.qo[1];
        store_row<8, true>(dst + d0, 8, a);
        store_row<8, true>(dst + d1, 8, b);
    }
}

template <class T, class C>
hipError_t launch_append_to(AppendArgs p, bool vec, hipStream_t stream)
{
    const int rows = 2 * p.heads + p.q_heads;
    p.items = rows * (vec ? p.dim / 16 : (p.dim + 1) / 2);
    const int threads = vec ? AV_NT : AP_NT;
    const dim3 grid((unsigned)p.tokens, (unsigned)((p.items + threads - 1) / threads));
    if (vec) hipLaunchKernelGGL((nm_append_vec_kernel<T, C>), grid, dim3(AV_NT), 0, stream, p);
    else hipLaunchKernelGGL((nm_append_kernel<T, C>), grid, dim3(AP_NT), 0, stream, p);
    return hipGetLastError();
}

template <class T>
hipError_t launch_append(const AppendArgs &p, nmspmm_dtype_t cache, bool vec, hipStream_t stream)
{
    if (cache == NMSPMM_F32) return launch_append_to<T, float>(p, vec, stream);
    return cache == NMSPMM_BF16 ? launch_append_to<T, bf16_t>(p, vec, stream) : launch_append_to<T, f16_t>(p, vec, stream);
}

// ---- nmspmm_kv_attend ------------------------------------------------------

constexpr int AT_NW = 4, AT_NT = 64 * AT_NW;

template <int LPT>
__device__ __forceinline__ float lanes_sum(float x)
{
    auto dpp = [](float v, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value,
                                                                     0xf, 0xf, false));
    };
    x += dpp(x, std::integral_constant<int, 0xb1>{});                          // lane ^ 1
    x += dpp(x, std::integral_constant<int, 0x4e>{});                          // lane ^ 2
    if constexpr (LPT >= 8) x += dpp(x, std::integral_constant<int, 0x141>{});  // the other four of eight
    if constexpr (LPT >= 16) x += dpp(x, std::integral_constant<int, 0x140>{}); // the other eight of sixteen
    if constexpr (LPT >= 32) x += __shfl_xor(x, 16);
    if constexpr (LPT >= 64) x += __shfl_xor(x, 32);
    return x;
}

// The attention of GT query heads that share one cache head, over one chunk
// of a sequence, on the vector ALU: LPT lanes hold a token's row, EPL
// elements each, so that a wave reads 64/LPT tokens with one load.  Each
// group of LPT lanes keeps its own running maximum, sum of weights and sums
// of values over the tokens it reads; the groups and the four waves are
// joined once at the end.  Bound by HBM for few heads (fp32, 16 x 1024
// positions, 32 heads of 64: 26 us from the Infinity Cache, 5.4 TB/s, 33-37
// from cold pages), by its multiply-adds, one a value and head, from about
// eight 16-bit heads on, which the matrix-core kernel takes.
template <class T, int LPT, int EPL, bool VEC, int GT>
__global__ __launch_bounds__(AT_NT) void nm_attend_kernel(AttendArgs p)
{
    constexpr int TPW = 64 / LPT, U = 4;
    __shared__ float s_acc[AT_NW][GT][LPT * EPL];
    __shared__ float2 s_ml[AT_NW][GT];
    const AttendTask t = attend_task(p, blockIdx.x, GT);
    if (t.begin >= t.end && p.splits > 1) {      // nothing here: the maximum says so
        if (threadIdx.x < t.heads_in_tile) {
            const int64_t row = t.seq * ((int64_t)p.heads * p.group) + t.first_head + threadIdx.x;
            p.part_ml[row * p.splits + t.split] = make_float2(NEG_INF, 0.f);
        }
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int grp = lane / LPT, d0 = lane % LPT * EPL;
    const int valid = p.dim - d0 < 0 ? 0 : p.dim - d0;

    float q[GT][EPL], acc[GT][EPL], m[GT], l[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
        m[g] = NEG_INF;
        l[g] = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) q[g][i] = acc[g][i] = 0.f;
        if (g < t.heads_in_tile) {
            const int64_t at = t.seq * p.qs[0] + (t.first_head + g) * p.qs[1] + d0;
#pragma unroll
            for (int i = 0; i < EPL; ++i)
                if (i < valid) {
                    q[g][i] = p.io == NMSPMM_F32 ? static_cast<const float *>(p.q)[at + i]
                            : p.io == NMSPMM_BF16 ? to_f32(static_cast<const bf16_t *>(p.q)[at + i])
                                                  : to_f32(static_cast<const f16_t *>(p.q)[at + i]);
                    q[g][i] *= p.scale2;
                }
        }
    }
    const int32_t *row = p.c.table + t.seq * p.c.table_stride;
    const T *kb = static_cast<const T *>(p.k) + t.head * p.c.ks[2] + d0;
    const T *vb = static_cast<const T *>(p.v) + t.head * p.c.vs[2] + d0;
    for (int base = t.begin + wave * (TPW * U); base < t.end; base += AT_NW * TPW * U) {
        float k[U][EPL], v[U][EPL];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pos = base + u * TPW + grp;
            in[u] = pos < t.end;
            Place at{0, 0, false};
            if (in[u]) at = place_of(p.c, row, pos);
            in[u] = in[u] && at.held;
            load_row<EPL, VEC>(kb + (in[u] ? at.page * p.c.ks[0] + at.slot * p.c.ks[1] : 0), in[u] ? valid : 0, k[u]);
            load_row<EPL, VEC>(vb + (in[u] ? at.page * p.c.vs[0] + at.slot * p.c.vs[1] : 0), in[u] ? valid : 0, v[u]);
        }
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            float s[U], top = m[g];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < EPL; ++i) x = fmaf(q[g][i], k[u][i], x);
                x = lanes_sum<LPT>(x);
                s[u] = in[u] ? x : NEG_INF;
                top = fmaxf(top, s[u]);
            }
            const float ref = softmax_ref(top), corr = exp2f(m[g] - ref);
            m[g] = top;
            l[g] *= corr;
#pragma unroll
            for (int i = 0; i < EPL; ++i) acc[g][i] *= corr;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float w = exp2f(s[u] - ref);
                l[g] += w;
#pragma unroll
                for (int i = 0; i < EPL; ++i) acc[g][i] = fmaf(w, v[u][i], acc[g][i]);
            }
        }
    }
    // join the wave's groups, then the waves
#pragma unroll
    for (int g = 0; g < GT; ++g) {
#pragma unroll
        for (int step = LPT; step < 64; step *= 2) {
            const float om = __shfl_xor(m[g], step), ol = __shfl_xor(l[g], step);
            const float top = fmaxf(m[g], om), ref = softmax_ref(top);
            const float mine = exp2f(m[g] - ref), theirs = exp2f(om - ref);
            m[g] = top;
            l[g] = l[g] * mine + ol * theirs;
#pragma unroll
            for (int i = 0; i < EPL; ++i) acc[g][i] = acc[g][i] * mine + __shfl_xor(acc[g][i], step) * theirs;
        }
        if (grp == 0) {
#pragma unroll
            for (int i = 0; i < EPL; ++i) s_acc[wave][g][d0 + i] = acc[g][i];
            if (lane == 0) s_ml[wave][g] = make_float2(m[g], l[g]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < t.heads_in_tile * p.dim; i += AT_NT) {
        const int g = i / p.dim, d = i % p.dim;
        float top = NEG_INF, x = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < AT_NW; ++w) top = fmaxf(top, s_ml[w][g].x);
        const float ref = softmax_ref(top);
#pragma unroll
        for (int w = 0; w < AT_NW; ++w) {
            const float c = exp2f(s_ml[w][g].x - ref);
            x += c * s_acc[w][g][d];
            sum += c * s_ml[w][g].y;
        }
        attend_store(p, t, t.first_head + g, d, x, top, sum);
    }
}

constexpr int JN_SPLITS = 2048, JN_U = 4;

// The parts of a split sequence joined, one query head a workgroup: the
// weights of all splits first, then DL threads take a split's dimensions and
// the workgroup's NT / DL groups the splits in turn, JN_U of each asked for
// at once; the groups are added in their order.  (One thread a dimension over
// all splits, one after another, took 180 us of 286 on one sequence of 131071
// positions; eight groups with one load at a time 52 of 176.)
template <int NT, int SPLITS, int DL, int DV>
__global__ __launch_bounds__(NT) void nm_attend_join_kernel(AttendArgs p)
{
    constexpr int GROUPS = NT / DL;
    __shared__ float s_w[SPLITS], s_x[GROUPS][DL * DV], s_top[NT / 64], s_sum[NT / 64];
    const int64_t row = blockIdx.x;
    const int64_t q_heads = (int64_t)p.heads * p.group;
    AttendTask t{};
    t.seq = row / q_heads;
    const int64_t head = row % q_heads;
    const float2 *ml = p.part_ml + row * p.splits;
    float top = NEG_INF;
    for (int s = threadIdx.x; s < p.splits; s += NT) top = fmaxf(top, ml[s].x);
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) top = fmaxf(top, __shfl_xor(top, step));
    if (threadIdx.x % 64 == 0) s_top[threadIdx.x / 64] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) top = fmaxf(top, s_top[w]);
    const float ref = softmax_ref(top);
    float sum = 0.f;
    for (int s = threadIdx.x; s < p.splits; s += NT) {
        const float2 e = ml[s];
        // a split with nothing in it wrote no sums: its weight says so (negative)
        const bool empty = e.x == NEG_INF && e.y == 0.f;
        const float c = empty ? 0.f : exp2f(e.x - ref);
        s_w[s] = empty ? -1.f : c;
        sum += c * e.y;
    }
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) sum += __shfl_xor(sum, step);
    if (threadIdx.x % 64 == 0) s_sum[threadIdx.x / 64] = sum;
    __syncthreads();
    const int group = threadIdx.x / DL, d = threadIdx.x % DL * DV;
    float x[DV] = {};
    if (d < p.dim)
        for (int s = group; s < p.splits; s += GROUPS * JN_U) {
            float v[JN_U][DV], w[JN_U];
#pragma unroll
            for (int u = 0; u < JN_U; ++u) {
                const int at = s + u * GROUPS;
                w[u] = at < p.splits ? s_w[at] : -1.f;
                if (w[u] < 0.f) continue;
#pragma unroll
                for (int i = 0; i < DV; ++i) v[u][i] = p.part_acc[(row * p.splits + at) * p.dim + d + i];
            }
#pragma unroll
            for (int u = 0; u < JN_U; ++u)
#pragma unroll
                for (int i = 0; i < DV; ++i) x[i] = w[u] < 0.f ? x[i] : fmaf(w[u], v[u][i], x[i]);
        }
#pragma unroll
    for (int i = 0; i < DV; ++i) s_x[group][d + i] = x[i];
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) sum += s_sum[w];
    AttendArgs whole = p;
    whole.splits = 1;
    for (int i = threadIdx.x; i < p.dim; i += NT) {
        float y = 0.f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) y += s_x[g][i];
        attend_store(whole, t, head, i, y, top, sum);
    }
}

template <int DL, int DV>
void launch_join_of(const AttendArgs &p, int64_t rows, hipStream_t stream)
{
    // few splits: small workgroups, of which a CU runs more (48 sequences x 64
    // heads of 8 splits: 9.9 us with 512 threads)
    constexpr int FEW = DL < 128 ? 128 : DL;
    if (p.splits <= 16)
        hipLaunchKernelGGL((nm_attend_join_kernel<FEW, 16, DL, DV>), dim3((unsigned)rows), dim3(FEW), 0, stream, p);
    else
        hipLaunchKernelGGL((nm_attend_join_kernel<512, JN_SPLITS, DL, DV>), dim3((unsigned)rows), dim3(512), 0, stream, p);
}

// Four dimensions a thread where they come in fours.
void launch_join(const AttendArgs &p, int64_t rows, hipStream_t stream)
{
    if (p.dim % 4 == 0 && p.dim <= 64) launch_join_of<16, 4>(p, rows, stream);
    else if (p.dim % 4 == 0 && p.dim <= 128) launch_join_of<32, 4>(p, rows, stream);
    else if (p.dim % 4 == 0) launch_join_of<128, 4>(p, rows, stream);
    else launch_join_of<512, 1>(p, rows, stream);
}

// How the work is cut: query heads a workgroup takes together, workgroups
// along a sequence and the positions of each.
struct AttendPlan {
    int GT, gtiles, splits, chunk;
    int64_t groups;             // workgroups
    int64_t rows;               // sequences x query heads
    int64_t ml_bytes, bytes;    // workspace
};

AttendPlan attend_plan(const nmspmm_kv_cache_t *c, int64_t q_heads, int64_t max_length, int64_t window, bool mfma,
                       bool split)
{
    AttendPlan a{};
    const int64_t group = q_heads / c->heads;
    a.GT = mfma ? ATTEND_MFMA_HEADS : group >= 5 ? 8 : group >= 3 ? 4 : (int)group;
    a.gtiles = (int)((group + a.GT - 1) / a.GT);
    int64_t span = std::min({max_length, table_positions(c), KV_MAX_LENGTH});
    if (window > 0) span = std::min(span, window);
    const int64_t base = c->sequences * c->heads * a.gtiles;
    // eight workgroups a CU (two or three run at once), each of 256 positions at
    // least; and of 1024 at most, for batches whose lengths differ, which only
    // the device knows (192 sequences of 0 to 5000 positions, 64 heads on 8: 273
    // us, with chunks of 2500 404; 64 of 8192 each: 420 and 407), up to 64
    // workgroups a CU (which bounds the workspace)
    int64_t splits = 1;
    if (split && base > 0) {
        splits = std::max<int64_t>(1, std::min<int64_t>((JN_SPLITS + base - 1) / base, span / 256));
        splits = std::max(splits, std::min<int64_t>({JN_SPLITS, (span + 1023) / 1024, 16384 / base}));
    }
    a.chunk = (int)std::max<int64_t>(128, ((span + splits - 1) / splits + 127) / 128 * 128);
    a.splits = (int)std::max<int64_t>(1, (span + a.chunk - 1) / a.chunk);     // 1 where splits is
    a.groups = base * a.splits;
    a.rows = c->sequences * q_heads;
    if (a.splits > 1) {
        a.ml_bytes = (a.rows * a.splits * 8 + 255) / 256 * 256;
        a.bytes = a.ml_bytes + a.rows * a.splits * c->dim * 4;
    }
    return a;
}

// Whether the matrix-core kernel takes the call: a bf16 cache, or fp16 queries
// over an fp16 cache (whose range would not hold the parts of others), rows of
// whole 16-byte pieces, and a cache whose pieces are counted in 32 bits.
bool attend_takes_mfma(const nmspmm_kv_cache_t *c, nmspmm_dtype_t dtype)
{
    if (c->dtype == NMSPMM_F32 || (c->dtype == NMSPMM_F16 && dtype != NMSPMM_F16) || c->dim > 256) return false;
    for (const int64_t *stride : {c->k_stride, c->v_stride}) {
        const int64_t limit = (int64_t)1 << 34;     // elements: 2^32 - 1 pieces hold every row's start
        if (stride[0] < 0 || stride[1] < 0 || stride[0] > limit || stride[1] > limit) return false;
        if (stride[0] && c->pages > limit / stride[0]) return false;
        if (stride[1] && c->page_size > limit / stride[1]) return false;
        if (c->pages * stride[0] + c->page_size * stride[1] > limit) return false;
    }
    return rows_aligned(c->k_pages, c->k_stride, 3, c->dim, 2) && rows_aligned(c->v_pages, c->v_stride, 3, c->dim, 2);
}

template <class T, int LPT, int EPL, bool VEC>
void launch_attend_heads(const AttendArgs &p, int GT, unsigned groups, hipStream_t stream)
{
    const dim3 grid(groups), block(AT_NT);
    if (GT == 1) hipLaunchKernelGGL((nm_attend_kernel<T, LPT, EPL, VEC, 1>), grid, block, 0, stream, p);
    else if (GT == 2) hipLaunchKernelGGL((nm_attend_kernel<T, LPT, EPL, VEC, 2>), grid, block, 0, stream, p);
    else if (GT == 4) hipLaunchKernelGGL((nm_attend_kernel<T, LPT, EPL, VEC, 4>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((nm_attend_kernel<T, LPT, EPL, VEC, 8>), grid, block, 0, stream, p);
}

template <class T>
void launch_attend(const AttendArgs &p, bool vec, int GT, unsigned groups, hipStream_t stream)
{
    constexpr int EPL = 16 / sizeof(T);
    if (!vec || p.dim > 64 * EPL) launch_attend_heads<T, 64, 8, false>(p, GT, groups, stream);
    else if (p.dim <= 8 * EPL) launch_attend_heads<T, 8, EPL, true>(p, GT, groups, stream);
    else if (p.dim <= 16 * EPL) launch_attend_heads<T, 16, EPL, true>(p, GT, groups, stream);
    else if (p.dim <= 32 * EPL) launch_attend_heads<T, 32, EPL, true>(p, GT, groups, stream);
    else launch_attend_heads<T, 64, EPL, true>(p, GT, groups, stream);
}

nmspmm_status_t check_attend_sizes(const nmspmm_kv_cache_t *c, int64_t q_heads, int64_t max_length, int64_t window)
{
    const nmspmm_status_t st = check_cache(c);
    if (st != NMSPMM_OK) return st;
    if (q_heads < 0 || q_heads % c->heads || max_length < 0 || window < 0) return NMSPMM_ERR_INVALID_ARG;
    // workgroups of 256 threads in one launch of fewer than 2^32 threads
    const int64_t limit = ((int64_t)1 << 24) - 1;
    if (q_heads > limit || (c->sequences && q_heads > limit / c->sequences)) return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

}  // namespace
}  // namespace nmspmm

using namespace nmspmm;

extern "C" nmspmm_status_t nmspmm_kv_append(const nmspmm_kv_cache_t *cache, const void *k_new, const int64_t *k_stride,
                                            const void *v_new, const int64_t *v_stride, nmspmm_dtype_t dtype,
                                            int64_t tokens, const int32_t *seq, const int32_t *pos, const float *cos,
                                            const float *sin, int64_t positions, int rot, int interleaved,
                                            const void *q, const int64_t *q_stride, void *q_out,
                                            const int64_t *q_out_stride, int64_t q_heads, hipStream_t stream)
{
    nmspmm_status_t st = check_cache(cache);
    if (st != NMSPMM_OK) return st;
    if (!dtype_ok(dtype) || tokens < 0 || positions < 0 || q_heads < 0 || rot < 0 || rot % 2 || rot > cache->dim)
        return NMSPMM_ERR_INVALID_ARG;
    if (tokens == 0) return NMSPMM_OK;
    st = check_cache_pointers(cache);
    if (st != NMSPMM_OK) return st;
    if (!k_new || !v_new || !k_stride || !v_stride || !seq || !pos) return NMSPMM_ERR_INVALID_ARG;
    if (rot > 0 && positions > 0 && (!cos || !sin)) return NMSPMM_ERR_INVALID_ARG;
    if (q_heads > 0 && (!q || !q_out || !q_stride || !q_out_stride)) return NMSPMM_ERR_INVALID_ARG;
    const int es = dtype_bytes(dtype);
    if (!aligned_to(k_new, es) || !aligned_to(v_new, es) || !aligned_to(seq, 4) || !aligned_to(pos, 4) ||
        !aligned_to(cos, 4) || !aligned_to(sin, 4) || !aligned_to(q, es) || !aligned_to(q_out, es))
        return NMSPMM_ERR_UNSUPPORTED;
    if (q_heads > INT31 || positions > INT31) return NMSPMM_ERR_UNSUPPORTED;
    const int64_t items = (2 * (int64_t)cache->heads + q_heads) * ((cache->dim + 1) / 2);
    // a launch takes fewer than 2^32 threads along x and 2^16 workgroups along y
    if (tokens > (((int64_t)1 << 32) - 1) / AP_NT || items > (int64_t)65535 * AP_NT) return NMSPMM_ERR_UNSUPPORTED;
    AppendArgs p{};
    p.c = device_view(cache);
    p.k_new = k_new;
    p.v_new = v_new;
    p.q = q;
    p.k_pages = cache->k_pages;
    p.v_pages = cache->v_pages;
    p.q_out = q_out;
    for (int i = 0; i < 2; ++i) {
        p.kn[i] = k_stride[i];
        p.vn[i] = v_stride[i];
        p.qn[i] = q_heads ? q_stride[i] : 0;
        p.qo[i] = q_heads ? q_out_stride[i] : 0;
    }
    p.seq = seq;
    p.pos = pos;
    p.cos = cos;
    p.sin = sin;
    p.tokens = tokens;
    p.positions = positions;
    p.sequences = cache->sequences;
    p.table_positions = table_positions(cache);
    p.heads = cache->heads;
    p.q_heads = (int)q_heads;
    p.dim = cache->dim;
    p.rot = rot;
    p.interleaved = interleaved != 0;
    const int cs = dtype_bytes(cache->dtype);
    const bool vec = cache->dim % 16 == 0 && rot % 16 == 0 && rows_aligned(k_new, k_stride, 2, cache->dim, es) &&
                     rows_aligned(v_new, v_stride, 2, cache->dim, es) && aligned_to(cos, 16) && aligned_to(sin, 16) &&
                     rows_aligned(cache->k_pages, cache->k_stride, 3, cache->dim, cs) &&
                     rows_aligned(cache->v_pages, cache->v_stride, 3, cache->dim, cs) &&
                     (q_heads == 0 || (rows_aligned(q, q_stride, 2, cache->dim, es) &&
                                       rows_aligned(q_out, q_out_stride, 2, cache->dim, es)));
    const hipError_t e = dtype == NMSPMM_F32 ? launch_append<float>(p, cache->dtype, vec, stream)
                       : dtype == NMSPMM_BF16 ? launch_append<bf16_t>(p, cache->dtype, vec, stream)
                                              : launch_append<f16_t>(p, cache->dtype, vec, stream);
    return e == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" int64_t nmspmm_kv_attend_workspace_bytes(const nmspmm_kv_cache_t *cache, int64_t q_heads,
                                                    int64_t max_length, int64_t window)
{
    if (check_attend_sizes(cache, q_heads, max_length, window) != NMSPMM_OK) return -1;
    if (q_heads == 0 || cache->sequences == 0) return 0;
    // of whichever kernel the types and strides will choose
    return std::max(attend_plan(cache, q_heads, max_length, window, false, true).bytes,
                    attend_plan(cache, q_heads, max_length, window, true, true).bytes);
}

extern "C" nmspmm_status_t nmspmm_kv_attend(const nmspmm_kv_cache_t *cache, const void *q, const int64_t *q_stride,
                                            nmspmm_dtype_t dtype, int64_t q_heads, const int32_t *lengths,
                                            int64_t max_length, int64_t window, float scale, void *out,
                                            const int64_t *out_stride, float *lse, void *workspace,
                                            size_t workspace_bytes, hipStream_t stream)
{
    nmspmm_status_t st = check_attend_sizes(cache, q_heads, max_length, window);
    if (st != NMSPMM_OK) return st;
    if (!dtype_ok(dtype)) return NMSPMM_ERR_INVALID_ARG;
    if (q_heads == 0 || cache->sequences == 0) return NMSPMM_OK;
    st = check_cache_pointers(cache);
    if (st != NMSPMM_OK) return st;
    if (!q || !q_stride || !out || !out_stride || !lengths) return NMSPMM_ERR_INVALID_ARG;
    const int es = dtype_bytes(dtype);
    if (!aligned_to(q, es) || !aligned_to(out, es) || !aligned_to(lengths, 4) || !aligned_to(lse, 4) ||
        !aligned_to(workspace, 256))
        return NMSPMM_ERR_UNSUPPORTED;
    int cached = -1;
    const bool mfma = attend_takes_mfma(cache, dtype);
    AttendPlan a = attend_plan(cache, q_heads, max_length, window, mfma, true);
    if (a.bytes > 0 && (!workspace || (uint64_t)a.bytes > (uint64_t)workspace_bytes)) {
        workspace = capturing(stream) ? nullptr : ws_acquire(stream, (size_t)a.bytes, &cached);
        if (!workspace) a = attend_plan(cache, q_heads, max_length, window, mfma, false);
    }
    AttendArgs p{};
    p.c = device_view(cache);
    p.q = q;
    p.k = cache->k_pages;
    p.v = cache->v_pages;
    p.out = out;
    p.lse = lse;
    p.part_ml = static_cast<float2 *>(workspace);
    p.part_acc = reinterpret_cast<float *>(static_cast<char *>(workspace) + a.ml_bytes);
    p.lengths = lengths;
    for (int i = 0; i < 2; ++i) {
        p.qs[i] = q_stride[i];
        p.os[i] = out_stride[i];
    }
    p.cap = (int)std::min({max_length, table_positions(cache), KV_MAX_LENGTH});
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
    const int cs = dtype_bytes(cache->dtype);
    const bool vec = rows_aligned(cache->k_pages, cache->k_stride, 3, cache->dim, cs) &&
                     rows_aligned(cache->v_pages, cache->v_stride, 3, cache->dim, cs);
    if (mfma) launch_attend_mfma(p, cache->dtype, (unsigned)a.groups, stream);
    else if (cache->dtype == NMSPMM_F32) launch_attend<float>(p, vec, a.GT, (unsigned)a.groups, stream);
    else if (cache->dtype == NMSPMM_BF16) launch_attend<bf16_t>(p, vec, a.GT, (unsigned)a.groups, stream);
    else launch_attend<f16_t>(p, vec, a.GT, (unsigned)a.groups, stream);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        launch_join(p, a.rows, stream);
        e = hipGetLastError();
    }
    const hipError_t f = cached >= 0 ? ws_done(cached, stream) : hipSuccess;
    return e == hipSuccess && f == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}
