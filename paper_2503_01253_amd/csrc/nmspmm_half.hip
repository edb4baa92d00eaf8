// The N:M sparse product in bf16 and fp16 (nmspmm_half_*): layout of the
// packed weight, the kernels for any shape, and the dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "nmspmm_half.h"
#include "nmspmm_half_short.h"
#include "nmspmm_half_tile.h"
#include "nmspmm_half_tiles.h"
#include "nmspmm_internal.h"
#include "nmspmm_workspace.h"

namespace nmspmm {
namespace {

bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// ---- the packed weight -----------------------------------------------------
//
// Where V is a multiple of 16 the values lie as the matrix instruction reads
// them (nmspmm_half_tile.h): MI columns by STEP compressed rows an operand, a
// column tile's operands in the order of its units and steps; the offsets lie
// in the same order, one per block and compressed row: the column c of the
// unit as c * 8 + half_swz(c), or KR * 8 in padding rows; rows u and u + 4 of
// each eight lie side by side, which is how a lane reads them, and a block's
// end with a step of padding.  The order of a unit's rows is the packing
// kernel's.  Other widths, and windows too long or of too
// many kept rows for a stage, keep Bc and idx as they are (MI = 0).
struct HalfLayout {
    int MI, STEP, G, S, KR;
    int64_t w, q, windows, units, steps;    // units and steps of a column tile
    int64_t offs_at, bytes;
};

HalfLayout half_layout(int64_t k, int64_t n, int N, int M, int V)
{
    HalfLayout l{};
    l.windows = k / M;
    l.w = l.windows * N;
    l.q = n / V;
    // the fewest windows whose rows fill their operands best: whole pieces of 8
    // columns, at most 128 (which bound the LDS a stage takes), and the operands
    // of a stage
    // (and a grid of units x blocks that the packing kernel can have)
    const int MI = V % 16 || l.q > 65535 || l.windows >= (int64_t)1 << 24 ? 0 : V % 32 ? 16 : 32;
    double best = 0;
    for (int G = 1; MI && G * M <= 128; ++G) {
        const int step = 512 / MI, S = (G * N + step - 1) / step;
        if (S > HALF_MAX_QS) break;
        const double fill = (double)(G * N) / (S * step);
        if (G * M % 8 == 0 && fill > best + 1e-9) {
            best = fill;
            l.G = G;
            l.S = S;
        }
    }
    if (l.G == 0) {
        l.offs_at = round_up(2 * l.w * n, 256);
        l.bytes = l.offs_at + l.w * l.q;
        return l;
    }
    l.MI = MI;
    l.STEP = 512 / MI;
    l.KR = l.G * M;
    l.units = (l.windows + l.G - 1) / l.G;
    l.steps = l.units * l.S;
    l.offs_at = round_up(n / l.MI * l.steps * 1024, 256);
    l.bytes = l.offs_at + l.q * (l.steps + 1) * 2 * l.STEP;
    return l;
}

struct PackArgs {
    const void *Bc;
    const uint8_t *idx;
    void *vals;
    uint16_t *offs;
    HalfLayout l;
    int64_t n;
    int N, M, V;
};

template <class T, class S>
__global__ __launch_bounds__(256) void nm_half_pack_raw_kernel(const S *Bc, const uint8_t *idx, T *vals,
                                                               uint8_t *offs, int64_t count, int64_t icount, int M)
{
    const int64_t stride = (int64_t)gridDim.x * 256, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t e = t; e < count; e += stride) vals[e] = from_f32<T>(to_f32(Bc[e]));
    for (int64_t e = t; e < icount; e += stride) offs[e] = (uint8_t)(idx[e] < M ? idx[e] : M - 1);
}

// One workgroup a unit of one column block.  The order of a unit's compressed
// rows is free, as long as offsets and values agree: it is chosen so that the
// LDS rows which one cycle of a transposed read touches (four of 64 bytes with
// MI = 32, eight of 32 with MI = 16) lie on different banks where the unit's
// columns allow.  Rows of one class of columns share their banks; the r-th row
// of a class goes to group r, and what a class has beyond the number of groups
// fills the places other classes leave, which are those of the last groups.
// (In the order of the columns a read took 2.2 cycles more than it needs.)
// 4096 x 11008 at 8:32 from fp32 46 us, 68 MB: once a weight.
template <class T, class S>
__global__ __launch_bounds__(128) void nm_half_pack_kernel(PackArgs p)
{
    constexpr int SLOTS = HALF_MAX_QS * 32;
    __shared__ int s_class[SLOTS], s_column[SLOTS], s_row[SLOTS];   // s_row: of a place, the row in it (-1: padding)
    const int MI = p.l.MI, STEP = p.l.STEP, slots = p.l.S * STEP, rows = p.l.G * p.N;
    const int64_t unit = blockIdx.x, block = blockIdx.y, first = unit * rows;
    const int held = (int)(p.l.w - first < rows ? p.l.w - first : rows);
    const int classes = MI == 32 ? 4 : 8, groups = slots / classes, i = threadIdx.x;
    if (i < slots) {
        s_row[i] = -1;
        if (i < held) {
            const int o = p.idx[(first + i) * p.l.q + block], c = i / p.N * p.M + (o < p.M ? o : p.M - 1);
            s_column[i] = c;
            s_class[i] = MI == 32 ? half_swz(c) >> 1 : half_swz(c);
        }
    }
    __syncthreads();
    // the place of class k's member of group g
    auto place = [&](int g, int k) { return MI == 32 ? 4 * g + k : g / 2 * 16 + g % 2 * 4 + k % 4 + k / 4 * 8; };
    if (i < held) {
        int count[8] = {}, rank = 0;
        for (int j = 0; j < held; ++j) {
            const int k = s_class[j];
            if (k == s_class[i] && j < i) ++rank;
#pragma unroll
            for (int c = 0; c < 8; ++c) count[c] += c == k;
        }
        int spare = rank - groups;      // among the rows that find their class full
        if (spare < 0) {
            s_row[place(rank, s_class[i])] = i;
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < s_class[i] && count[c] > groups) spare += count[c] - groups;
            // the spare-th free place: from the last group down, as every class fills from the first
            for (int g = groups - 1; g >= 0 && spare >= 0; --g)
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < classes && count[c] <= g && spare-- == 0) s_row[place(g, c)] = i;
        }
    }
    __syncthreads();
    const S *Bc = static_cast<const S *>(p.Bc);
    T *vals = static_cast<T *>(p.vals);
    // a lane's eight rows, of every operand of the unit in the block's tiles
    const int lane = i % 64;
    for (int o = i / 64; o < p.V / MI * p.l.S; o += 2) {
        const int s = o % p.l.S;
        const int64_t tile = block * (p.V / MI) + o / p.l.S, col = tile * MI + lane % MI;
        T *dst = vals + ((tile * p.l.steps + unit * p.l.S + s) * 64 + lane) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = s_row[s * STEP + lane / MI * 8 + j];
            dst[j] = r < 0 ? from_f32<T>(0.f) : from_f32<T>(to_f32(Bc[(first + r) * p.n + col]));
        }
    }
    uint16_t *offs = p.offs + block * (p.l.steps + 1) * STEP;
    const uint16_t padding = (uint16_t)(p.l.KR * 8);
    for (int e = i; e < slots; e += 128) {
        const int r = s_row[e / STEP * STEP + e % STEP / 8 * 8 + e % 8 / 2 + 4 * (e % 2)];
        offs[unit * slots + e] = r < 0 ? padding : (uint16_t)(s_column[r] * 8 + half_swz(s_column[r]));
    }
    if (unit == p.l.units - 1 && i < STEP) offs[p.l.steps * STEP + i] = padding;     // the block's last step
}

// ---- any shape -------------------------------------------------------------

struct GeneralArgs {
    const void *A;
    const void *vals;
    const void *offs;
    HalfLayout l;
    int64_t lda, m, n;
    int N, M, V;
    HalfEpilogue epi;
};

constexpr int HG_ROWS = 8;

// Any shape: a thread owns one column and HG_ROWS rows of C and walks the
// compressed rows of either layout; bound by the loads of A, one value per
// multiply-add: 3 to 6 TFLOP/s (4096^3 at 16:32 11.6 ms).
template <class T, class O>
__global__ __launch_bounds__(256) void nm_half_general_kernel(GeneralArgs p)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= p.n) return;
    const T *A = static_cast<const T *>(p.A), *vals = static_cast<const T *>(p.vals);
    for (int64_t i0 = (int64_t)blockIdx.y * HG_ROWS; i0 < p.m; i0 += (int64_t)gridDim.y * HG_ROWS) {
        float sum[HG_ROWS] = {};
        auto add = [&](int64_t at, float b) {
            const T *a = A + i0 * p.lda + at;
#pragma unroll
            for (int i = 0; i < HG_ROWS; ++i)
                if (i0 + i < p.m) sum[i] = fmaf(to_f32(a[i * p.lda]), b, sum[i]);
        };
        if (p.l.MI == 0) {
            const uint8_t *offs = static_cast<const uint8_t *>(p.offs) + j / p.V;
            int64_t window = 0;
            for (int64_t u = 0, r = 0; u < p.l.w; ++u) {
                add(window + offs[u * p.l.q], to_f32(vals[u * p.n + j]));
                if (++r == p.N) {
                    r = 0;
                    window += p.M;
                }
            }
        } else {
            const uint16_t *offs = static_cast<const uint16_t *>(p.offs) + j / p.V * (p.l.steps + 1) * p.l.STEP;
            const T *tile = vals + (j / p.l.MI * p.l.steps * 64 + j % p.l.MI) * 8;
            for (int64_t step = 0; step < p.l.steps; ++step)
                for (int u = 0; u < p.l.STEP; ++u) {
                    const uint16_t o = offs[step * p.l.STEP + u / 8 * 8 + u % 4 * 2 + u % 8 / 4];
                    if (o / 8 < p.l.KR)
                        add(step / p.l.S * p.l.KR + o / 8, to_f32(tile[(step * 64 + u / 8 * p.l.MI) * 8 + u % 8]));
                }
        }
#pragma unroll
        for (int i = 0; i < HG_ROWS; ++i)
            if (i0 + i < p.m) half_store<O>(p.epi, i0 + i, j, sum[i]);
    }
}

template <class T>
hipError_t launch_general(const GeneralArgs &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.n + 255) / 256),
                    (unsigned)std::min<int64_t>(65535, (p.m + HG_ROWS - 1) / HG_ROWS));
    if (p.epi.f32) hipLaunchKernelGGL((nm_half_general_kernel<T, float>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((nm_half_general_kernel<T, T>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

// ---- the tiled kernel ------------------------------------------------------

// The split parts of C added in order, then the epilogue, eight columns a
// thread (n is a multiple of 16 here).
template <class O>
__global__ __launch_bounds__(256) void nm_half_join_kernel(const float *part, int64_t m, int64_t n, int splits,
                                                           HalfEpilogue epi)
{
    const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (e >= m * n) return;
    float sum[8] = {}, x[8];
    for (int s = 0; s < splits; ++s) {
        load_row<8, true>(part + s * m * n + e, 8, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += x[i];
    }
    const int64_t row = e / n;
    half_store8<O>(epi, row, e - row * n, sum);
}

struct HalfTileInfo {
    int MI, CT, WK, BM, BN, kmax, rows;
    bool any;       // takes any alignment of A
};

#define NMSPMM_HALF_SHAPE(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS) HalfTile<MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS>
#define NMSPMM_HALF_INFO(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS, ANY)                       \
    {MI, CT, WK, NMSPMM_HALF_SHAPE(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS)::BM,             \
     NMSPMM_HALF_SHAPE(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS)::BN,                         \
     NMSPMM_HALF_SHAPE(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS)::KMAX,                       \
     NMSPMM_HALF_SHAPE(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS)::ROWS, ANY != 0},
const HalfTileInfo half_tiles[] = {NMSPMM_HALF_TILES(NMSPMM_HALF_INFO)};
#undef NMSPMM_HALF_INFO
#undef NMSPMM_HALF_SHAPE
constexpr int half_tile_count = sizeof half_tiles / sizeof half_tiles[0];

constexpr int HALF_SHORT = 1000;

struct HalfPlan {
    int tile = -1;      // the tiled kernel's shape, HALF_SHORT, or none: the general kernel
    int QS = 0, P = 0, nst = 0, tiles_m = 0, tiles_n = 0, splits = 1;
    int chunk_units = 0, chunks = 0;    // of HALF_SHORT
    bool wide = false;
    bool vec = true;
    int64_t ws_bytes = 0;
};

// An estimate of the tiled kernel's time in us.  A CU's W workgroups run two
// at a time, each through its stages; a stage takes 0.8 us at least (its
// barrier, the latencies of its loads and reads), and where the CU is full
// what it loads from L2 (134 bytes a ns), writes into LDS (100, 32-row tiles
// half that) and multiplies (6.45 GFLOP/s a CU) take their time one after
// another.  (Fitted on MI355X: 4096^3 at 16:32 and V = 64 128 x 256 tiles, CT = 1,
// 94 us measured, 96 estimated; 128 x 128 114 and 131; 37 x 4096 x 11008 at 8:32 64 x 64 tiles 15.6 and
// 15.8, 64 x 128 17.3 and 16.4; 128 x 4096 x 4096 at 16:32 32 x 64 13.0 and
// 11.7, 64 x 64 17.6 and 16.4.)
double half_cost(const HalfTileInfo &t, const HalfLayout &l, int P, int QS, int64_t workgroups, int stages)
{
    const double a = 2.0 * t.BM * P * l.KR, slots = (double)QS * t.WK * l.STEP;
    const double full = (a / 134 + a / (t.BM == 32 ? 50 : 100) + 2.0 * t.BN * slots / 134) * 1e-3 +
                        2.0 * t.BM * t.BN * slots / 6.45e6;
    const double W = (double)((workgroups + 255) / 256);
    return 3 + stages * std::max(0.8 * std::ceil(W / 2), W * full);
}

// vec: A's rows start on 16 bytes.
HalfPlan half_plan(int64_t m, const HalfLayout &l, const nmspmm_half_weight_t &w, bool vec, bool may_split)
{
    HalfPlan best;
    if (l.MI == 0 || w.k == 0 || w.k >= (int64_t)1 << 21) return best;
    double best_cost = 1e300;
    // (a launch takes fewer than 2^32 threads)
    if (m <= HS_ROWS && vec && l.S * l.STEP == l.G * w.N && l.windows % l.G == 0 &&
        w.n / l.MI < ((int64_t)1 << 32) / HS_NT) {
        // the largest chunk of A that a slot holds, then the chunks made even
        best.wide = w.n / l.MI <= 256;
        const int slot = best.wide ? HS_SLOT_WIDE : HS_SLOT;
        int64_t units = round_up(l.units, HS_NW);
        while (units > 0 && m * half_short_pitch((int)std::min<int64_t>(units, 1 << 16), l.KR) > slot) units -= HS_NW;
        if (units > 0) {
            best.tile = HALF_SHORT;
            best.chunks = (int)((l.units + units - 1) / units);
            best.chunk_units = (int)round_up((l.units + best.chunks - 1) / best.chunks, HS_NW);
            best.chunks = (int)((l.units + best.chunk_units - 1) / best.chunk_units);
            best_cost = 0;
        }
    }
    for (int i = 0; i < half_tile_count; ++i) {
        const HalfTileInfo &t = half_tiles[i];
        if (t.MI != l.MI) continue;
        HalfPlan c;
        c.tile = i;
        // the longest stage that LDS and registers hold
        for (int QS = HALF_MAX_QS; QS >= 1 && c.QS == 0; --QS)
            if (QS % l.S == 0 && QS / l.S * t.WK * l.KR <= t.kmax && QS / l.S * t.WK * (l.KR + 1) <= t.rows) c.QS = QS;
        if (c.QS == 0) continue;
        c.P = c.QS / l.S * t.WK;
        c.vec = vec;
        if (!c.vec && !t.any) continue;
        if (w.V % (t.CT * t.MI)) continue;
        const int64_t tiles_m = (m + t.BM - 1) / t.BM, tiles_n = (w.n + t.BN - 1) / t.BN;
        if (tiles_m * tiles_n > ((int64_t)1 << 22)) continue;
        c.nst = (int)((l.units + c.P - 1) / c.P);
        c.tiles_m = (int)tiles_m;
        c.tiles_n = (int)tiles_n;
        // k in several slices where the tiles leave CUs idle; joining them costs
        // a launch and the parts' way through memory
        const int most = may_split && tiles_m * tiles_n < 256 ? std::min(c.nst, 16) : 1;
        for (c.splits = 1; c.splits <= most; ++c.splits) {
            c.ws_bytes = c.splits > 1 ? c.splits * m * w.n * 4 : 0;
            double cost = half_cost(t, l, c.P, c.QS, tiles_m * tiles_n * c.splits, (c.nst + c.splits - 1) / c.splits);
            if (c.splits > 1) cost += 3 + (c.splits + 1) * m * w.n * 4 / 2e6;
            if (cost < best_cost) {
                best_cost = cost;
                best = c;
            }
        }
    }
    return best;
}

nmspmm_status_t check_weight(const nmspmm_half_weight_t *w, int64_t m)
{
    if (!w || !shape_ok(m, w->n, w->k, w->N, w->M, w->V)) return NMSPMM_ERR_INVALID_ARG;
    if (w->dtype != NMSPMM_BF16 && w->dtype != NMSPMM_F16) return NMSPMM_ERR_INVALID_ARG;
    // a launch takes fewer than 2^32 threads, one a column
    if (!sizes_fit(m, w->n, w->k) || w->n >= (int64_t)1 << 31) return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

template <class T>
hipError_t pack(const void *Bc, nmspmm_dtype_t type, const uint8_t *idx, const nmspmm_half_weight_t &w,
                hipStream_t stream)
{
    PackArgs p{};
    p.l = half_layout(w.k, w.n, w.N, w.M, w.V);
    p.Bc = Bc;
    p.idx = idx;
    p.vals = const_cast<void *>(w.packed);
    p.offs = reinterpret_cast<uint16_t *>(static_cast<char *>(p.vals) + p.l.offs_at);
    p.n = w.n;
    p.N = w.N;
    p.M = w.M;
    p.V = w.V;
    const int64_t count = p.l.w * w.n, icount = p.l.w * p.l.q;
    const dim3 grid((unsigned)std::min<int64_t>(8192, (count + 255) / 256));
    if (p.l.MI == 0) {
        T *vals = static_cast<T *>(p.vals);
        uint8_t *offs = reinterpret_cast<uint8_t *>(p.offs);
        if (type == NMSPMM_F32)
            hipLaunchKernelGGL((nm_half_pack_raw_kernel<T, float>), grid, dim3(256), 0, stream,
                               static_cast<const float *>(Bc), idx, vals, offs, count, icount, w.M);
        else
            hipLaunchKernelGGL((nm_half_pack_raw_kernel<T, T>), grid, dim3(256), 0, stream,
                               static_cast<const T *>(Bc), idx, vals, offs, count, icount, w.M);
    } else {
        // (a layout with more blocks or units than a grid takes does not arise: see half_layout)
        const dim3 units((unsigned)p.l.units, (unsigned)p.l.q);
        if (type == NMSPMM_F32) hipLaunchKernelGGL((nm_half_pack_kernel<T, float>), units, dim3(128), 0, stream, p);
        else hipLaunchKernelGGL((nm_half_pack_kernel<T, T>), units, dim3(128), 0, stream, p);
    }
    return hipGetLastError();
}

template <class T>
hipError_t run(const HalfPlan &c, const HalfLayout &l, const void *A, int64_t lda, const nmspmm_half_weight_t &w,
               int64_t m, const HalfEpilogue &epi, void *workspace, hipStream_t stream)
{
    const char *base = static_cast<const char *>(w.packed);
    if (c.tile < 0) {
        GeneralArgs p{};
        p.A = A;
        p.vals = base;
        p.offs = base + l.offs_at;
        p.l = l;
        p.lda = lda;
        p.m = m;
        p.n = w.n;
        p.N = w.N;
        p.M = w.M;
        p.V = w.V;
        p.epi = epi;
        return launch_general<T>(p, stream);
    }
    if (c.tile == HALF_SHORT) {
        HalfShortArgs p{};
        p.A = A;
        p.vals = reinterpret_cast<const unsigned char *>(base);
        p.offs = reinterpret_cast<const uint16_t *>(base + l.offs_at);
        p.lda = lda;
        p.n = w.n;
        p.k = w.k;
        p.m = (int)m;
        p.V = w.V;
        p.S = l.S;
        p.KR = l.KR;
        p.steps = (int)l.steps;
        p.chunk_units = c.chunk_units;
        p.chunks = c.chunks;
        p.epi = epi;
        return launch_half_short(l.MI, p, w.dtype == NMSPMM_BF16, c.wide, stream);
    }
    HalfTileArgs p{};
    p.A = A;
    p.vals = reinterpret_cast<const unsigned char *>(base);
    p.offs = reinterpret_cast<const uint16_t *>(base + l.offs_at);
    p.part = static_cast<float *>(workspace);
    p.lda = lda;
    p.m = m;
    p.n = w.n;
    p.k = w.k;
    p.V = w.V;
    p.S = l.S;
    p.KR = l.KR;
    p.P = c.P;
    p.steps = (int)l.steps;
    p.nst = c.nst;
    p.tiles_m = c.tiles_m;
    p.tiles_n = c.tiles_n;
    p.splits = c.splits;
    p.epi = epi;
    const bool bf16 = w.dtype == NMSPMM_BF16;
    hipError_t e = c.QS == 1 ? launch_half_q1(c.tile, p, bf16, c.vec, stream)
                 : c.QS == 2 ? launch_half_q2(c.tile, p, bf16, c.vec, stream)
                 : c.QS == 3 ? launch_half_q3(c.tile, p, bf16, c.vec, stream)
                             : launch_half_q4(c.tile, p, bf16, c.vec, stream);
    if (e == hipSuccess && c.splits > 1) {
        const unsigned blocks = (unsigned)((m * w.n + 2047) / 2048);
        if (epi.f32)
            hipLaunchKernelGGL((nm_half_join_kernel<float>), dim3(blocks), dim3(256), 0, stream, p.part, m, w.n, c.splits, epi);
        else
            hipLaunchKernelGGL((nm_half_join_kernel<T>), dim3(blocks), dim3(256), 0, stream, p.part, m, w.n, c.splits, epi);
        e = hipGetLastError();
    }
    return e;
}

// The plan of a call.  Where a row of A lies so far from the next that a
// tile's rows span 2^29 bytes, the general kernel runs.
HalfPlan plan_for(const void *A, int64_t lda, int64_t m, const HalfLayout &l, const nmspmm_half_weight_t &w,
                  bool may_split)
{
    if (lda >= (int64_t)1 << 21) return HalfPlan{};
    return half_plan(m, l, w, aligned_to(A, 16) && (m == 1 || lda % 8 == 0), may_split);
}

}  // namespace
}  // namespace nmspmm

using namespace nmspmm;

extern "C" int64_t nmspmm_half_bytes(int64_t k, int64_t n, int N, int M, int V)
{
    if (!shape_ok(0, n, k, N, M, V) || !sizes_fit(1, n, k)) return -1;
    if (k == 0 || n == 0) return 0;
    return half_layout(k, n, N, M, V).bytes;
}

extern "C" nmspmm_status_t nmspmm_half_pack(const void *Bc, nmspmm_dtype_t bc_dtype, const uint8_t *idx,
                                            const nmspmm_half_weight_t *weight, hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, 0);
    if (st != NMSPMM_OK) return st;
    if (bc_dtype != NMSPMM_F32 && bc_dtype != weight->dtype) return NMSPMM_ERR_INVALID_ARG;
    if (weight->k == 0 || weight->n == 0) return NMSPMM_OK;
    if (!Bc || !idx || !weight->packed) return NMSPMM_ERR_INVALID_ARG;
    if (!aligned_to(Bc, dtype_bytes(bc_dtype)) || !aligned_to(weight->packed, 256)) return NMSPMM_ERR_UNSUPPORTED;
    const hipError_t e = weight->dtype == NMSPMM_BF16 ? pack<bf16_t>(Bc, bc_dtype, idx, *weight, stream)
                                                      : pack<f16_t>(Bc, bc_dtype, idx, *weight, stream);
    return e == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" int64_t nmspmm_half_workspace_bytes(int64_t m, const nmspmm_half_weight_t *weight)
{
    if (check_weight(weight, m) != NMSPMM_OK) return -1;
    if (m == 0 || weight->n == 0) return 0;
    const HalfLayout l = half_layout(weight->k, weight->n, weight->N, weight->M, weight->V);
    // of whichever plan A's place will choose
    return std::max(half_plan(m, l, *weight, true, true).ws_bytes, half_plan(m, l, *weight, false, true).ws_bytes);
}

extern "C" const char *nmspmm_half_kernel_name(int64_t m, const nmspmm_half_weight_t *weight, int with_workspace)
{
    if (check_weight(weight, m) != NMSPMM_OK) return "invalid";
    if (m == 0 || weight->n == 0) return "none";
    const HalfLayout l = half_layout(weight->k, weight->n, weight->N, weight->M, weight->V);
    const HalfPlan c = half_plan(m, l, *weight, true, with_workspace != 0);
    if (c.tile < 0) return "nm_half_general_kernel";
    thread_local char buf[128];
    if (c.tile == HALF_SHORT) {
        std::snprintf(buf, sizeof buf, "nm_half_short_kernel<mi%d>,chunks%d", l.MI, c.chunks);
        return buf;
    }
    const HalfTileInfo &t = half_tiles[c.tile];
    std::snprintf(buf, sizeof buf, "nm_half_tile_kernel<%dx%d,mi%d,ct%d,wk%d,qs%d>,stage%d,split%d", t.BM, t.BN, t.MI,
                  t.CT, t.WK, c.QS, c.P * l.KR, c.splits);
    return buf;
}

extern "C" nmspmm_status_t nmspmm_half_run(const void *A, int64_t lda, const nmspmm_half_weight_t *weight, void *C,
                                           int64_t ldc, nmspmm_dtype_t c_dtype, int64_t m, float alpha,
                                           const float *bias, nmspmm_half_act_t act, const void *mul, int64_t ld_mul,
                                           const void *residual, int64_t ld_residual, void *workspace,
                                           size_t workspace_bytes, hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, m);
    if (st != NMSPMM_OK) return st;
    const nmspmm_half_weight_t &w = *weight;
    if ((c_dtype != NMSPMM_F32 && c_dtype != w.dtype) || act < NMSPMM_HALF_ACT_NONE || act > NMSPMM_HALF_ACT_SILU)
        return NMSPMM_ERR_INVALID_ARG;
    if (m == 0 || w.n == 0) return NMSPMM_OK;
    if (!C || (w.k > 0 && (!A || !w.packed))) return NMSPMM_ERR_INVALID_ARG;
    if (m > 1 && (lda < w.k || ldc < w.n || (mul && ld_mul < w.n) || (residual && ld_residual < w.n)))
        return NMSPMM_ERR_INVALID_ARG;
    const int cs = dtype_bytes(c_dtype);
    if (!aligned_to(A, 2) || !aligned_to(w.packed, 256) || !aligned_to(C, cs) || !aligned_to(bias, 4) ||
        !aligned_to(mul, cs) || !aligned_to(residual, cs) || !aligned_to(workspace, 256))
        return NMSPMM_ERR_UNSUPPORTED;
    if (!sizes_fit(m, std::max({ldc, ld_mul, ld_residual}), lda)) return NMSPMM_ERR_UNSUPPORTED;
    const HalfLayout l = half_layout(w.k, w.n, w.N, w.M, w.V);
    if (m == 1) lda = w.k;
    const auto rows16 = [cs](const void *ptr, int64_t ld) { return !ptr || (aligned_to(ptr, 16) && ld * cs % 16 == 0); };
    const HalfEpilogue epi = {C, bias, mul, residual, ldc, ld_mul, ld_residual, alpha, act, c_dtype == NMSPMM_F32,
                              rows16(C, ldc) && rows16(mul, ld_mul) && rows16(residual, ld_residual) &&
                                  aligned_to(bias, 16)};
    int cached = -1;
    HalfPlan c = plan_for(A, lda, m, l, w, true);
    if (c.ws_bytes > 0 && (!workspace || (uint64_t)c.ws_bytes > (uint64_t)workspace_bytes)) {
        workspace = capturing(stream) ? nullptr : ws_acquire(stream, (size_t)c.ws_bytes, &cached);
        if (!workspace) c = plan_for(A, lda, m, l, w, false);
    }
    const hipError_t e = w.dtype == NMSPMM_BF16 ? run<bf16_t>(c, l, A, lda, w, m, epi, workspace, stream)
                                                : run<f16_t>(c, l, A, lda, w, m, epi, workspace, stream);
    const hipError_t f = cached >= 0 ? ws_done(cached, stream) : hipSuccess;
    return e == hipSuccess && f == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}
