// The product with a weight in 4 bits (nmspmm_mx4_*): rounding to 4 bits,
// layout of the packed weight, the kernel for any shape, and the dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>

#include "nmspmm_half.h"
#include "nmspmm_internal.h"
#include "nmspmm_fp4.h"
#include "nmspmm_mx4.h"
#include "nmspmm_mx4_tile.h"
#include "nmspmm_workspace.h"

namespace nmspmm {
namespace {

bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// ---- rounding to 4 bits ------------------------------------------------------

// One column's group of 32 rows a thread, so that a wave reads rows in whole
// lines; the rows are read twice, the second time from L2.
template <class S>
__global__ __launch_bounds__(256) void nm_mx4_quantize_kernel(const S *Bc, int64_t w, int64_t n, uint8_t *codes,
                                                              uint8_t *scales)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= n) return;
    for (int64_t g = blockIdx.y; g * 32 < w; g += gridDim.y) {
        const S *x = Bc + g * 32 * n + j;
        const int held = (int)min<int64_t>(32, w - g * 32);
        uint32_t top = 0;
        for (int u = 0; u < held; ++u) top = max(top, __builtin_bit_cast(uint32_t, to_f32(x[u * n])) & 0x7fffffffu);
        const uint32_t s = mx4_scale_of(top);
        scales[g * n + j] = (uint8_t)s;
        for (int u0 = 0; u0 < held; u0 += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = u0 + i < held ? to_f32(x[(u0 + i) * n]) : 0.f;
            const uint32_t c = mx4_codes(v, s);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (u0 + i < held) codes[(g * 32 + u0 + i) * n + j] = (uint8_t)(c >> (4 * i) & 15);
        }
    }
}

// ---- the packed weight -----------------------------------------------------
//
// Where V is a multiple of 16 (and the pattern dense or such that a workgroup's
// LDS holds the columns of two groups of one row) the codes lie as the lanes of
// the matrix instruction read them, 16 columns by 32 compressed rows a word
// (nmspmm_mx4_tile.h), the scales beside them, and the offsets, in the same order,
// as byte offsets from the group's first window; padding rows have code 0.
//   dense    four groups (a step) of a column tile in 1 KB, 64 bytes of scales
//   sparse   one group of CT column tiles in CT * 256 bytes; 32 offsets a block
// Other widths keep two compressed rows' codes a byte, row-major, the scales and
// the offsets (none where N = M: row r of a window is its r-th).
enum class Mx4Kind { Raw, Dense, Sparse };

struct Mx4Layout {
    Mx4Kind kind;
    int CT;                         // of Sparse
    int64_t w, q, groups, steps;    // steps: of Dense fours of groups, of Sparse groups
    int64_t scales_at, offs_at, bytes;
};

// Columns of A that `groups` neighbouring groups can meet, from a multiple of 8 on.
int64_t mx4_columns(int64_t groups, int64_t k, int N, int M)
{
    const int64_t rows = groups * 32, windows = 32 % N == 0 ? rows / N : (rows - 1) / N + 2;
    return std::min(k, windows * M) + (M % 8 ? 7 : 0);
}

// Bytes of such a row in LDS: rows start four banks apart.
int64_t mx4_pitch(int64_t columns) { return round_up(columns * 2, 128) + 16; }

// LDS of the kernel for up to 16 rows: two workgroups a CU, or one.
constexpr int MX4_LDS = 80 * 1024, MX4_LDS_WIDE = 156 * 1024;

Mx4Layout mx4_layout(int64_t k, int64_t n, int N, int M, int V)
{
    Mx4Layout l{};
    l.w = k / M * N;
    l.q = n / V;
    l.groups = (l.w + 31) / 32;
    const int64_t tiles = n / 16;
    // (the kernels count compressed rows in 32 bits, and a launch takes fewer than 2^32 threads)
    const bool fits = V % 16 == 0 && l.w < ((int64_t)1 << 31) - 4096 && n < (int64_t)1 << 27;
    if (fits && N == M) {
        l.kind = Mx4Kind::Dense;
        l.steps = (l.groups + 3) / 4;
        l.scales_at = tiles * l.steps * 1024;
        l.offs_at = round_up(l.scales_at + tiles * l.steps * 64, 256);
        l.bytes = l.offs_at;
    } else if (fits && mx4_pitch(mx4_columns(2, k, N, M)) <= MX4_LDS / 2) {
        l.kind = Mx4Kind::Sparse;
        l.CT = V % 64 == 0 ? 4 : V % 32 == 0 ? 2 : 1;
        l.steps = l.groups;
        l.scales_at = tiles * l.steps * 256;
        l.offs_at = round_up(l.scales_at + tiles / l.CT * l.steps * 16 * l.CT, 256);
        l.bytes = l.offs_at + l.q * l.steps * 64;
    } else {
        l.kind = Mx4Kind::Raw;
        l.scales_at = round_up((l.w + 1) / 2 * n, 256);
        l.offs_at = round_up(l.scales_at + l.groups * n, 256);
        l.bytes = l.offs_at + (N == M ? 0 : l.w * l.q);
    }
    return l;
}

// A word of eight codes, a column's scale or an offset of a group a thread and
// step; once a weight.
__global__ __launch_bounds__(256) void nm_mx4_pack_kernel(const uint8_t *codes, const uint8_t *scales,
                                                          const uint8_t *idx, uint8_t *out, Mx4Layout l, int64_t n,
                                                          int N, int M, int V)
{
    const int64_t stride = (int64_t)gridDim.x * 256, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const bool dense = l.kind == Mx4Kind::Dense;
    const int per = dense ? 4 : l.CT;           // words of a lane's piece: groups, or column tiles
    const int64_t pieces = n / 16 * l.steps / (dense ? 1 : per);
    for (int64_t e = t; e < pieces * 64 * per; e += stride) {
        const int i = (int)(e % per), lane = (int)(e / per % 64);
        const int64_t run = e / per / 64 / l.steps, step = e / per / 64 % l.steps;
        const int64_t group = dense ? step * 4 + i : step;
        const int64_t j = (dense ? run : run * per + i) * 16 + lane % 16, u0 = group * 32 + lane / 16 * 8;
        uint32_t word = 0;
        for (int r = 0; r < 8; ++r)
            if (u0 + r < l.w) word |= (codes[(u0 + r) * n + j] & 15u) << (4 * r);
        reinterpret_cast<uint32_t *>(out)[e] = word;
    }
    for (int64_t e = t; e < pieces * 16 * per; e += stride) {
        const int i = (int)(e % per), col = (int)(e / per % 16);
        const int64_t run = e / per / 16 / l.steps, step = e / per / 16 % l.steps;
        const int64_t group = dense ? step * 4 + i : step, j = (dense ? run : run * per + i) * 16 + col;
        out[l.scales_at + e] = group < l.groups ? scales[group * n + j] : (uint8_t)127;
    }
    if (dense) return;
    uint16_t *offs = reinterpret_cast<uint16_t *>(out + l.offs_at);
    for (int64_t e = t; e < l.q * l.steps * 32; e += stride) {
        const int64_t block = e / 32 / l.steps, group = e / 32 % l.steps, u = group * 32 + e % 32;
        uint32_t at = 0;
        if (u < l.w) {
            const int o = idx[u * l.q + block];
            at = (uint32_t)((u / N - group * 32 / N) * M) + (o < M ? o : M - 1);
        }
        // rows r and r + 4 of each eight side by side: the lanes' order of both gathers
        offs[e - e % 8 + e % 4 * 2 + e % 8 / 4] = (uint16_t)(at * 2);
    }
}

__global__ __launch_bounds__(256) void nm_mx4_pack_raw_kernel(const uint8_t *codes, const uint8_t *scales,
                                                              const uint8_t *idx, uint8_t *out, Mx4Layout l, int64_t n,
                                                              int M)
{
    const int64_t stride = (int64_t)gridDim.x * 256, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t e = t; e < (l.w + 1) / 2 * n; e += stride) {
        const int64_t u = e / n * 2, j = e % n;
        const uint32_t hi = u + 1 < l.w ? codes[(u + 1) * n + j] & 15u : 0u;
        out[e] = (uint8_t)((codes[u * n + j] & 15u) | hi << 4);
    }
    for (int64_t e = t; e < l.groups * n; e += stride) out[l.scales_at + e] = scales[e];
    for (int64_t e = t; e < l.bytes - l.offs_at; e += stride) out[l.offs_at + e] = (uint8_t)(idx[e] < M ? idx[e] : M - 1);
}

// ---- any shape -------------------------------------------------------------

struct Mx4GeneralArgs {
    const void *A;
    const unsigned char *packed;
    Mx4Layout l;
    int64_t lda, m, n;
    int N, M, V;
    HalfEpilogue epi;
    int64_t first;      // column of the launch
};

constexpr int MG_ROWS = 8, MG_COLS = 32, MG_SLICES = 8;

// Any shape: a thread owns one column, MG_ROWS rows of C and a slice of the
// compressed rows, which it walks; the slices' sums are added in order.  Bound by
// the loads of A, one value per multiply-add (8 x 4096 x 4096 at 16:32, V = 8: 222
// us; one thread for all of k, 256 columns a workgroup: 1377).
template <class T, class O>
__global__ __launch_bounds__(MG_COLS * MG_SLICES) void nm_mx4_general_kernel(Mx4GeneralArgs p)
{
    __shared__ float part[MG_SLICES][MG_ROWS][MG_COLS];
    const int col = threadIdx.x % MG_COLS, slice = threadIdx.x / MG_COLS;
    const int64_t j = p.first + (int64_t)blockIdx.x * MG_COLS + col;
    const bool mine = j < p.n;
    const T *A = static_cast<const T *>(p.A);
    const unsigned char *scales = p.packed + p.l.scales_at;
    const unsigned char *offs = p.N == p.M ? nullptr : p.packed + p.l.offs_at + j / p.V;
    const int64_t rows = (p.l.groups + MG_SLICES - 1) / MG_SLICES * 32;
    const int64_t begin = slice * rows, end = begin + rows < p.l.w ? begin + rows : p.l.w;
    for (int64_t i0 = (int64_t)blockIdx.y * MG_ROWS; i0 < p.m; i0 += (int64_t)gridDim.y * MG_ROWS) {
        float sum[MG_ROWS] = {};
        int64_t window = begin / p.N * p.M, r = begin % p.N;
        for (int64_t u = begin; mine && u < end; ++u) {
            const uint32_t code = p.packed[u / 2 * p.n + j] >> (u % 2 * 4) & 15u;
            const float s = mx4_scale<0>(scales[u / 32 * p.n + j]);
            const float b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0)[0];
            const T *a = A + i0 * p.lda + window + (offs ? offs[u * p.l.q] : r);
#pragma unroll
            for (int i = 0; i < MG_ROWS; ++i)
                if (i0 + i < p.m) sum[i] = fmaf(to_f32(a[i * p.lda]), b, sum[i]);
            if (++r == p.N) {
                r = 0;
                window += p.M;
            }
        }
#pragma unroll
        for (int i = 0; i < MG_ROWS; ++i) part[slice][i][col] = sum[i];
        __syncthreads();
        // a row a slice's threads
        float all = 0.f;
#pragma unroll
        for (int x = 0; x < MG_SLICES; ++x) all += part[x][slice][col];
        if (mine && i0 + slice < p.m) half_store<O>(p.epi, i0 + slice, j, all);
        __syncthreads();
    }
}

template <class T>
hipError_t launch_general(Mx4GeneralArgs p, hipStream_t stream)
{
    static_assert(MG_ROWS == MG_SLICES, "a row a slice's threads");
    const int64_t most = (int64_t)1 << 28;      // (a grid takes fewer than 2^32 threads)
    for (; p.first < p.n; p.first += most) {
        const dim3 grid((unsigned)((std::min(most, p.n - p.first) + MG_COLS - 1) / MG_COLS),
                        (unsigned)std::min<int64_t>(65535, (p.m + MG_ROWS - 1) / MG_ROWS));
        const dim3 block(MG_COLS * MG_SLICES);
        if (p.epi.f32) hipLaunchKernelGGL((nm_mx4_general_kernel<T, float>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((nm_mx4_general_kernel<T, T>), grid, block, 0, stream, p);
    }
    return hipGetLastError();
}

// ---- the kernels for few rows ------------------------------------------------

// The slices of C added in order, then the epilogue, four columns a thread (n is
// a multiple of 16 here): eight slices' loads, and those of the epilogue, on their
// way at once (64 x 4096 from 8 slices and a term 3.9 us; one slice after another 12).
template <class T>
__global__ __launch_bounds__(128) void nm_mx4_join_kernel(const float *part, int64_t m, int64_t n, int splits,
                                                          HalfEpilogue epi)
{
    const int64_t e = ((int64_t)blockIdx.x * 128 + threadIdx.x) * 4;
    if (e >= m * n) return;
    const int64_t row = e / n, j = e - row * n;
    const Mx4Ahead ahead = mx4_fetch<T>(epi, row, j);
    float sum[4] = {};
    for (int s0 = 0; s0 < splits; s0 += 8) {
        float x[8][4];
#pragma unroll
        for (int s = 0; s < 8; ++s) load_row<4, true>(part + min(s0 + s, splits - 1) * m * n + e, 4, x[s]);
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += s0 + s < splits ? x[s][i] : 0.f;
    }
    mx4_emit<T>(epi, row, j, sum, ahead);
}

}  // namespace

// nmspmm_mx4_wide.hip
void launch_mx4_wide(int MT, int CT, int WC, int D, bool bf16, const Mx4Args &p, const dim3 &grid, hipStream_t stream);

namespace {

struct Mx4Plan {
    bool general = true;
    int MT = 1, CT = 1, WC = 1, D = 0, splits = 1;
    int rows = 16, chunk = 0, pitch = 0, slot = 0;      // of a workgroup; of a chunk of A
    bool wide = false;                      // one workgroup a CU
    int64_t per_split = 0, ws_bytes = 0;
};

Mx4Plan mx4_plan(int64_t m, const Mx4Layout &l, const nmspmm_mx4_weight_t &w, bool may_split)
{
    Mx4Plan c;
    if (l.kind == Mx4Kind::Raw || l.w == 0) return c;
    c.general = false;
    c.MT = m <= 16 ? 1 : m <= 32 ? 2 : 4;
    const auto pitch = [&](int64_t groups) { return mx4_pitch(mx4_columns(groups, w.k, w.N, w.M)); };
    if (l.kind == Mx4Kind::Dense) {
        // one workgroup a CU, as far as four tiles each go; more than 16 rows, of which
        // every workgroup reads all of A: four (1 x 4096 x 11008, 688 tiles:
        // CT = 1 to 4 9.3, 8.3, 7.0 and 7.9 us; 1 x 8192 x 8192, 512 tiles: 12.0, 9.2, 10.5, 11.5;
        // 1 x 4096 x 16384, 1024: 12.2, 9.4, 10.5, 9.0)
        c.CT = c.MT > 1 ? 4 : (int)std::min<int64_t>(4, (w.n / 16 + 255) / 256);
    } else {
        c.CT = l.CT;
        // the k-major kernel, where a slot holds a chunk: D groups of each of the waves that
        // share columns
        if (c.MT > 1) {
            for (c.WC = 4; c.WC <= 8 && c.D == 0; c.WC *= 2)
                for (int D = c.WC == 4 ? 4 : 1; D >= 1 && c.D == 0; D /= 2)
                    if (mx4_columns(D * (MX4_NW / c.WC), w.k, w.N, w.M) <= mx4_wide_columns(c.MT)) c.D = D;
            c.WC /= 2;
            c.chunk = c.D * (MX4_NW / c.WC);
            if (c.D == 0) c.MT = 1;
        }
        if (c.MT == 1) {
            c.rows = (int)std::min<int64_t>(m, 16);
            // one workgroup a CU, where A's rows may take all of its LDS, as far as four
            // runs of tiles each go (13 x 4096 x 11008 at 8:32, 344 runs: WC = 1, 2 and 4
            // 10.6, 8.1 and 10.7 us; 1 x 8192 x 8192 at 4:32, 128 runs: 4.6, 5.7, 8.0)
            const int64_t runs = w.n / (16 * l.CT);
            c.WC = runs <= 256 ? 1 : runs <= 512 ? 2 : 4;
            c.wide = (runs + c.WC - 1) / c.WC * ((m + c.rows - 1) / c.rows) <= 256;
            const int64_t lds = c.wide ? MX4_LDS_WIDE : MX4_LDS;
            for (;; c.WC < 4 ? (void)(c.WC = 4) : (void)(c.rows = (c.rows + 1) / 2)) {
                const int WK = MX4_NW / c.WC;
                int64_t chunk = round_up(l.steps, WK);
                if (c.rows * pitch(chunk) <= lds) {         // all of k
                    c.slot = (int)lds;
                } else {
                    c.slot = (int)lds / 2;
                    while (chunk > WK && c.rows * pitch(chunk) > c.slot) chunk -= WK;
                    if (c.rows * pitch(chunk) > c.slot) continue;
                }
                c.chunk = (int)chunk;
                c.pitch = (int)pitch(chunk);
                break;
            }
        }
    }
    if (c.MT > 1 || l.kind == Mx4Kind::Dense) c.rows = (int)std::min<int64_t>(m, 16 * c.MT);
    if (may_split && c.MT > 1) {
        const int64_t columns = l.kind == Mx4Kind::Dense ? (w.n / 16 + c.CT - 1) / c.CT
                                                         : (w.n / (16 * c.CT) + c.WC - 1) / c.WC;
        const int64_t tiles = columns * ((m + 16 * c.MT - 1) / (16 * c.MT));
        // k in slices where the tiles leave CUs idle, of eight steps at least (64 x 11008 x
        // 4096 at 16:32, 32 tiles: 1, 2, 4 and 8 slices 49, 30, 21 and 17 us; 40 x 4096 x
        // 11008 at 4:32, 86 tiles, 16 steps: 1 and 2 13.9 and 13.1, 4 half as much again)
        c.splits = (int)std::max<int64_t>(1, std::min<int64_t>({256 / tiles, l.steps / 8, 16}));
    }
    c.per_split = (l.steps + c.splits - 1) / c.splits;
    c.splits = (int)((l.steps + c.per_split - 1) / c.per_split);
    c.ws_bytes = c.splits > 1 ? c.splits * m * w.n * 4 : 0;
    return c;
}

template <class T, int MT, int CT>
void launch_dense(const Mx4Args &p, const dim3 &grid, hipStream_t stream)
{
    constexpr int D = MT <= 2 ? 2 : 1;
    if (p.vec) hipLaunchKernelGGL((nm_mx4_dense_kernel<T, MT, CT, D, true>), grid, dim3(MX4_NT), 0, stream, p);
    else hipLaunchKernelGGL((nm_mx4_dense_kernel<T, MT, CT, 1, false>), grid, dim3(MX4_NT), 0, stream, p);
}

template <class T, int CT, int WC>
void launch_short(const Mx4Args &p, const dim3 &grid, bool wide, hipStream_t stream)
{
    if (wide) hipLaunchKernelGGL((nm_mx4_sparse_kernel<T, CT, WC, 4, MX4_LDS_WIDE>), grid, dim3(MX4_NT), 0, stream, p);
    else hipLaunchKernelGGL((nm_mx4_sparse_kernel<T, CT, WC, 4, MX4_LDS>), grid, dim3(MX4_NT), 0, stream, p);
}

template <class T, int MT, int CT>
void launch_sparse(const Mx4Plan &c, const Mx4Args &p, const dim3 &grid, hipStream_t stream)
{
    if constexpr (MT == 1) {
        if (c.WC == 1) launch_short<T, CT, 1>(p, grid, c.wide, stream);
        else if (c.WC == 2) launch_short<T, CT, 2>(p, grid, c.wide, stream);
        else launch_short<T, CT, 4>(p, grid, c.wide, stream);
    } else {
        launch_mx4_wide(MT, CT, c.WC, c.D, __is_same(T, bf16_t), p, grid, stream);
    }
}

template <class T, int MT>
void launch_tiles(const Mx4Plan &c, Mx4Kind kind, Mx4Args p, hipStream_t stream)
{
    const int run = kind == Mx4Kind::Dense ? c.CT : c.WC;
    // (a grid takes fewer than 2^16 workgroups along y)
    const int64_t most = (int64_t)65535 * c.rows;
    for (; p.first_row < p.m; p.first_row += most) {
        const dim3 grid((unsigned)((p.tiles + run - 1) / run * c.splits),
                        (unsigned)((std::min(most, p.m - p.first_row) + c.rows - 1) / c.rows));
        if (kind == Mx4Kind::Dense) {
            if constexpr (MT == 1) {
                if (c.CT == 1) launch_dense<T, 1, 1>(p, grid, stream);
                else if (c.CT == 2) launch_dense<T, 1, 2>(p, grid, stream);
                else if (c.CT == 3) launch_dense<T, 1, 3>(p, grid, stream);
                else launch_dense<T, 1, 4>(p, grid, stream);
            } else {
                launch_dense<T, MT, 4>(p, grid, stream);
            }
        } else {
            if (c.CT == 1) launch_sparse<T, MT, 1>(c, p, grid, stream);
            else if (c.CT == 2) launch_sparse<T, MT, 2>(c, p, grid, stream);
            else launch_sparse<T, MT, 4>(c, p, grid, stream);
        }
    }
}

template <class T>
hipError_t run_tiles(const Mx4Plan &c, const Mx4Layout &l, const void *A, int64_t lda, const nmspmm_mx4_weight_t &w,
                     int64_t m, const HalfEpilogue &epi, void *workspace, hipStream_t stream)
{
    const unsigned char *base = static_cast<const unsigned char *>(w.packed);
    Mx4Args p{};
    p.A = A;
    p.vals = base;
    p.scales = base + l.scales_at;
    p.offs = reinterpret_cast<const uint16_t *>(base + l.offs_at);
    p.part = static_cast<float *>(workspace);
    p.lda = lda;
    p.m = m;
    p.n = w.n;
    p.k = w.k;
    p.w = (int)l.w;
    p.N = w.N;
    p.M = w.M;
    p.V = w.V;
    p.steps = (int)l.steps;
    p.splits = c.splits;
    p.per_split = (int)c.per_split;
    p.tiles = (int)(l.kind == Mx4Kind::Dense ? w.n / 16 : w.n / (16 * l.CT));
    p.rows = c.rows;
    p.chunk = c.chunk;
    p.pitch = c.pitch;
    p.slot = c.slot;
    // (the sparse kernel counts a workgroup's bytes of A in 32 bits)
    p.vec = aligned_to(A, 16) && (m == 1 || lda % 8 == 0) && w.k % 8 == 0 && lda < (int64_t)1 << 23;
    p.epi = epi;
    if (c.MT == 1) launch_tiles<T, 1>(c, l.kind, p, stream);
    else if (c.MT == 2) launch_tiles<T, 2>(c, l.kind, p, stream);
    else launch_tiles<T, 4>(c, l.kind, p, stream);
    if (c.splits > 1) {
        const dim3 grid((unsigned)((m * w.n + 511) / 512));
        hipLaunchKernelGGL((nm_mx4_join_kernel<T>), grid, dim3(128), 0, stream, p.part, m, w.n, c.splits, epi);
    }
    return hipGetLastError();
}

nmspmm_status_t check_weight(const nmspmm_mx4_weight_t *w, int64_t m)
{
    if (!w || !shape_ok(m, w->n, w->k, w->N, w->M, w->V)) return NMSPMM_ERR_INVALID_ARG;
    // a launch takes fewer than 2^32 threads, one a column
    if (!sizes_fit(m, w->n, w->k) || w->n >= ((int64_t)1 << 31) - 255) return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

}  // namespace
}  // namespace nmspmm

using namespace nmspmm;

extern "C" int64_t nmspmm_mx4_bytes(int64_t k, int64_t n, int N, int M, int V)
{
    if (!shape_ok(0, n, k, N, M, V) || !sizes_fit(1, n, k)) return -1;
    if (k == 0 || n == 0) return 0;
    return mx4_layout(k, n, N, M, V).bytes;
}

extern "C" nmspmm_status_t nmspmm_mx4_quantize(const void *Bc, nmspmm_dtype_t bc_dtype, int64_t w, int64_t n,
                                               uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    if (w < 0 || n < 0 || !dtype_ok(bc_dtype)) return NMSPMM_ERR_INVALID_ARG;
    if (w == 0 || n == 0) return NMSPMM_OK;
    if (!Bc || !codes || !scales) return NMSPMM_ERR_INVALID_ARG;
    if (!aligned_to(Bc, dtype_bytes(bc_dtype)) || !sizes_fit(1, n, w) || w >= ((int64_t)1 << 31) - 255 ||
        n >= ((int64_t)1 << 31) - 255)
        return NMSPMM_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((n + 255) / 256), (unsigned)std::min<int64_t>(65535, (w + 31) / 32));
    if (bc_dtype == NMSPMM_F32)
        hipLaunchKernelGGL((nm_mx4_quantize_kernel<float>), grid, dim3(256), 0, stream, static_cast<const float *>(Bc),
                           w, n, codes, scales);
    else if (bc_dtype == NMSPMM_BF16)
        hipLaunchKernelGGL((nm_mx4_quantize_kernel<bf16_t>), grid, dim3(256), 0, stream,
                           static_cast<const bf16_t *>(Bc), w, n, codes, scales);
    else
        hipLaunchKernelGGL((nm_mx4_quantize_kernel<f16_t>), grid, dim3(256), 0, stream, static_cast<const f16_t *>(Bc),
                           w, n, codes, scales);
    return hipGetLastError() == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" nmspmm_status_t nmspmm_mx4_pack(const uint8_t *codes, const uint8_t *scales, const uint8_t *idx,
                                           const nmspmm_mx4_weight_t *weight, hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, 0);
    if (st != NMSPMM_OK) return st;
    const nmspmm_mx4_weight_t &w = *weight;
    if (w.k == 0 || w.n == 0) return NMSPMM_OK;
    if (!codes || !scales || (!idx && w.N != w.M) || !w.packed) return NMSPMM_ERR_INVALID_ARG;
    if (!aligned_to(w.packed, 256)) return NMSPMM_ERR_UNSUPPORTED;
    const Mx4Layout l = mx4_layout(w.k, w.n, w.N, w.M, w.V);
    const dim3 grid((unsigned)std::min<int64_t>(8192, (l.w * w.n + 511) / 512));
    uint8_t *out = static_cast<uint8_t *>(const_cast<void *>(w.packed));
    if (l.kind == Mx4Kind::Raw)
        hipLaunchKernelGGL(nm_mx4_pack_raw_kernel, grid, dim3(256), 0, stream, codes, scales, idx, out, l, w.n, w.M);
    else
        hipLaunchKernelGGL(nm_mx4_pack_kernel, grid, dim3(256), 0, stream, codes, scales, idx, out, l, w.n, w.N, w.M, w.V);
    return hipGetLastError() == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" int64_t nmspmm_mx4_workspace_bytes(int64_t m, const nmspmm_mx4_weight_t *weight)
{
    if (check_weight(weight, m) != NMSPMM_OK) return -1;
    if (m == 0 || weight->n == 0 || weight->k == 0) return 0;
    return mx4_plan(m, mx4_layout(weight->k, weight->n, weight->N, weight->M, weight->V), *weight, true).ws_bytes;
}

extern "C" const char *nmspmm_mx4_kernel_name(int64_t m, const nmspmm_mx4_weight_t *weight, int with_workspace)
{
    if (check_weight(weight, m) != NMSPMM_OK) return "invalid";
    if (m == 0 || weight->n == 0) return "none";
    const Mx4Layout l = mx4_layout(weight->k, weight->n, weight->N, weight->M, weight->V);
    const Mx4Plan c = mx4_plan(m, l, *weight, with_workspace != 0);
    if (c.general) return "nm_mx4_general_kernel";
    thread_local char buf[128];
    if (l.kind == Mx4Kind::Dense)
        std::snprintf(buf, sizeof buf, "nm_mx4_dense_kernel<mt%d,ct%d>,split%d", c.MT, c.CT, c.splits);
    else
        std::snprintf(buf, sizeof buf, "%s<mt%d,ct%d,wc%d>,rows%d,chunk%d,split%d",
                      c.MT > 1 ? "nm_mx4_wide_kernel" : "nm_mx4_sparse_kernel", c.MT, c.CT, c.WC, c.rows, c.chunk, c.splits);
    return buf;
}

extern "C" nmspmm_status_t nmspmm_mx4_run(const void *A, int64_t lda, nmspmm_dtype_t a_dtype,
                                          const nmspmm_mx4_weight_t *weight, void *C, int64_t ldc,
                                          nmspmm_dtype_t c_dtype, int64_t m, float alpha, const float *bias,
                                          nmspmm_half_act_t act, const void *mul, int64_t ld_mul, const void *residual,
                                          int64_t ld_residual, void *workspace, size_t workspace_bytes,
                                          hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, m);
    if (st != NMSPMM_OK) return st;
    const nmspmm_mx4_weight_t &w = *weight;
    if ((a_dtype != NMSPMM_BF16 && a_dtype != NMSPMM_F16) || (c_dtype != NMSPMM_F32 && c_dtype != a_dtype) ||
        act < NMSPMM_HALF_ACT_NONE || act > NMSPMM_HALF_ACT_SILU)
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
    const Mx4Layout l = mx4_layout(w.k, w.n, w.N, w.M, w.V);
    if (m == 1) lda = w.k;
    const auto rows16 = [cs](const void *ptr, int64_t ld) { return !ptr || (aligned_to(ptr, 16) && ld * cs % 16 == 0); };
    const HalfEpilogue epi = {C, bias, mul, residual, ldc, ld_mul, ld_residual, alpha, act, c_dtype == NMSPMM_F32,
                              rows16(C, ldc) && rows16(mul, ld_mul) && rows16(residual, ld_residual) &&
                                  aligned_to(bias, 16)};
    int cached = -1;
    Mx4Plan c = mx4_plan(m, l, w, true);
    if (c.ws_bytes > 0 && (!workspace || (uint64_t)c.ws_bytes > (uint64_t)workspace_bytes)) {
        workspace = capturing(stream) ? nullptr : ws_acquire(stream, (size_t)c.ws_bytes, &cached);
        if (!workspace) c = mx4_plan(m, l, w, false);
    }
    hipError_t e;
    if (c.general) {
        const Mx4GeneralArgs p{A, static_cast<const unsigned char *>(w.packed), l, lda, m, w.n, w.N, w.M, w.V, epi, 0};
        e = a_dtype == NMSPMM_BF16 ? launch_general<bf16_t>(p, stream) : launch_general<f16_t>(p, stream);
    } else {
        e = a_dtype == NMSPMM_BF16 ? run_tiles<bf16_t>(c, l, A, lda, w, m, epi, workspace, stream)
                                   : run_tiles<f16_t>(c, l, A, lda, w, m, epi, workspace, stream);
    }
    const hipError_t f = cached >= 0 ? ws_done(cached, stream) : hipSuccess;
    return e == hipSuccess && f == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}
