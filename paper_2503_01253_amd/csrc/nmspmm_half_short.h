// Kernel of the 16-bit N:M product for up to 16 rows (device code), bound by
// the weight's bytes and by latency.
//
// A workgroup of eight waves owns MI columns (one tile of packed operands) and
// all rows of C.  The waves share out the units of every chunk of k, so that a
// workgroup's operands are asked for by eight waves at once, D steps of each
// ahead, before anything else is waited for.
//   A_s : the rows of A over one chunk of columns (all of k for a few rows),
//         row-major as it lies in memory, by 16-byte buffer -> LDS DMA; the
//         next chunk lands in the second slot meanwhile.
//   gather: eight 2-byte LDS reads make an A operand (a row a lane; rows
//         start four banks apart).  The tiled kernel's transposed reads need
//         A_s k-major, 32 rows wide whatever m is, and a transposition first.
// The waves' sums meet in LDS and are added in their order; one output a
// thread goes through the epilogue.  1 x 8192 x 8192 at 4:32 takes 7.2 us (2.3
// TB/s of weight), 1 x 4096 x 11008 at 8:32 10.3 with its launch; the tiled
// kernel 16.5 on the former.  A weight whose operands hold padding rows
// (which would need zeros in A_s) takes the tiled kernel.
#ifndef NMSPMM_HALF_SHORT_H
#define NMSPMM_HALF_SHORT_H

#include "nmspmm_half_tile.h"

namespace nmspmm {

constexpr int HS_NW = 8, HS_NT = 64 * HS_NW, HS_D = 8, HS_ROWS = 16;
// A chunk of A: two slots, and two workgroups a CU, or one where there are no
// more than CUs (16 x 8192 x 8192 at 4:32, 256 workgroups: 8 chunks 12.5 us, 4
// chunks 11.9).
constexpr int HS_SLOT = 38 * 1024, HS_SLOT_WIDE = 76 * 1024;

struct HalfShortArgs {
    const void *A;
    const unsigned char *vals;
    const uint16_t *offs;
    int64_t lda, n, k;
    int32_t m, V, S, KR, steps;
    int32_t chunk_units, chunks;        // units a chunk (a multiple of HS_NW) and chunks
    HalfEpilogue epi;
};

// Bytes of a row of A_s: rows start four banks apart.
__host__ __device__ constexpr int half_short_pitch(int units, int KR) { return (units * KR * 2 + 127) / 128 * 128 + 16; }

template <class T, int MI, int SLOT>
__global__ __launch_bounds__(HS_NT, SLOT == HS_SLOT ? 4 : 2) void nm_half_short_kernel(HalfShortArgs p)
{
    typedef typename MfmaAcc<MI>::type acc_t;
    constexpr int E = MfmaAcc<MI>::E, STEP = 512 / MI;
    static_assert(HS_NW * MI * MI * 4 <= 2 * SLOT && HS_ROWS <= MI, "LDS");
    __shared__ __align__(256) unsigned char lds[2 * SLOT];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t tile = blockIdx.x;

    // ---- B operands and offsets ----
    const __amdgpu_buffer_rsrc_t b_rsrc = make_rsrc(p.vals + (int64_t)tile * p.steps * 1024, (uint32_t)p.steps * 1024);
    const unsigned char *op = reinterpret_cast<const unsigned char *>(p.offs) +
                              (int64_t)(tile * MI / p.V) * (p.steps + 1) * (2 * STEP) + lane / MI * 16;
    const int per = p.chunk_units / HS_NW * p.S;        // steps a wave takes of a chunk
    s16x8 rb[HS_D];
    u32x4 ro[HS_D];
    auto step_of = [&](int chunk, int q) { return chunk * p.chunk_units * p.S + wave * per + q; };
    auto load_b = [&](int i, int chunk, int q) {
        const uint32_t step = q < per ? (uint32_t)step_of(chunk, q) : (uint32_t)p.steps;    // past the last: zeros
        rb[i] = __builtin_bit_cast(s16x8, __builtin_amdgcn_raw_buffer_load_b128(b_rsrc, (int)(step * 1024 + lane * 16), 0, 0));
        ro[i] = *reinterpret_cast<const u32x4 *>(op + (int64_t)min(step, (uint32_t)p.steps) * (2 * STEP));
    };

    // ---- A: a few waves a row, or a few rows a wave ----
    const int row_bytes = p.chunk_units * p.KR * 2, pitch = half_short_pitch(p.chunk_units, p.KR);
    // (k is a multiple of 8 here, of whole units, so no row ends inside a word)
    const __amdgpu_buffer_rsrc_t a_rsrc = make_rsrc(p.A, (uint32_t)(((p.m - 1) * p.lda + p.k) * 2));
    const int share = p.m == 1 ? 3 : p.m == 2 ? 2 : p.m <= 4 ? 1 : 0;      // log2 of the waves of a row
    auto load_a = [&](int chunk, int slot) {
        for (int row = wave >> share; row < p.m; row += HS_NW >> share)
            for (int at = (wave & ((1 << share) - 1)) * 1024; at < row_bytes; at += 1024 << share) {
                const int64_t c = (int64_t)chunk * row_bytes + at + lane * 16;
                // (columns past k, of the last chunk, belong to no step that is computed)
                if (at + lane * 16 < row_bytes && c < p.k * 2)
                    lds_dma<16>(a_rsrc, lds + slot * SLOT + row * pitch + at, (uint32_t)(row * p.lda * 2 + c));
            }
    };

    load_a(0, 0);
    asm volatile("" ::: "memory");      // the slab of A, then exactly 2 * HS_D loads
#pragma unroll
    for (int i = 0; i < HS_D; ++i) load_b(i, 0, i);
    asm volatile("" ::: "memory");
    acc_t acc;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;

    // a lane's row of A_s (rows past the last read the last: their outputs are not stored)
    const int a_row = min(lane % MI, p.m - 1) * pitch;
    const int first_unit = wave * (p.chunk_units / HS_NW);
    auto compute = [&](int i, int chunk, int q, int slot) {     // q: the step within the wave's steps of the chunk
        if (step_of(chunk, q) >= p.steps) return;
        const int base = slot * SLOT + a_row + (first_unit + q / p.S) * p.KR * 2;
        s16x8 a;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t v = j < 4 ? ro[i][j] & 0xffffu : ro[i][j - 4] >> 16;
            a[j] = *reinterpret_cast<const short *>(lds + base + (v >> 3) * 2);
        }
        acc = half_mfma<T, MI>(a, rb[i], acc);
    };

    // slot i of the ring holds the steps i, i + D, ... of a chunk, then step i of the next
    for (int chunk = 0; chunk < p.chunks; ++chunk) {
        if (chunk == 0) {
            static_assert(2 * HS_D == 16, "the count below");
            // all but the 16 youngest loads: the slab of A, and not the operands
            __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8) | (1 << 14));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        } else {
            stage_sync();
        }
        if (chunk + 1 < p.chunks) load_a(chunk + 1, (chunk + 1) & 1);
        int q = 0;
        for (; q + HS_D <= per; q += HS_D) {
#pragma unroll
            for (int i = 0; i < HS_D; ++i) {
                compute(i, chunk, q + i, chunk & 1);
                const bool same = q + i + HS_D < per;
                load_b(i, same ? chunk : chunk + 1, same ? q + i + HS_D : i);
            }
        }
#pragma unroll
        for (int i = 0; i < HS_D; ++i)
            if (q + i < per) {
                compute(i, chunk, q + i, chunk & 1);
                load_b(i, chunk + 1, i);
            }
    }

    // ---- the waves' sums, added in their order ----
    lds_sync();
    float *red = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int e = 0; e < E; ++e) red[(wave * E + e) * 64 + lane] = acc[e];
    lds_sync();
    for (int i = tid; i < p.m * MI; i += HS_NT) {
        const int row = i / MI, col = i % MI;
        const int e = MI == 32 ? row / 8 * 4 + row % 4 : row % 4, at = MI == 32 ? row / 4 % 2 * 32 + col : row / 4 * 16 + col;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < HS_NW; ++w) sum += red[(w * E + e) * 64 + at];
        const int64_t j = (int64_t)tile * MI + col;
        if (p.epi.f32) half_store<float>(p.epi, row, j, sum);
        else half_store<T>(p.epi, row, j, sum);
    }
}

}  // namespace nmspmm

#endif
