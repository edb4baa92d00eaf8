// Tiled kernel of the 16-bit N:M product (device code, included by the units
// that instantiate it).
//
// The packed weight (nmspmm_half_pack) holds the matrix instruction's B
// operands as its lanes read them.  MI columns (32 where V is a multiple of
// 32, else 16) and STEP = 512/MI compressed rows make one operand: 64 lanes of
// eight consecutive rows, 1 KB in one piece.  Compressed rows are counted in
// units of G whole windows (KR = G*M columns of A, G*N rows padded to S
// operands), and every padding row has an offset of its own kind.
//
// A workgroup of WR x WC x WK waves owns BM x BN outputs (and, with split-k,
// one slice of k).  It walks k in stages of P units:
//   A_s : the BM x P*KR slab of A in LDS, k-major: row c holds column c of A,
//         BM rows of C, 16 to a granule of 32 bytes; after every unit one row
//         of zeros, where padding offsets lead, so that no value of A meets a
//         padding row's zero.  Global -> registers (4 rows x 8 columns a
//         block) -> transposed by byte permutes -> LDS: two slots, and the
//         AD slabs after them on their way to registers.
//   gather: ds_read_b64_tr_b16 hands 16 lanes four LDS rows of 16 outputs,
//         each row at its own address, already transposed into the A operand:
//         the gather of Eq. 1 costs nothing beyond the read.
//   B, offsets: straight from memory into registers, one stage ahead (a stage
//         has a fixed number of operands a wave, QS, so that every wait counts
//         the loads that are younger exactly; with a run-time number, each wait
//         for B waited for the slab of A that had just been asked for as well:
//         4096^3 at 16:32 174 us, with fixed stages 151).
// Granule g of a unit's row c lies at place g ^ swz(c), which spreads reads and
// writes over the banks; the packed offset holds swz(c) beside c, so that a
// lane forms its address with four instructions.  The WK waves of a tile share
// out the units of every stage and are joined through LDS at the end.
//
// 4096^3 at 16:32 takes 93-95 us in the kernel with V = 32 (730 TFLOP/s useful),
// 88 with V = 64 and two operands a gather, 2048 x 4096 x 11008 at 8:32 97: at 2.2
// GHz, matrix instructions 32 % busy, LDS 34 % (24 with V = 64).  Little overlaps:
// in a row of calls (101 us, V = 32) a copy takes 89 us without A's loads, 75
// without its LDS writes too, 92 without B, 42 without gathers and matrix
// instructions, 18 without all of them.
#ifndef NMSPMM_HALF_TILE_H
#define NMSPMM_HALF_TILE_H

#include "nmspmm_half.h"
#include "nmspmm_tiled.h"

namespace nmspmm {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) unsigned char lds_u8;

struct HalfTileArgs {
    const void *A;
    const unsigned char *vals;
    const uint16_t *offs;
    float *part;            // with split-k: splits x m x n partial sums
    int64_t lda, m, n, k;
    int32_t V, S, KR, P, steps, nst;     // S operands a unit, P units a stage, `steps` operands a column tile
    int32_t tiles_m, tiles_n, splits;
    HalfEpilogue epi;
};

template <int MI> struct MfmaAcc;
template <> struct MfmaAcc<32> { typedef f32x16 type; static constexpr int E = 16; };
template <> struct MfmaAcc<16> { typedef f32x4 type; static constexpr int E = 4; };

template <class T, int MI>
__device__ __forceinline__ typename MfmaAcc<MI>::type half_mfma(s16x8 a, s16x8 b, typename MfmaAcc<MI>::type c)
{
    if constexpr (__is_same(T, bf16_t)) {
        const bf16x8 x = __builtin_bit_cast(bf16x8, a), y = __builtin_bit_cast(bf16x8, b);
        if constexpr (MI == 32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    } else {
        const f16x8 x = __builtin_bit_cast(f16x8, a), y = __builtin_bit_cast(f16x8, b);
        if constexpr (MI == 32) return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
    }
}

// The shape of a tile: MI x MI accumulators, RT of them down a wave's rows and
// CT across the columns of each of its NG gathers; NB blocks of A a thread
// and stage; LDS_KB of LDS.
template <int MI_, int CT_, int NG_, int RT_, int WR_, int WC_, int WK_, int NB_, int AD_, int LDS_KB_>
struct HalfTile {
    static constexpr int MI = MI_, CT = CT_, NG = NG_, RT = RT_, WR = WR_, WC = WC_, WK = WK_, NB = NB_, AD = AD_;
    static constexpr int BM = MI * RT * WR, BN = MI * CT * NG * WC, NT = 64 * WR * WC * WK;
    static constexpr int STEP = 512 / MI, PSHIFT = BM == 128 ? 8 : BM == 64 ? 7 : 6, PITCH = 1 << PSHIFT,
                         LDS_BYTES = 1024 * LDS_KB_;
    static constexpr int ACCS = RT * CT * NG;
    // waves a SIMD: two workgroups a CU where their LDS leaves room
    static constexpr int WPS = NT / 256 * (160 / LDS_KB_);
    static constexpr int RED_BYTES = WK > 1 ? (WK / 2) * WR * WC * ACCS * MI * MI * 4 : 0;
    static constexpr int CW = CT * NG * MI, CPITCH = CW + 8;        // a wave's columns, and rows 4 apart on other banks
    static_assert((RT & (RT - 1)) == 0 && PITCH == 2 * BM && RED_BYTES <= LDS_BYTES && WR * WC * (MI * CPITCH * 4 + 4 * MI * CW) <= LDS_BYTES &&
                      64 / (CW / 8) <= MI, "tile shape");
    // rows of a slot, and columns of A of a stage, at most
    static constexpr int ROWS = LDS_BYTES / 2 / PITCH, KMAX = NB * NT / (2 * BM) * 64;
    // the bits of swz(c) that a row of BM outputs has room for
    static constexpr int SWZ = BM / 16 - 1 < 7 ? BM / 16 - 1 : 7;
};

// What the granules of a unit's row c are XORed with: rows next to each other
// (of a transposed read) and rows 8 apart (of a write) lie on different banks.
__host__ __device__ constexpr int half_swz(int c) { return (c ^ (c >> 3)) & 7; }

// Columns 4*half .. 4*half+3 of 4 rows x 8 columns of 16-bit values: out[j]
// holds column 4*half + j.
__device__ __forceinline__ void transpose_4x4(const u32x4 (&r)[4], int half, u32x2 (&out)[4])
{
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int w = 2 * half + j;
        out[2 * j] = u32x2{__builtin_amdgcn_perm(r[1][w], r[0][w], 0x05040100u),
                           __builtin_amdgcn_perm(r[3][w], r[2][w], 0x05040100u)};
        out[2 * j + 1] = u32x2{__builtin_amdgcn_perm(r[1][w], r[0][w], 0x07060302u),
                               __builtin_amdgcn_perm(r[3][w], r[2][w], 0x07060302u)};
    }
}

template <class T, class C, int QS, bool VEC>
__global__ __launch_bounds__(C::NT, C::WPS) void nm_half_tile_kernel(HalfTileArgs p)
{
    constexpr int MI = C::MI, CT = C::CT, NG = C::NG, RT = C::RT, WR = C::WR, WC = C::WC, WK = C::WK, NB = C::NB, AD = C::AD;
    constexpr int BM = C::BM, BN = C::BN, NT = C::NT, STEP = C::STEP, PITCH = C::PITCH;
    typedef typename MfmaAcc<MI>::type acc_t;
    constexpr int E = MfmaAcc<MI>::E;
    __shared__ __align__(256) unsigned char lds[C::LDS_BYTES];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wk = wave / (WR * WC), wr = wave / WC % WR, wc = wave % WC;
    int tm, tn, split;
    map_tile(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_n, tm, tn, split);
    const int64_t row0 = (int64_t)tm * BM, col0 = (int64_t)tn * BN;
    const int sps = (p.nst + p.splits - 1) / p.splits;
    const int s_begin = split * sps, s_end = min(p.nst, s_begin + sps);

    // ---- A: global -> registers -> LDS ----
    const int kstage = p.P * p.KR, slot_bytes = p.P * (p.KR + 1) * PITCH;
    const int rows_valid = (int)min64(BM, p.m - row0);
    // (rows past the last and columns past k read zeros or a neighbour's
    // values: the former's outputs are not stored, no offset leads to the latter.
    // Wide loads are checked by whole words of 4 bytes: an odd k's last value
    // needs the word it lies in, which starts inside A)
    const uint32_t a_bytes = (uint32_t)(((rows_valid - 1) * p.lda + p.k) * 2);
    const __amdgpu_buffer_rsrc_t a_rsrc = make_rsrc(static_cast<const T *>(p.A) + row0 * p.lda,
                                                    VEC ? (a_bytes + 3) & ~3u : a_bytes);
    u32x4 ra[AD][NB][4];
    uint32_t a_off[NB], a_dst[NB];
    // block b of this thread: rows 4*rb.., columns 8*kc.. of the stage.  A wave
    // takes eight pieces of a row: whole 128-byte lines of A (halves of lines in
    // different instructions waited for each other in L1); 16 of its lanes four
    // pieces of four blocks of rows, which a cycle of a write finds on different
    // banks (two of eight took twice the cycles).
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int x = tid + b * NT, rb = ((x >> 2) & 3) + 4 * ((x >> 5) % (BM / 16));
        const int kc = (x & 3) + 4 * ((x >> 4) & 1) + 8 * (x / (2 * BM));
        const int unit = 8 * kc / p.KR, c = 8 * kc - unit * p.KR;
        a_off[b] = 8 * kc < kstage ? (uint32_t)((4 * rb * p.lda + 8 * kc) * 2) : OOB;
        a_dst[b] = 8 * kc < kstage ? (uint32_t)((unit * (p.KR + 1) + c) * PITCH +
                                                (((rb >> 2) ^ (half_swz(c) & C::SWZ)) << 5) + 8 * (rb & 3)) : OOB;
    }
    constexpr int PAST = 0x40000000;    // past every tile's rows of A (under 2^29 bytes), and no overflow beside OOB
    auto load_a = [&](int d, int b, int st) {
        const int at = st < s_end ? st * kstage * 2 : PAST;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t off = a_off[b] + (uint32_t)(r * p.lda * 2);
            if constexpr (VEC) {
                ra[d][b][r] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, (int)a_off[b], (int)(at + r * (int)p.lda * 2), 0));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t lo = __builtin_amdgcn_raw_buffer_load_b16(a_rsrc, (int)(off + 4 * j), at, 0);
                    const uint32_t hi = __builtin_amdgcn_raw_buffer_load_b16(a_rsrc, (int)(off + 4 * j + 2), at, 0);
                    ra[d][b][r][j] = (lo & 0xffffu) | hi << 16;
                }
            }
        }
    };
    // half a block: four columns
    auto store_a = [&](int d, int b, int half, int slot) {
        u32x2 col[4];
        transpose_4x4(ra[d][b], half, col);
        if (a_dst[b] != OOB) {
            unsigned char *dst = lds + slot * slot_bytes;
#pragma unroll
            for (int j = 4 * half; j < 4 * half + 4; ++j)
                *reinterpret_cast<u32x2 *>(dst + j * PITCH + (a_dst[b] ^ ((j & C::SWZ) << 5))) = col[j - 4 * half];
        }
    };

    // ---- B operands and offsets, one stage ahead: a wave takes QS steps in a
    // row of every stage.  Past a tile's last operand the loads read zeros,
    // and the offsets those of padding ----
    const uint32_t ctiles = (uint32_t)(p.n / MI);
    __amdgpu_buffer_rsrc_t b_rsrc[NG][CT];
    const unsigned char *op[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        const uint32_t first = (uint32_t)(col0 / MI) + (wc * NG + g) * CT;
#pragma unroll
        for (int c = 0; c < CT; ++c)
            b_rsrc[g][c] = make_rsrc(p.vals + (int64_t)min(first + c, ctiles - 1) * p.steps * 1024,
                                     (uint32_t)p.steps * 1024);
        op[g] = reinterpret_cast<const unsigned char *>(p.offs) +
                (int64_t)(min(first, ctiles - 1) * MI / p.V) * (p.steps + 1) * (2 * STEP);
    }
    const uint32_t pair = ((lane / MI) * 4 + ((lane >> 2) & 3)) * 4;
    s16x8 rb_[QS][NG][CT];
    uint32_t ro[QS][NG];
    auto load_b = [&](int i, int st) {
        const uint32_t step = (uint32_t)(st * p.P * p.S + wk * QS + i);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            ro[i][g] = *reinterpret_cast<const uint32_t *>(op[g] + min(step, (uint32_t)p.steps) * (2 * STEP) + pair);
#pragma unroll
            for (int t = 0; t < CT; ++t)
                rb_[i][g][t] = __builtin_bit_cast(s16x8, __builtin_amdgcn_raw_buffer_load_b128(b_rsrc[g][t], (int)(step * 1024 + lane * 16), 0, 0));
        }
    };

    acc_t acc[NG][RT][CT];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[g][t][c][e] = 0.f;

    // where a lane of a transposed read looks: its piece of 4 outputs in its
    // granule (MI = 32: of a pair)
    const int piece = 8 * (lane & 3);
    constexpr int TSHIFT = MI == 32 ? 6 : 5;
    const int g0 = (wr * RT << TSHIFT) + (MI == 32 ? 32 * ((lane >> 4) & 1) : 0);

    auto compute = [&](int i, uint32_t slot) {
        const uint32_t base = slot + (uint32_t)(wk * QS + i) / (uint32_t)p.S * (p.KR + 1) * PITCH;  // the step's unit
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            uint32_t at[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t v = x == 0 ? ro[i][g] & 0xffffu : ro[i][g] >> 16;    // row * 8 + swz(row)
                const uint32_t place = PITCH == 256 ? v << 5 : (v >> 3 << C::PSHIFT) + ((v & C::SWZ) << 5);
                at[x] = (place ^ (g0 + piece)) + base;
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                s16x4 v[2];
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    v[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds_u8 *)(uintptr_t)(at[x] ^ (t << TSHIFT)));
                const s16x8 a = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) acc[g][t][ct] = half_mfma<T, MI>(a, rb_[i][g][ct], acc[g][t][ct]);
            }
        }
    };

    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8 *)(lds_void *)lds;
    if (s_begin < s_end) {
        // the rows of zeros of both slots' units
        for (int i = tid; i < 2 * p.P * (PITCH / 4); i += NT) {
            const int unit = i / (PITCH / 4);
            *reinterpret_cast<uint32_t *>(lds + (unit * (p.KR + 1) + p.KR) * PITCH + i % (PITCH / 4) * 4) = 0;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) load_a(0, b, s_begin);
#pragma unroll
        for (int i = 0; i < QS; ++i) load_b(i, s_begin);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            store_a(0, b, 0, 0);
            store_a(0, b, 1, 0);
        }
#pragma unroll
        for (int d = 1; d <= AD; ++d)
#pragma unroll
            for (int b = 0; b < NB; ++b) load_a(d % AD, b, s_begin + d);
        lds_sync();
        // (debug build) NaN in the places that this thread's next stores will fill
        auto poison_a = [&](int slot) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
                if (a_dst[b] != OOB)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<u32x2 *>(lds + slot * slot_bytes + j * PITCH + (a_dst[b] ^ ((j & C::SWZ) << 5))) =
                            u32x2{0x7fff7fffu, 0x7fff7fffu};
            asm volatile("" ::: "memory");
        };
        // the next stage's slab, which has been on its way for AD stages, is
        // written a part a step, and each block's registers take the one AD
        // stages on
        auto stage = [&](int st, int d, int slot) {
            if constexpr (NMSPMM_POISON_LDS) poison_a(slot ^ 1);
#pragma unroll
            for (int i = 0; i < QS; ++i) {
#pragma unroll
                for (int part = i * 2 * NB / QS; part < (i + 1) * 2 * NB / QS; ++part) {
                    store_a(d, part / 2, part % 2, slot ^ 1);
                    if (part % 2) load_a(d, part / 2, st + 1 + AD);
                }
                compute(i, lds0 + slot * slot_bytes);
                load_b(i, st + 1);
            }
            lds_sync();
        };
        for (int st = s_begin; st < s_end; st += 2) {
            stage(st, 1 % AD, 0);
            if (st + 1 < s_end) stage(st + 1, 0, 1);
        }
    }

    // ---- the WK waves of a tile, joined in a fixed order ----
    if constexpr (WK > 1) {
        float *red = reinterpret_cast<float *>(lds);
        const int pos = wr * WC + wc;
#pragma unroll
        for (int half = WK / 2; half >= 1; half /= 2) {
            lds_sync();
            float *mine = red + (((wk >= half ? wk - half : wk) * WR * WC + pos) * C::ACCS * E) * 64 + lane;
            if (wk >= half && wk < 2 * half) {
                int i = 0;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int t = 0; t < RT; ++t)
#pragma unroll
                        for (int c = 0; c < CT; ++c)
#pragma unroll
                            for (int e = 0; e < E; ++e) mine[64 * i++] = acc[g][t][c][e];
            }
            lds_sync();
            if (wk < half) {
                int i = 0;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int t = 0; t < RT; ++t)
#pragma unroll
                        for (int c = 0; c < CT; ++c)
#pragma unroll
                            for (int e = 0; e < E; ++e) acc[g][t][c][e] += mine[64 * i++];
            }
        }
    }

    // ---- C: every wave turns its accumulators, MI rows at a time, in a piece
    // of LDS of its own, so that a lane stores eight columns of one row.
    // Element e of lane l: row 8*(e/4) + 4*(l/32) + e%4 (MI = 32) or
    // 4*(l/16) + e of the accumulator, column l % MI ----
    lds_sync();
    if (wk > 0) return;
    constexpr int CW = C::CW, CP = C::CPITCH, LPR = CW / 8, RPP = 64 / LPR;
    float *turn = reinterpret_cast<float *>(lds) + wave * (MI * CP);
    const int64_t j = col0 + wc * CW + lane % LPR * 8;
    // What the epilogue reads of mul (or residual) comes by DMA into LDS, the
    // rows of two accumulators at once, each lane's pieces where it will look
    // for them: loaded where they are used, eight waves a CU had too few bytes
    // on their way (2048 x 4096 x 11008 at 8:32 with a factor 129 us, 125 so;
    // 4096^3 at 16:32 with a term 108 and 103).
    constexpr int PIECES = MI / RPP, AHEAD = 2 * MI * CW * 2;      // a lane's of an accumulator; bytes of a wave
    unsigned char *fetched = lds + WR * WC * (MI * CP * 4) + wave * AHEAD;
    const void *other = p.epi.mul ? p.epi.mul : p.epi.residual;
    const int64_t ld_other = p.epi.mul ? p.epi.ld_mul : p.epi.ld_residual;
    const bool fetch = other && p.epi.vec && !p.epi.f32 && p.splits == 1 && ld_other < (int64_t)1 << 21;
    const __amdgpu_buffer_rsrc_t o_rsrc =
        make_rsrc(static_cast<const T *>(other) + row0 * ld_other + col0,
                  fetch ? (uint32_t)(((rows_valid - 1) * ld_other + min64(BN, p.n - col0)) * 2) : 0u);
    // One copy of the code: unrolled over the row tiles it was larger than the
    // instruction cache, and fetching it cost 40 us at 4096^3.  The row tiles
    // move down through the first one's registers.
#pragma unroll 1
    for (int t = 0; t < RT; ++t) {
        if (fetch && t % 2 == 0) {
#pragma unroll 1
            for (int u = 0; u < 2 * PIECES; ++u) {      // (rows past the last: zeros)
                const int r = (wr * RT + t) * MI + u * RPP + lane / LPR;
                const uint32_t off = r < rows_valid && j < p.n ? (uint32_t)((r * ld_other + j - col0) * 2) : OOB;
                lds_dma<16>(o_rsrc, fetched + u * 1024, off);
            }
        }
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int r = MI == 32 ? 8 * (e / 4) + 4 * (lane / 32) + e % 4 : 4 * (lane / 16) + e;
                    turn[r * CP + (g * CT + c) * MI + lane % MI] = acc[g][0][c][e];
                }
        asm volatile("" ::: "memory");
        if (fetch && t % 2 == 0) {
            __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8) | (0 << 14));     // vmcnt(0)
            asm volatile("" ::: "memory");
        }
#pragma unroll 1
        for (int r = lane / LPR; r < MI; r += RPP) {
            const int64_t i = row0 + (wr * RT + t) * MI + r;
            float x[8];
            load_row<8, true>(turn + r * CP + lane % LPR * 8, 8, x);
            if (i < p.m && j < p.n) {
                if (p.splits > 1) store_row<8, true>(p.part + ((int64_t)split * p.m + i) * p.n + j, 8, x);
                else if (p.epi.f32) half_store8<float>(p.epi, i, j, x);
                else half_store8<T>(p.epi, i, j, x, fetch ? reinterpret_cast<const T *>(
                         fetched + (t % 2 * PIECES + r / RPP) * 1024 + lane * 16) : nullptr);
            }
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int u = 0; u + 1 < RT; ++u)
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int c = 0; c < CT; ++c) acc[g][u][c] = acc[g][u + 1][c];
    }
}

}  // namespace nmspmm

#endif
