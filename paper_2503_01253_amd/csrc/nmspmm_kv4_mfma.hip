// nmspmm_kv4_attend on the matrix cores: pages of whole fours of tokens, at most
// 256 dimensions.
//
// A workgroup of four waves takes a tile of 16 query heads of one cache head
// (fewer leave columns unused) and a chunk of one sequence, a wave 32 tokens at a
// time, all of it in registers:
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16: A operand 16 tokens, a group of 32
//                 dimensions, whose word of eight codes a lane converts with the
//                 group's scale in four instructions (what codes stand for is exact in
//                 bf16); B operand the queries, in as many bf16 parts as hold their bits;
//   P^T           running maximum of each head (a lane's column), weights in fp32;
//   O^T += V^T P^T  the weights lie in the lanes just as the B operand wants them (k
//                 index 8g+j stands for token 4g+j, or 16+4g+j-4 from j = 4 on), in
//                 three bf16 parts, all 24 bits.  The page holds the words of four
//                 tokens side by side, so that a lane reads those of its eight tokens for
//                 its eight dimensions in two pieces, and a permute brings the values of
//                 two tokens together: nothing goes through LDS.
// The next tokens' codes are on their way meanwhile, their pages looked up before.
// The waves are joined in LDS.
// 128 x 8192 positions, 32 heads on 8 of 128, 218-222 us (5.2 TB/s), one sequence of
// 131071, 64 heads on 8, 37-38 with its joining (3.8 TB/s).  A tile of 32 tokens takes a
// SIMD some 230 vector and 32 matrix instructions, 0.5 us of them alone, and 4.3 KB, 0.2
// us at the HBM's rate: four waves a SIMD keep enough of them on their way.  Two tiles
// ahead a wave took the registers of a fourth wave (219 -> 225 us).
#include "nmspmm_kv4.h"

namespace nmspmm {
namespace {

typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int A4M_NW = 4, A4M_NT = 64 * A4M_NW, A4M_TOKENS = 32;

__device__ __forceinline__ f32x4 mfma_bf16(s16x8 a, s16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// x as PARTS bf16 values, each the leading eight bits of what those before it
// leave: three hold all 24 bits of an fp32 value, two an fp16 one's, and all have
// its sign, so that no product of theirs that overflows meets one of the other sign.
template <int PARTS>
__device__ __forceinline__ void split_parts(float x, short *part)
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        const uint32_t h = __builtin_bit_cast(uint32_t, x);
        part[i] = (short)(h >> 16);
        if (i + 1 < PARTS) x -= __builtin_bit_cast(float, h & 0xffff0000u);
    }
}

// The values of the lanes 16 and 32 away: after the swap one result holds the
// even rows' value in both rows of a pair, the other the odd rows'.
template <class F>
__device__ __forceinline__ float across_groups(float x, F f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float y = f(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    const uint32_t v = __builtin_bit_cast(uint32_t, y);
    auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

// Byte B of a word, as the values of its two codes in bf16.
template <int B>
__device__ __forceinline__ uint32_t two_values(uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}

__device__ __forceinline__ s16x8 eight_values(uint32_t w, float scale)
{
    return __builtin_bit_cast(s16x8, u32x4{two_values<0>(w, scale), two_values<1>(w, scale), two_values<2>(w, scale),
                                           two_values<3>(w, scale)});
}

// The scale of group c of a row's bytes.
template <int C>
__device__ __forceinline__ float group_scale(const uint32_t *bytes)
{
    return mx4_scale<C % 4>(bytes[C / 4]);
}

// DK: groups of a row, 1 to 4, or 8 for any number from 5 to 8.  QP: parts of a
// query value.  PIECE: pages are of whole pieces of 16, 8 or 4 tokens.  The pages of
// pieces of 16 and 8 are looked up once a wave, those of 4 by every lane for itself.
template <int DK, int QP, int PIECE>
__global__ __launch_bounds__(A4M_NT, DK > 4 && QP > 2 ? 1 : DK > 4 || QP > 1 ? 2 : 3) void nm_attend4_mfma_kernel(AttendArgs p, Kv4Pages f)
{
    constexpr int GT = ATTEND_MFMA_HEADS, PP = 3;
    // the values' words of a lane (VU of them, dimension words 16 apart) and the codes
    // that it takes of each: with few groups, 16 / (4 DK) lanes share a word's codes
    constexpr int VU = DK == 8 ? 2 : 1, SHARE = DK == 1 ? 4 : DK == 2 ? 2 : 1, NI = 8 / SHARE, LD = 16 / SHARE;
    constexpr int NT = VU * NI, AP = DK * 32 + 4, SW = DK > 4 ? 2 : 1;
    __shared__ __align__(16) float acc[A4M_NW * GT * AP];
    __shared__ float2 s_ml[A4M_NW][GT];
    // A sequence's chunks start at one that differs from sequence to sequence: in the
    // same order, where their number divides the CUs', a CU meets first chunks only, or
    // last ones, which few sequences fill (192 sequences of 0 to 5000 positions in four
    // chunks 130 us, so 97).
    const uint32_t tiles = p.gtiles * p.heads, run = blockIdx.x / tiles, seq = run / p.splits;
    const uint32_t split = (run % p.splits + (seq * 0x9e3779b1u >> 20)) % p.splits;
    const AttendTask t = attend_task(p, (seq * p.splits + split) * tiles + blockIdx.x % tiles, GT);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 15, grp = lane >> 4;
    const int G = DK == 8 ? f.l.G : DK;

    // ---- the tokens.  What lies outside the chunk or in no page is left out by its
    // score and by zeros for its values: loads go to a place that is there (the
    // table's last position, the cache's first page) and wait for no comparison ----
    const int32_t *row = p.c.table + t.seq * p.c.table_stride;
    const unsigned char *blocks = f.pages + t.head * f.l.block;
    const int end = p.c.pages > 0 ? t.end : 0, last = p.cap - 1;
    // of the tile's pieces of PIECE tokens (4: of this lane's keys, then of its values):
    // the table's entries and the slots
    constexpr int PIECES = PIECE == 4 ? 4 : 32 / PIECE;
    struct Where {
        int32_t page[PIECES], slot[PIECES];
    };
    auto look_up = [&](int base) {
        Where w;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int pos = base + (PIECE > 4 ? i * PIECE : i < 2 ? 16 * i + col : 16 * (i - 2) + 4 * grp);
            const uint32_t in = (uint32_t)min(pos, last), at = p.c.size.div(in);
            w.page[i] = row[at];
            w.slot[i] = (int32_t)(in - at * p.c.size.d);
            if (PIECE > 4) w.slot[i] &= ~(PIECE - 1);       // (past the end: the last piece)
        }
        return w;
    };
    // (selections, no branches: what is selected is there)
    const uint32_t pages = (uint32_t)p.c.pages;
    auto held = [&](int32_t page) { return (uint32_t)page < pages; };
    // Where piece i starts, `at` bytes into its page's block and `unit` bytes a slot on:
    // the same for all lanes (but with pieces of 4), to which a lane adds its own bytes.
    auto start = [&](const Where &w, int i, int64_t at, uint32_t slots, uint32_t unit) {
        return blocks + (int64_t)(held(w.page[i]) ? w.page[i] : 0) * f.stride + at + slots * unit;
    };
    // of sixteen s, what a lane reads for its token (keys) or its four tokens (values)
    auto place = [&](const Where &w, int s, bool values, int64_t at, uint32_t unit, uint32_t mine) {
        const int shift = values ? 2 : 0;       // values: slots by fours
        if constexpr (PIECE == 16) return start(w, s, at, (uint32_t)w.slot[s] >> shift, unit) + mine;
        else if constexpr (PIECE == 8) {
            const unsigned char *one = start(w, 2 * s, at, (uint32_t)w.slot[2 * s] >> shift, unit);
            const unsigned char *two = start(w, 2 * s + 1, at, (uint32_t)w.slot[2 * s + 1] >> shift, unit);
            return ((values ? grp > 1 : col > 7) ? two : one) + mine;
        } else {
            const int i = (values ? 2 : 0) + s;
            return start(w, i, at, (uint32_t)w.slot[i] >> shift, unit) + mine;
        }
    };
    const uint32_t k_slot = PIECE == 16 ? col : PIECE == 8 ? col & 7 : 0, v_quad = PIECE == 16 ? grp : PIECE == 8 ? grp & 1 : 0;
    const uint32_t k_mine = k_slot * (16 * G) + grp * G * 4, ks_mine = k_slot * f.l.sp;
    uint32_t v_mine[VU], vs_mine[VU];
#pragma unroll
    for (int u = 0; u < VU; ++u) {
        // (lanes past a row's words read the last: their sums are not stored)
        const int D = min(col % LD + 16 * u, 4 * G - 1);
        v_mine[u] = v_quad * (64 * G) + D * 16;
        vs_mine[u] = v_quad * (4 * G) + D / 4 * 4;
    }
    // a bit for every token of the tile at base: in the chunk, and (with pieces of 4:
    // where this lane holds its values) in a page
    auto tokens = [&](const Where &w, int base) {
        const int lo = t.begin - base, hi = end - base;
        uint32_t bits = hi >= 32 ? ~0u : hi > 0 ? (1u << hi) - 1 : 0u;
        if (lo > 0) bits &= lo < 32 ? ~0u << lo : 0u;
        uint32_t there = 0;
#pragma unroll
        for (int i = 0; i < (PIECE == 4 ? 2 : PIECES); ++i) {
            const uint32_t of = PIECE == 16 ? 0xffffu : PIECE == 8 ? 0xffu : 0xfu << (4 * grp);
            const int page = w.page[PIECE == 4 ? 2 + i : i];
            there |= held(page) ? of << (PIECE == 4 ? 16 * i : PIECE * i) : 0u;
        }
        if (PIECE == 4) there |= ~(0xf000fu << (4 * grp));      // (other lanes' tokens)
        return bits & there;
    };
    // the first tile's entries are asked for together with the sequence's length
    Where first;
    if (p.cap > 0 && p.window == 0) first = look_up(t.split * p.chunk + wave * A4M_TOKENS);
    if (t.begin >= t.end && p.splits > 1) {      // nothing here: the maximum says so
        if (threadIdx.x < t.heads_in_tile) {
            const int64_t row = t.seq * ((int64_t)p.heads * p.group) + t.first_head + threadIdx.x;
            p.part_ml[row * p.splits + t.split] = make_float2(NEG_INF, 0.f);
        }
        return;
    }

    uint32_t kw[2][DK], ks[2][SW], vs[2][VU];
    u32x4 vw[2][VU];
    auto load_k = [&](const Where &w) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const unsigned char *at = place(w, s, false, 0, 16 * G, k_mine);
            if constexpr (DK <= 4) {
                __builtin_memcpy(kw[s], __builtin_assume_aligned(at, 4 * (DK & -DK)), 4 * DK);
            } else {
                if (G == 8) __builtin_memcpy(kw[s], __builtin_assume_aligned(at, 16), 32);
                else
#pragma unroll
                    for (int c = 0; c < DK; ++c) kw[s][c] = c < G ? *reinterpret_cast<const uint32_t *>(at + 4 * c) : 0u;
            }
            const unsigned char *sc = place(w, s, false, f.l.ks_at, f.l.sp, ks_mine);
            if constexpr (DK == 1) ks[s][0] = *sc;
            else if constexpr (DK == 2) ks[s][0] = *reinterpret_cast<const uint16_t *>(sc);
            else __builtin_memcpy(ks[s], __builtin_assume_aligned(sc, 4 * SW), 4 * SW);
        }
    };
    auto load_v = [&](const Where &w) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int u = 0; u < VU; ++u) {
                vw[s][u] = *reinterpret_cast<const u32x4 *>(place(w, s, true, f.l.v_at, 64 * G, v_mine[u]));
                vs[s][u] = *reinterpret_cast<const uint32_t *>(place(w, s, true, f.l.vs_at, 4 * G, vs_mine[u]));
            }
    };

    s16x8 q[QP][DK];
    auto load_q = [&]() {
#pragma unroll
        for (int c = 0; c < DK; ++c) {
            const int d = c * 32 + grp * 8, valid = col < t.heads_in_tile ? p.dim - d : 0;
            const int64_t at = t.seq * p.qs[0] + (t.first_head + col) * p.qs[1] + d;
            float x[8];
            if constexpr (QP == 1) {
                if (p.q_vec) load_row<8, true>(static_cast<const bf16_t *>(p.q) + at, valid, x);
                else load_row<8, false>(static_cast<const bf16_t *>(p.q) + at, valid, x);
            } else if constexpr (QP == 2) {
                if (p.q_vec) load_row<8, true>(static_cast<const f16_t *>(p.q) + at, valid, x);
                else load_row<8, false>(static_cast<const f16_t *>(p.q) + at, valid, x);
            } else {
                if (p.q_vec && p.dim % 8 == 0) load_row<8, true>(static_cast<const float *>(p.q) + at, valid, x);
                else load_row<8, false>(static_cast<const float *>(p.q) + at, valid, x);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                short part[QP];
                split_parts<QP>(x[j], part);
                const bool whole = fabsf(x[j]) == -NEG_INF;     // (of an infinity a difference leaves NaN)
#pragma unroll
                for (int i = 0; i < QP; ++i) q[i][c][j] = i > 0 && whole ? (short)0 : part[i];
            }
        }
    };

    f32x4 o[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = NEG_INF, l = 0.f;

    int base = (t.begin & ~(A4M_TOKENS - 1)) + wave * A4M_TOKENS;
    constexpr int STEP = A4M_NW * A4M_TOKENS;
    Where cur, next;        // of the tile that is in the registers, and of the one after it
    if (base < end) {
        cur = p.window > 0 ? look_up(base) : first;
        next = look_up(base + STEP);
        load_k(cur);
        load_v(cur);
    }
    load_q();
    for (; base < end; base += STEP) {
        f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        auto group = [&](auto index) {
            constexpr int c = decltype(index)::value;
            if constexpr (c < DK) {
                if (c >= 5 && c >= G) return;      // (scale bytes past a row's groups hold anything)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const s16x8 k = eight_values(kw[h][c], group_scale<c>(ks[h]));
#pragma unroll
                    for (int i = QP - 1; i >= 0; --i) s[h] = mfma_bf16(k, q[i][c], s[h]);      // the smallest parts first
                }
            }
        };
        group(std::integral_constant<int, 0>{});
        group(std::integral_constant<int, 1>{});
        group(std::integral_constant<int, 2>{});
        group(std::integral_constant<int, 3>{});
        group(std::integral_constant<int, 4>{});
        group(std::integral_constant<int, 5>{});
        group(std::integral_constant<int, 6>{});
        group(std::integral_constant<int, 7>{});
        load_k(next);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = s[j / 4][j % 4] * p.scale2;
        // tokens outside the chunk, or of no page: no weight, and zeros for values
        const uint32_t bits = tokens(cur, base);
        if (PIECE == 4 ? __any(bits != ~0u) : bits != ~0u) {
            const int mine = (int)(bits >> (grp * 4));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t in = (uint32_t)(mine << (31 - (j / 4 * 16 + j % 4)) >> 31);     // all ones, or none
                x[j] = in ? x[j] : NEG_INF;
#pragma unroll
                for (int u = 0; u < VU; ++u) {
                    vw[j / 4][u][j % 4] &= in;
                    vs[j / 4][u] &= in | ~(0x80u << (j % 4 * 8));      // a scale that is not NaN
                }
            }
        }
        float top = m;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, x[j]);
        top = across_groups(top, [](float a, float b) { return fmaxf(a, b); });
        const float ref = softmax_ref(top);
        if (__any(top > m)) {       // a larger maximum: what has been summed is taken relative to it
            const float corr = __builtin_amdgcn_exp2f(m - ref);
            l *= corr;
#pragma unroll
            for (int b = 0; b < NT; ++b) o[b] *= corr;
            m = top;
        }
        s16x8 w[PP];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = __builtin_amdgcn_exp2f(x[j] - ref);
            l += e;
            short part[PP];
            split_parts<PP>(e, part);
#pragma unroll
            for (int i = 0; i < PP; ++i) w[i][j] = part[i];
        }
        // two dimensions at a time: the values of the eight tokens in one byte of their words
        auto byte = [&](auto index, int u) {
            constexpr int B = decltype(index)::value;
            if constexpr (2 * B < NI) {
                uint32_t v[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t sc = vs[h][u];
                    const int shift = SHARE > 1 ? col / LD * (4 * NI) : 0;
                    v[4 * h] = two_values<B>(vw[h][u][0] >> shift, mx4_scale<0>(sc));
                    v[4 * h + 1] = two_values<B>(vw[h][u][1] >> shift, mx4_scale<1>(sc));
                    v[4 * h + 2] = two_values<B>(vw[h][u][2] >> shift, mx4_scale<2>(sc));
                    v[4 * h + 3] = two_values<B>(vw[h][u][3] >> shift, mx4_scale<3>(sc));
                }
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const uint32_t sel = n == 0 ? 0x05040100u : 0x07060302u;
                    const s16x8 a = __builtin_bit_cast(s16x8, u32x4{
                        __builtin_amdgcn_perm(v[1], v[0], sel), __builtin_amdgcn_perm(v[3], v[2], sel),
                        __builtin_amdgcn_perm(v[5], v[4], sel), __builtin_amdgcn_perm(v[7], v[6], sel)});
                    f32x4 &to = o[u * NI + 2 * B + n];
#pragma unroll
                    for (int i = PP - 1; i >= 0; --i) to = mfma_bf16(a, w[i], to);
                }
            }
        };
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            byte(std::integral_constant<int, 0>{}, u);
            byte(std::integral_constant<int, 1>{}, u);
            byte(std::integral_constant<int, 2>{}, u);
            byte(std::integral_constant<int, 3>{}, u);
        }
        load_v(next);
        cur = next;
        next = look_up(base + 2 * STEP);
    }

    // ---- the four waves joined ----
    l = across_groups(l, [](float a, float b) { return a + b; });
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int at = grp * 4 + r;     // the lane's column of the A operand that this row of the sums is
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int D = at % LD + 16 * u;
            if ((DK == 3 || DK == 8) && D >= 4 * G) continue;
            float *dst = acc + (wave * GT + col) * AP + D * 8 + at / LD * NI;
            if constexpr (NI == 2) {
                *reinterpret_cast<f32x2 *>(dst) = f32x2{o[0][r], o[1][r]};
            } else {
#pragma unroll
                for (int n = 0; n < NI; n += 4)
                    *reinterpret_cast<f32x4 *>(dst + n) = f32x4{o[u * NI + n][r], o[u * NI + n + 1][r], o[u * NI + n + 2][r],
                                                                o[u * NI + n + 3][r]};
            }
        }
    }
    if (grp == 0) s_ml[wave][col] = make_float2(m, l);
    __syncthreads();
    for (int i = threadIdx.x; i < t.heads_in_tile * p.dim; i += A4M_NT) {
        const int g = i / p.dim, d = i - g * p.dim;
        float top = NEG_INF, x = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < A4M_NW; ++w) top = fmaxf(top, s_ml[w][g].x);
        const float ref = softmax_ref(top);
#pragma unroll
        for (int w = 0; w < A4M_NW; ++w) {
            const float c = __builtin_amdgcn_exp2f(s_ml[w][g].x - ref);
            x += c * acc[(w * GT + g) * AP + d];
            sum += c * s_ml[w][g].y;
        }
        attend_store(p, t, t.first_head + g, d, x, top, sum);
    }
}

template <int DK, int QP>
void launch(const AttendArgs &p, const Kv4Pages &f, int page_size, unsigned groups, hipStream_t stream)
{
    const dim3 grid(groups), block(A4M_NT);
    if (page_size % 16 == 0) hipLaunchKernelGGL((nm_attend4_mfma_kernel<DK, QP, 16>), grid, block, 0, stream, p, f);
    else if (page_size % 8 == 0) hipLaunchKernelGGL((nm_attend4_mfma_kernel<DK, QP, 8>), grid, block, 0, stream, p, f);
    else hipLaunchKernelGGL((nm_attend4_mfma_kernel<DK, QP, 4>), grid, block, 0, stream, p, f);
}

template <int QP>
void launch_groups(const AttendArgs &p, const Kv4Pages &f, int page_size, unsigned groups, hipStream_t stream)
{
    if (f.l.G == 1) launch<1, QP>(p, f, page_size, groups, stream);
    else if (f.l.G == 2) launch<2, QP>(p, f, page_size, groups, stream);
    else if (f.l.G == 3) launch<3, QP>(p, f, page_size, groups, stream);
    else if (f.l.G == 4) launch<4, QP>(p, f, page_size, groups, stream);
    else launch<8, QP>(p, f, page_size, groups, stream);
}

}  // namespace

// A bf16 query is one part, an fp16 one two (16 bits), an fp32 one three (24).
void launch_attend4_mfma(const AttendArgs &p, const Kv4Pages &f, int page_size, unsigned groups, hipStream_t stream)
{
    if (p.io == NMSPMM_BF16) launch_groups<1>(p, f, page_size, groups, stream);
    else if (p.io == NMSPMM_F16) launch_groups<2>(p, f, page_size, groups, stream);
    else launch_groups<3>(p, f, page_size, groups, stream);
}

}  // namespace nmspmm
