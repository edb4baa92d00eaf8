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
// query value.  UNI: pages of whole sixteens of tokens, so that a tile's page is the
// same for all lanes.
template <int DK, int QP, bool UNI>
__global__ __launch_bounds__(A4M_NT, DK > 4 && QP > 2 ? 1 : DK > 4 || QP > 1 ? 2 : 3) void nm_attend4_mfma_kernel(AttendArgs p, Kv4Pages f)
{
    constexpr int GT = ATTEND_MFMA_HEADS, PP = 3;
    // the values' words of a lane (VU of them, dimension words 16 apart) and the codes
    // that it takes of each: with few groups, 16 / (4 DK) lanes share a word's codes
    constexpr int VU = DK == 8 ? 2 : 1, SHARE = DK == 1 ? 4 : DK == 2 ? 2 : 1, NI = 8 / SHARE, LD = 16 / SHARE;
    constexpr int NT = VU * NI, AP = DK * 32 + 4, SW = DK > 4 ? 2 : 1;
    __shared__ __align__(16) float acc[A4M_NW * GT * AP];
    __shared__ float2 s_ml[A4M_NW][GT];
    const AttendTask t = attend_task(p, blockIdx.x, GT);
    if (t.begin >= t.end && p.splits > 1) {      // nothing here: the maximum says so
        if (threadIdx.x < t.heads_in_tile) {
            const int64_t row = t.seq * ((int64_t)p.heads * p.group) + t.first_head + threadIdx.x;
            p.part_ml[row * p.splits + t.split] = make_float2(NEG_INF, 0.f);
        }
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 15, grp = lane >> 4;
    const int G = DK == 8 ? f.l.G : DK;

    s16x8 q[QP][DK];
#pragma unroll
    for (int c = 0; c < DK; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int d = c * 32 + grp * 8 + j;
            const bool there = col < t.heads_in_tile && d < p.dim;
            const int64_t at = t.seq * p.qs[0] + (t.first_head + col) * p.qs[1] + d;
            if constexpr (QP == 1) {
                if (p.q_vec) {      // eight at once
                    if (j == 0) {
                        q[0][c] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
                        if (there) q[0][c] = *reinterpret_cast<const s16x8 *>(static_cast<const short *>(p.q) + at);
                    }
                    continue;
                }
                q[0][c][j] = there ? static_cast<const short *>(p.q)[at] : (short)0;
            } else {
                const float x = !there ? 0.f : p.io == NMSPMM_F32 ? static_cast<const float *>(p.q)[at]
                                                                  : to_f32(static_cast<const f16_t *>(p.q)[at]);
                short part[QP];
                split_parts<QP>(x, part);
#pragma unroll
                for (int i = 0; i < QP; ++i) q[i][c][j] = part[i];
            }
        }

    // ---- the tokens ----
    const int32_t *row = p.c.table + t.seq * p.c.table_stride;
    const unsigned char *blocks = f.pages + t.head * f.l.block;
    struct Where {      // of the tile's two sixteens: pages (-1: none) and slots of this lane's keys and values
        int32_t k_page[2], v_page[2], k_slot[2], v_slot[2];
    };
    auto find = [&](int pos, int32_t &page, int32_t &slot) {
        page = -1, slot = 0;
        if (pos < t.end) {
            const Place at = place_of(p.c, row, pos);
            page = at.held ? (int32_t)at.page : -1;
            slot = at.slot;
        }
    };
    auto look_up = [&](int base) {
        Where w;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if constexpr (UNI) {
                find(base + 16 * s, w.k_page[s], w.k_slot[s]);
                w.k_page[s] = __builtin_amdgcn_readfirstlane(w.k_page[s]);
                w.k_slot[s] = __builtin_amdgcn_readfirstlane(w.k_slot[s]);
                w.v_page[s] = w.k_page[s];
                w.v_slot[s] = w.k_slot[s];
            } else {
                find(base + 16 * s + col, w.k_page[s], w.k_slot[s]);
                find(base + 16 * s + 4 * grp, w.v_page[s], w.v_slot[s]);
            }
        }
        return w;
    };
    uint32_t kw[2][DK], ks[2][SW];
    u32x4 vw[2][VU];
    uint32_t vs[2][VU];
    auto load_k = [&](const Where &w) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int c = 0; c < DK; ++c) kw[s][c] = 0;
#pragma unroll
            for (int i = 0; i < SW; ++i) ks[s][i] = 0x7f7f7f7fu;
            if (w.k_page[s] < 0) continue;
            const unsigned char *b = blocks + w.k_page[s] * f.stride;
            const uint32_t slot = (uint32_t)w.k_slot[s] + (UNI ? col : 0);
            const unsigned char *at = b + slot * (uint32_t)(16 * G) + (uint32_t)(grp * G * 4);
            if constexpr (DK <= 4) {
                __builtin_memcpy(kw[s], __builtin_assume_aligned(at, 4 * (DK & -DK)), 4 * DK);
            } else {
                if (G == 8) __builtin_memcpy(kw[s], __builtin_assume_aligned(at, 16), 32);
                else
#pragma unroll
                    for (int c = 0; c < DK; ++c)
                        if (c < G) kw[s][c] = *reinterpret_cast<const uint32_t *>(at + 4 * c);
            }
            const unsigned char *sc = b + f.l.ks_at + slot * (uint32_t)f.l.sp;
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
                const int D = col % LD + 16 * u;
                vw[s][u] = u32x4{0, 0, 0, 0};
                vs[s][u] = 0x7f7f7f7fu;
                if (w.v_page[s] < 0 || ((DK == 3 || DK == 8) && D >= 4 * G)) continue;
                const unsigned char *b = blocks + w.v_page[s] * f.stride;
                const uint32_t quad = (uint32_t)w.v_slot[s] / 4 + (UNI ? grp : 0);
                vw[s][u] = *reinterpret_cast<const u32x4 *>(b + f.l.v_at + quad * (uint32_t)(64 * G) + (uint32_t)(D * 16));
                vs[s][u] = *reinterpret_cast<const uint32_t *>(b + f.l.vs_at + quad * (uint32_t)(4 * G) + (uint32_t)(D / 4 * 4));
            }
    };

    f32x4 o[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = NEG_INF, l = 0.f;

    int base = (t.begin & ~(A4M_TOKENS - 1)) + wave * A4M_TOKENS;
    constexpr int STEP = A4M_NW * A4M_TOKENS;
    Where cur = look_up(base), next = look_up(base + STEP);
    load_k(cur);
    load_v(cur);
    for (; base < t.end; base += STEP) {
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
        const bool whole = base >= t.begin && base + A4M_TOKENS <= t.end && cur.v_page[0] >= 0 && cur.v_page[1] >= 0;
        if (!(UNI ? whole : __all(whole))) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int pos = base + j / 4 * 16 + grp * 4 + j % 4;
                if (pos >= t.begin && pos < t.end && cur.v_page[j / 4] >= 0) continue;
                x[j] = NEG_INF;
#pragma unroll
                for (int u = 0; u < VU; ++u) {
                    vw[j / 4][u][j % 4] = 0;
                    vs[j / 4][u] = (vs[j / 4][u] & ~(0xffu << (j % 4 * 8))) | 0x7fu << (j % 4 * 8);
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
void launch(const AttendArgs &p, const Kv4Pages &f, bool uniform, unsigned groups, hipStream_t stream)
{
    const dim3 grid(groups), block(A4M_NT);
    if (uniform) hipLaunchKernelGGL((nm_attend4_mfma_kernel<DK, QP, true>), grid, block, 0, stream, p, f);
    else hipLaunchKernelGGL((nm_attend4_mfma_kernel<DK, QP, false>), grid, block, 0, stream, p, f);
}

template <int QP>
void launch_groups(const AttendArgs &p, const Kv4Pages &f, bool uniform, unsigned groups, hipStream_t stream)
{
    if (f.l.G == 1) launch<1, QP>(p, f, uniform, groups, stream);
    else if (f.l.G == 2) launch<2, QP>(p, f, uniform, groups, stream);
    else if (f.l.G == 3) launch<3, QP>(p, f, uniform, groups, stream);
    else if (f.l.G == 4) launch<4, QP>(p, f, uniform, groups, stream);
    else launch<8, QP>(p, f, uniform, groups, stream);
}

}  // namespace

// A bf16 query is one part, an fp16 one two (16 bits), an fp32 one three (24).
void launch_attend4_mfma(const AttendArgs &p, const Kv4Pages &f, bool uniform, unsigned groups, hipStream_t stream)
{
    if (p.io == NMSPMM_BF16) launch_groups<1>(p, f, uniform, groups, stream);
    else if (p.io == NMSPMM_F16) launch_groups<2>(p, f, uniform, groups, stream);
    else launch_groups<3>(p, f, uniform, groups, stream);
}

}  // namespace nmspmm
