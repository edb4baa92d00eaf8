// nmspmm_kv_attend on the matrix cores: queries and cache of one 16-bit type, or
// queries of another type over a bf16 cache.
//
// A workgroup of four waves takes a tile of 16 query heads of one cache head
// (fewer heads leave columns unused: the kernel is bound by the cache's bytes)
// and a chunk of one sequence.  A wave takes 32 tokens at a time:
//   S^T = K Q^T   v_mfma_f32_16x16x32: A operand 16 tokens, read from memory
//                 as its lanes hold them (16 bytes of a token's row a lane),
//                 B operand the queries, kept in registers;
//                 Queries that are not bf16 over a bf16 cache: three bf16 parts
//                 of every query value, which hold all 24 bits (a batch of
//                 42 x 676 positions, 7 heads of 256, 87 us on the vector ALU);
//   P^T           running maximum of each head (a lane's column), weights in
//                 fp32;
//   O^T += V^T P^T  the weights lie in the lanes just as the B operand wants
//                 them (k index 8g+j stands for token 4g+j, or 16+4g+j-4 from
//                 j = 4 on); V goes through LDS, a wave's own piece, whose
//                 transposed reads give V^T.
// A weight enters in 16-bit parts that keep fp32's precision.  bf16: three, all
// 24 bits (two left up to 2^-17 out, which turned single bf16 results; three
// are no slower).  fp16, whose smallest step a long sequence's weights come near:
// two of the weight times 2^14, which leave at most 2^-22 out from 2^-17 of the
// maximum on; where a tile has smaller weights, two more of what is left, times
// 2^24, so that what is lost lies under the rounding of any fp16 result.  (64
// sequences of 4096, 8 heads of 128, fp16: 212 us, 214 where most tiles have
// small weights; with V converted and the weights as they are on
// v_mfma_f32_16x16x4_f32 219, 32 ragged sequences of 4 heads of 256 82, 88 and 99.)
// The next tokens' K is on its way while the weights form, the next V while
// it is multiplied.  The waves are joined in LDS.  Bound by HBM: 128 x 8192
// positions, 32 heads on 8 of 128, 781-787 us (5.5 TB/s), one sequence of 131071
// 113-115 us (4.7 TB/s).
#include "nmspmm_kv.h"

namespace nmspmm {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int AM_NW = 4, AM_NT = 64 * AM_NW, AM_TOKENS = 32;
constexpr uint32_t NOWHERE = 0xffffffffu;

template <class T>
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c)
{
    if constexpr (__is_same(T, bf16_t))
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// x as PARTS 16-bit values, each the nearest to what those before it leave;
// returns what they all leave.
template <class T, int PARTS>
__device__ __forceinline__ float split_parts(float x, short *part)
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        const T h = from_f32<T>(x);
        part[i] = __builtin_bit_cast(short, h);
        x -= to_f32(h);
    }
    return x;
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

// Workgroups of a CU: as many as its registers hold (with three, the fp16 kernel
// for 128 dimensions kept registers in memory: 64 x 4096 positions 374 us, with
// two 212).
constexpr int attend_groups(bool f16, int DK, int QP) { return DK > 4 ? 1 : QP > 1 || (DK > 2 && f16) ? 2 : 3; }

// DK: pieces of 32 dimensions.  QP: parts of a query value.
template <class T, int DK, int QP>
__global__ __launch_bounds__(AM_NT, attend_groups(__is_same(T, f16_t), DK, QP)) void nm_attend_mfma_kernel(AttendArgs p)
{
    constexpr bool F16 = __is_same(T, f16_t);
    constexpr int PP = F16 ? 2 : 3;     // parts of a weight
    // what an fp16 weight's parts are multiplied by, what the two parts of their
    // rest are beside that, and the weight from which on no rest is needed
    constexpr float LIFT = F16 ? 0x1p14f : 1.f, REST = 0x1p24f, WHOLE = 0x1p-17f;
    constexpr int GT = 16, CPR = DK * 4, VL = CPR / 2, VPITCH = DK * 64 + 32, AP = DK * 32 + 4;
    static_assert(AM_NW * GT * AP * 4 <= AM_NW * AM_TOKENS * VPITCH, "the joining of the waves");
    __shared__ __align__(16) unsigned char lds[AM_NW * AM_TOKENS * VPITCH];
    __shared__ float2 s_ml[AM_NW][GT];
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
                split_parts<T, QP>(x, part);
#pragma unroll
                for (int i = 0; i < QP; ++i) q[i][c][j] = part[i];
            }
        }

    const int32_t *row = p.c.table + t.seq * p.c.table_stride;
    const unsigned char *kb = static_cast<const unsigned char *>(p.k) + t.head * p.c.ks[2] * 2;
    const unsigned char *vb = static_cast<const unsigned char *>(p.v) + t.head * p.c.vs[2] * 2;
    // lane l looks token l % 32 up: where its rows of K and V start, in pieces of 16 bytes
    struct Rows {
        uint32_t k, v;
    };
    auto look_up = [&](int base) {
        const int pos = base + (lane & 31);
        Place at{0, 0, false};
        if (pos < t.end) at = place_of(p.c, row, pos);
        return Rows{at.held ? (uint32_t)((at.page * p.c.ks[0] + at.slot * p.c.ks[1]) >> 3) : NOWHERE,
                    at.held ? (uint32_t)((at.page * p.c.vs[0] + at.slot * p.c.vs[1]) >> 3) : NOWHERE};
    };
    s16x8 kr[2][DK], vr[VL];
    auto load_k = [&](const Rows &r) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t at = __shfl(r.k, s * 16 + col);
#pragma unroll
            for (int c = 0; c < DK; ++c) {
                const int d = c * 32 + grp * 8;
                kr[s][c] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
                if (at != NOWHERE && d < p.dim)
                    kr[s][c] = *reinterpret_cast<const s16x8 *>(kb + (uint64_t)at * 16 + d * 2);
            }
        }
    };
    auto load_v = [&](const Rows &r) {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int e = i * 64 + lane, token = e / CPR, d = e % CPR * 8;
            const uint32_t at = __shfl(r.v, token);
            vr[i] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (at != NOWHERE && d < p.dim) vr[i] = *reinterpret_cast<const s16x8 *>(vb + (uint64_t)at * 16 + d * 2);
        }
    };

    f32x4 o[DK * 2];
#pragma unroll
    for (int b = 0; b < DK * 2; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = NEG_INF, l = 0.f;
    unsigned char *vs = lds + wave * (AM_TOKENS * VPITCH);
    const uint32_t vt = (uint32_t)(uintptr_t)(lds_u8 *)(lds_void *)vs +
                        (uint32_t)((grp * 4 + ((lane >> 2) & 3)) * VPITCH + (lane & 3) * 8);

    // dimensions 16 b and on of the tile's V^T, as the A operand's lanes hold them
    auto values = [&](int b) {
        s16x4 v[2];
#pragma unroll
        for (int y = 0; y < 2; ++y)
            v[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds_u8 *)(uintptr_t)(vt + b * 32 + y * 16 * VPITCH));
        return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };

    int base = t.begin + wave * AM_TOKENS;
    Rows cur = look_up(base), next = look_up(base + AM_NW * AM_TOKENS);
    load_k(cur);
    load_v(cur);
    for (; base < t.end; base += AM_NW * AM_TOKENS) {
        const uint32_t held = (uint32_t)__ballot(cur.k != NOWHERE);
        f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int c = 0; c < DK; ++c) {
#pragma unroll
            for (int i = QP - 1; i >= 0; --i) {     // the smallest parts first
                s[0] = mfma16<T>(kr[0][c], q[i][c], s[0]);
                s[1] = mfma16<T>(kr[1][c], q[i][c], s[1]);
            }
        }
        load_k(next);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = s[j / 4][j % 4] * p.scale2;
        if (held != 0xffffffffu) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!(held >> (j / 4 * 16 + grp * 4 + j % 4) & 1)) x[j] = NEG_INF;
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
            for (int b = 0; b < DK * 2; ++b) o[b] *= corr;
            m = top;
        }
        s16x8 w[PP];
        float left[8];
        bool small = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = __builtin_amdgcn_exp2f(x[j] - ref) * LIFT;
            l += e;
            small |= e > 0.f && e < WHOLE * LIFT;
            short part[PP];
            left[j] = split_parts<T, PP>(e, part);
#pragma unroll
            for (int i = 0; i < PP; ++i) w[i][j] = part[i];
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int e = i * 64 + lane;
            *reinterpret_cast<s16x8 *>(vs + e / CPR * VPITCH + e % CPR * 16) = vr[i];
        }
        asm volatile("" ::: "memory");
        load_v(next);
        cur = next;
        next = look_up(base + 2 * AM_NW * AM_TOKENS);
#pragma unroll
        for (int b = 0; b < DK * 2; ++b) {
            const s16x8 a = values(b);
#pragma unroll
            for (int i = PP - 1; i >= 0; --i) o[b] = mfma16<T>(a, w[i], o[b]);
        }
        if (F16 && __any(small)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                short part[2];
                split_parts<T, 2>(left[j] * REST, part);
                w[0][j] = part[0];
                w[1][j] = part[1];
            }
#pragma unroll
            for (int b = 0; b < DK * 2; ++b) {
                const s16x8 a = values(b);
                const f32x4 rest = mfma16<T>(a, w[0], mfma16<T>(a, w[1], f32x4{0.f, 0.f, 0.f, 0.f}));
#pragma unroll
                for (int i = 0; i < 4; ++i) o[b][i] = fmaf(rest[i], 1.f / REST, o[b][i]);
            }
        }
    }

    // ---- the four waves joined ----
    l = across_groups(l, [](float a, float b) { return a + b; }) / LIFT;
    __syncthreads();
    float *acc = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int b = 0; b < DK * 2; ++b)
        *reinterpret_cast<f32x4 *>(acc + (wave * GT + col) * AP + b * 16 + grp * 4) = o[b] / LIFT;
    if (grp == 0) s_ml[wave][col] = make_float2(m, l);
    __syncthreads();
    for (int i = threadIdx.x; i < t.heads_in_tile * p.dim; i += AM_NT) {
        const int g = i / p.dim, d = i - g * p.dim;
        float top = NEG_INF, x = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < AM_NW; ++w) top = fmaxf(top, s_ml[w][g].x);
        const float ref = softmax_ref(top);
#pragma unroll
        for (int w = 0; w < AM_NW; ++w) {
            const float c = __builtin_amdgcn_exp2f(s_ml[w][g].x - ref);
            x += c * acc[(w * GT + g) * AP + d];
            sum += c * s_ml[w][g].y;
        }
        attend_store(p, t, t.first_head + g, d, x, top, sum);
    }
}

template <class T, int QP>
void launch(const AttendArgs &p, unsigned groups, hipStream_t stream)
{
    const dim3 grid(groups), block(AM_NT);
    if (p.dim <= 64) hipLaunchKernelGGL((nm_attend_mfma_kernel<T, 2, QP>), grid, block, 0, stream, p);
    else if (p.dim <= 96) hipLaunchKernelGGL((nm_attend_mfma_kernel<T, 3, QP>), grid, block, 0, stream, p);
    else if (p.dim <= 128) hipLaunchKernelGGL((nm_attend_mfma_kernel<T, 4, QP>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((nm_attend_mfma_kernel<T, 8, QP>), grid, block, 0, stream, p);
}

}  // namespace

void launch_attend_mfma(const AttendArgs &p, nmspmm_dtype_t cache, unsigned groups, hipStream_t stream)
{
    if (cache == NMSPMM_F16) launch<f16_t, 1>(p, groups, stream);
    else if (p.io == NMSPMM_BF16) launch<bf16_t, 1>(p, groups, stream);
    else launch<bf16_t, 3>(p, groups, stream);
}

}  // namespace nmspmm
