// Products of up to 16 tokens with r-bit planes that have a scale and a zero-point for every group of inputs: what the matrix-vector
// product (mq_grouped.hip) and the layer of experts for a few tokens (mq_experts_ffn.hip) share.
#pragma once

#include "mq_common.h"

namespace mq {

// y[t, n] = sum over groups of alpha (2^s sum code x - z sum x).  A wave takes 16 rows of the plane (the matrix core's columns: lane
// & 15) and all 16 places for tokens (its rows).  A row is cut into chunks of C codes, each inside one group: the four quarters of the
// wave (lane >> 4) take C / 4 consecutive codes of it each, from one load of C r / 32 bytes, so one 16x16x32 product takes 8 codes of
// every quarter and never mixes groups.  Two products run side by side: tokens x codes and tokens x ones, whose result is sum x in the
// very lanes that hold the tokens' products; both are whole sums in fp32 before they meet alpha and z.  Codes of 4 and 2 bits enter as
// 128 + code (a bf16 number that holds the code exactly: shift, mask and or for two of them), which sum x takes out again.
//
// In operand order a register holds codes j and j + 4 (r = 4; j and j + 8 for r = 2) of the quarter's run, since that is what one shift and
// mask leaves.  Tokens in their own order are turned to it in registers; the layer's gated products are stored in it.
constexpr int kGroupedTokens = 16, kGroupedRows = 16;

template <int R>
constexpr float kCodeOffset = R == 8 ? 0.0f : 128.0f;

// place of input k of a row that is stored in operand order
template <int R>
__device__ __forceinline__ int operand_place(int k) {
    if constexpr (R == 4) return (k & ~7) | ((k & 3) << 1) | (k >> 2 & 1);
    if constexpr (R == 2) return (k & ~15) | ((k & 7) << 1) | (k >> 3 & 1);
    return k;
}

// group of a chunk, cpg chunks to a group
struct GroupOf {
    uint32_t cpg, magic;  // magic = ceil(2^32 / cpg): exact while chunk * cpg < 2^32
    __device__ __forceinline__ uint32_t operator()(uint32_t chunk) const { return cpg == 1 ? chunk : __umulhi(chunk, magic); }
};
inline GroupOf group_of(int64_t cpg) { return GroupOf{(uint32_t)cpg, cpg == 1 ? 0u : (uint32_t)(((1ull << 32) + cpg - 1) / cpg)}; }

// codes of a chunk: the most that a load of 16 bytes to a lane takes, as far as groups allow it
template <int R>
constexpr int kChunkMost = 512 / R;
template <int R>
constexpr int kChunkLeast = R == 2 ? 64 : 32;
// inputs of a group have to be a whole number of 16-byte pieces of codes and of matrix products
inline int64_t group_unit(int r) { return r == 2 ? 64 : 32; }
inline int chunk_codes(int r, int64_t group) {
    int c = 512 / r;
    while (group % c != 0) c >>= 1;
    return c;
}

template <int N>
struct Dwords;
template <>
struct Dwords<1> {
    typedef uint32_t type;
};
template <>
struct Dwords<2> {
    typedef u32x2 type;
};
template <>
struct Dwords<4> {
    typedef u32x4 type;
};

__device__ __forceinline__ uint32_t halves_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t halves_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// the eight codes of step s out of a lane's run of a chunk, as bf16
template <int R>
__device__ __forceinline__ u32x4 codes_operand(const uint32_t *w, int s) {
    u32x4 o;
    if constexpr (R == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = ((w[s] >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
    } else if constexpr (R == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = ((w[s >> 1] >> (8 * (s & 1) + 2 * i)) & 0x00030003u) | 0x43004300u;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t d = w[2 * s + (i >> 1)];
            const float lo = (float)((d >> (16 * (i & 1))) & 0xFFu), hi = (float)((d >> (16 * (i & 1) + 8)) & 0xFFu);
            o[i] = halves_hi(__float_as_uint(lo), __float_as_uint(hi));  // (0 .. 255 are bf16 numbers)
        }
    }
    return o;
}

// step s of a lane's run of tokens that are stored in their own order
template <int R>
__device__ __forceinline__ u32x4 token_operand(const u32x4 *x, int s) {
    if constexpr (R == 4)
        return u32x4{halves_lo(x[s].x, x[s].z), halves_hi(x[s].x, x[s].z), halves_lo(x[s].y, x[s].w), halves_hi(x[s].y, x[s].w)};
    if constexpr (R == 2) {
        const u32x4 a = x[s & ~1], b = x[s | 1];
        if (s & 1) return u32x4{halves_lo(a.z, b.z), halves_hi(a.z, b.z), halves_lo(a.w, b.w), halves_hi(a.w, b.w)};
        return u32x4{halves_lo(a.x, b.x), halves_hi(a.x, b.x), halves_lo(a.y, b.y), halves_hi(a.y, b.y)};
    }
    return x[s];
}

__device__ __forceinline__ f32x4 mfma_tokens(u32x4 tokens, u32x4 codes, f32x4 c) {
    Frag8 a, b;
    a.u = tokens;
    b.u = codes;
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
}

// One lane's row of the plane and one lane's token, both from the start of its quarter's run of chunk 0.
struct GroupedLane {
    const uint8_t *codes;
    const uint16_t *alpha, *zero;  // of the row, group 0
    const uint16_t *x;             // the token, or its leading bf16 part in operand order
    const uint16_t *rest;          // what the leading part leaves (bf16, operand order), with PARTS == 2
};

// Adds SPAN codes from chunk `first` on (what is behind the last chunk is left out) to y: lane = row, component i = token 4 (lane >> 4) + i.
// PARTS 1: tokens in their own order; 2: values as the sum of two bf16 numbers, both in operand order.
template <int R, int C, int SPAN, int PARTS>
__device__ __forceinline__ void grouped_span(const GroupedLane &p, int first, int chunks, GroupOf group, f32x4 &y) {
    constexpr int NC = SPAN / C, STEPS = C / 32, DW = C * R / 128, NP = (NC + 3) / 4;
    static_assert(NC >= 1 && SPAN % C == 0 && (R != 2 || STEPS % 2 == 0), "");
    typedef typename Dwords<DW>::type Piece;
    const int lane = threadIdx.x & 63, quarter = lane >> 4;
    const float step = (float)(1 << (8 - R));
    union {
        Piece piece[NC];
        uint32_t dw[NC * DW];
    } w;
    uint32_t params[NP];
    u32x4 x[PARTS][NC * STEPS];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = min(first + j, chunks - 1);
        w.piece[j] = __builtin_nontemporal_load(reinterpret_cast<const Piece *>(p.codes + (int64_t)c * (C * R / 8)));
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {  // quarter q of the wave looks up chunk 4 i + q for all of them
        const uint32_t g = group((uint32_t)min(first + 4 * i + quarter, chunks - 1));
        params[i] = (uint32_t)p.alpha[g] | (uint32_t)p.zero[g] << 16;
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int64_t at = (int64_t)min(first + j, chunks - 1) * C;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            x[0][j * STEPS + s] = *reinterpret_cast<const u32x4 *>(p.x + at + 8 * s);
            if constexpr (PARTS == 2) x[PARTS - 1][j * STEPS + s] = *reinterpret_cast<const u32x4 *>(p.rest + at + 8 * s);
        }
    }
    const u32x4 ones{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        f32x4 dot{0.f, 0.f, 0.f, 0.f}, sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const u32x4 codes = codes_operand<R>(w.dw + j * DW, s);
            const u32x4 t = PARTS == 2 ? x[0][j * STEPS + s] : token_operand<R>(x[0] + j * STEPS, s);
            dot = mfma_tokens(t, codes, dot);
            sum = mfma_tokens(t, ones, sum);
            if constexpr (PARTS == 2) {
                dot = mfma_tokens(x[PARTS - 1][j * STEPS + s], codes, dot);
                sum = mfma_tokens(x[PARTS - 1][j * STEPS + s], ones, sum);
            }
        }
        const uint32_t az = (uint32_t)__builtin_amdgcn_ds_bpermute(((lane & 15) + 16 * (j & 3)) << 2, (int)params[j >> 2]);
        const float alpha = first + j < chunks ? bf16_lo(az) : 0.f;  // (behind the last chunk: the last again, which counts for nothing)
        const float scale = alpha * step, shift = alpha * __builtin_fmaf(step, kCodeOffset<R>, bf16_hi(az));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_fmaf(scale, dot[i], __builtin_fmaf(-shift, sum[i], y[i]));
    }
}

// What is refused about a plane of `rows` rows and K inputs before a launch.
mq_status grouped_check(const uint8_t *packed, const uint16_t *alpha, const uint16_t *zero, int64_t rows, int64_t K, int64_t group, int r);

}  // namespace mq
