// Products of up to 16 tokens with r-bit planes that have a scale and a zero-point for every group of inputs: what the matrix-vector
// product (mq_grouped.hip) and the layer of experts for a few tokens (mq_experts_ffn.hip) share.
#pragma once

#include "mq_common.h"
#include "mq_grouped_plan.h"

namespace mq {

// y[t, n] = sum over groups of alpha (2^s sum code x - z sum x).  A wave takes tiles of 16 rows of the plane (the matrix core's columns: lane
// & 15) and up to 16 tokens (its rows), 32 codes to a step.  Two products run side by side: tokens x codes and tokens x ones, whose result is
// sum x in the very lanes that hold the tokens' products; both are whole sums in fp32 over a chunk (a part of one group) before they meet
// z, and alpha meets their difference, the codes' offset gone: large sums that take each other out do so before they are scaled, with one
// rounding of what is left.  Codes of 4 bits enter as 128 + code (a bf16 number that holds the code exactly: shift, mask and or for two of them), which
// sum x takes out again.  Two bits at mantissa bits 0, 2 or 4 under the exponent of 128, 32 or 8 are such numbers too, so codes of 2 bits need two
// shifts to a register instead of seven; a third product, of the tokens with the negative of these, stands in the sums before the codes do.
//
// Memory is read in pieces of a row, its 128-byte lines, by eight neighbouring lanes (and tokens alike): lanes that lie apart cost the address unit a
// cycle each, 64 for a load whose lanes are all in different rows.  A wave's own part of LDS turns pieces into the matrix core's operands; pieces under
// way stand in registers, of which a compute unit has three times as much as LDS.
//
// In operand order a register holds codes j and j + 4 (r = 4; j and j + 8 for r = 2) of a lane's run of 8 (16), since that is what one shift and
// mask leaves.

// what sum x takes out of the products
template <int R>
constexpr float kCodeOffset = R == 4 ? 128.0f : 0.0f;

// place of input k of a row that is stored in operand order
template <int R>
__device__ __forceinline__ int operand_place(int k) {
    if constexpr (R == 4) return (k & ~7) | ((k & 3) << 1) | (k >> 2 & 1);
    if constexpr (R == 2) return (k & ~15) | ((k & 7) << 1) | (k >> 3 & 1);
    return k;
}

// group of a chunk, cpg chunks to a group
struct GroupOf {
    uint32_t magic, whole;  // ceil(2^32 / cpg), 0 (exact while chunk * cpg < 2^32); for cpg = 1: 0, all bits
    __device__ __forceinline__ uint32_t operator()(uint32_t chunk) const { return __umulhi(chunk, magic) + (chunk & whole); }
};
inline GroupOf group_of(int64_t cpg) {
    return cpg == 1 ? GroupOf{0u, ~0u} : GroupOf{(uint32_t)(((1ull << 32) + cpg - 1) / cpg), 0u};
}

__device__ __forceinline__ uint32_t halves_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t halves_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

__device__ __forceinline__ f32x4 mfma_tokens(u32x4 tokens, u32x4 codes, f32x4 c) {
    Frag8 a, b;
    a.u = tokens;
    b.u = codes;
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
}

template <int R>
constexpr int kHalfCodes = 512 / R;

// T: tokens that are loaded, 4, 8 or 16 (the rows of the matrix core behind them repeat them); C codes to a chunk; RG tiles of 16 rows.
template <int R, int C, int RG, int T>
struct Grouped {
    static constexpr int PC = kHalfCodes<R>, NC = PC / C, STEPS = C / 32;
    static constexpr int XS = PC / 8;                                // 16-byte slots of a token in half a piece
    static constexpr int XI = T * XS < 64 ? 1 : T * XS / 64;         // loads of them for a wave
    static constexpr int CODES = RG * 2048, TOKENS = XI * 1024;      // bytes of LDS
    static constexpr int LDS = CODES + TOKENS + RG * 4 * NC * 128;
};

// A stretch of a product that one wave does: two pieces of 16 RG rows.  Bases are the same for the whole wave.
template <int XI>
struct Stretch {
    const uint8_t *codes;          // row 0 of the tiles, code 0 of the rows
    const uint16_t *alpha, *zero;  // row 0 of the tiles, group 0
    uint32_t token[XI];            // the first input that a lane loads of its token, as if half piece 0 came first (bytes, from the first token)
    int first;                     // first half piece
    // the layer's down product: whose outputs a lane's y are
    int count;                     // tokens
    uint32_t tokens;               // those of components 0 .. 3, a byte each
    f32x4 share;                   // their weights
};
// Between what lanes of a wave leave in LDS and what others of it read there: LDS serves a wave in order, so the compiler alone has to keep it.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Which token a lane's i-th load of half a piece is for, and which of the half piece's inputs is the first that it brings.
template <typename G>
__device__ __forceinline__ int load_token(int i) {
    return (64 * i + (int)(threadIdx.x & 63)) / G::XS;
}
template <typename G>
__device__ __forceinline__ int load_input(int i) {
    return (64 * i + (int)(threadIdx.x & 63)) % G::XS * 8;
}

// `bytes` bytes of tokens (less than 2^31) from x: a load behind them gives zeros.
constexpr uint32_t kBehind = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t token_buffer(const uint16_t *x, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(x), 0, (int)bytes, 0x00020000);  // (no stride, data of 32 bits)
}

// Does stretch after stretch: next(s) gives the wave's next one or says that there is none, end(s) follows each (next has been asked for the one
// behind it by then); products are added to y[tile] (lane & 15 = row, component i = token 4 (lane >> 4) + i).  While a piece is
// multiplied the D - 1 behind it are on their way; nothing is requested behind the last stretch.  ORDERED: tokens are in operand order.
// What lies behind the end of rows of K inputs is read as their end again, but for tokens, which are zeros there (a scale of zero alone would make
// no number of sums that overflow there alone): the places are out of the buffer's range, so the load gives zeros without a branch or a select of
// what it brings.
template <int R, int C, int RG, int T, bool ORDERED, int D, typename Next, typename End>
__device__ __forceinline__ void grouped_stream(uint8_t *lds, __amdgpu_buffer_rsrc_t tokens, int rows, int K, int groups, GroupOf group, f32x4 (&y)[RG], Next next, End end) {
    using G = Grouped<R, C, RG, T>;
    constexpr int PC = G::PC, NC = G::NC, STEPS = G::STEPS, XS = G::XS, XI = G::XI;
    static_assert((D == 1 || D == 2) && NC >= 1 && STEPS >= 1 && (R != 2 || STEPS % 2 == 0), "");
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // (places in LDS are computed here, for each stream anew, instead of being kept in registers around it)
    const int li = lane & 15, quarter = lane >> 4, part = lane & 3;
    const int bytes = K / 8 * R, chunks = K / C, halves = (K + PC - 1) / PC;
    const float step = (float)(1 << (8 - R));
    const u32x4 ones{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    // (in registers: one instruction for "and" and "or", which takes no two literals)
    uint32_t mask[3] = {R == 4 ? 0x000F000Fu : 0x00030003u, 0x000C000Cu, 0x00300030u}, base[3] = {0x43004300u, 0x42004200u, 0x41004100u};
    asm volatile("" : "+s"(mask[0]), "+s"(mask[1]), "+s"(mask[2]), "+v"(base[0]), "+v"(base[1]), "+v"(base[2]));
    // code pair j of a register of 2-bit codes stands at position j % 3 after a shift by 6 (j / 3)
    const u32x4 minus[2] = {{0xC300C300u, 0xC200C200u, 0xC100C100u, 0xC300C300u}, {0xC200C200u, 0xC100C100u, 0xC300C300u, 0xC200C200u}};
    uint8_t *const lds_x = lds + G::CODES;
    // alpha 2^s, what sum x is multiplied with before it
    f32pair_t *const lds_params = reinterpret_cast<f32pair_t *>(lds_x + G::TOKENS);

    uint32_t row_codes[RG][2], row_params[RG];
#pragma unroll
    for (int t = 0; t < RG; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) row_codes[t][i] = (uint32_t)min(16 * t + 8 * i + (lane >> 3), rows - 1) * (uint32_t)bytes;
        row_params[t] = (uint32_t)min(16 * t + (lane >> 2), rows - 1) * (uint32_t)groups;
    }
    // 16-byte slots are spread over the banks by the row's, the token's number
    const int codes_to = (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4);
    const int codes_from = li * 128, codes_turn = li & 7;
    int x_to[XI];
#pragma unroll
    for (int i = 0; i < XI; ++i) {
        const int token = load_token<G>(i), slot = (64 * i + lane) % XS;
        x_to[i] = token * (XS * 16) + ((slot ^ (token & (XS - 1) & 15)) << 4);
    }
    const int x_token = li % T, x_from = x_token * (XS * 16), x_turn = x_token & (XS - 1) & 15;

    u32x4 w[D][RG][2], x[D][kHalves][XI];
    uint16_t alpha[RG][NC], zero[RG][NC];
    auto fetch = [&](const Stretch<XI> &s, int j, int slot) {
        const uint32_t at = (uint32_t)min((s.first + kHalves * j) * 64 + (lane & 7) * 16, bytes - 16);
#pragma unroll
        for (int t = 0; t < RG; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) w[slot][t][i] = *reinterpret_cast<const u32x4 *>(s.codes + (row_codes[t][i] + at));
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int i = 0; i < XI; ++i) {
                const int begin = (s.first + kHalves * j + h) * PC;
                const uint32_t v = load_input<G>(i) < K - begin ? s.token[i] : kBehind;
                // (a scalar offset inside the buffer: the range that is left for v is the buffer's less this one)
                x[slot][h][i] = __builtin_amdgcn_raw_buffer_load_b128(tokens, (int)v, 2 * min(begin, K - 8), 0);
            }
    };
    auto fetch_params = [&](const Stretch<XI> &s) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const uint32_t g = group((uint32_t)min(s.first * NC + 4 * i + part, chunks - 1));
#pragma unroll
            for (int t = 0; t < RG; ++t) {
                alpha[t][i] = s.alpha[row_params[t] + g];
                zero[t][i] = s.zero[row_params[t] + g];
            }
        }
    };
    auto multiply = [&](const Stretch<XI> &s, int half, int slot) {
        const int h = half % kHalves;
        if (h == 0)
#pragma unroll
            for (int t = 0; t < RG; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) *reinterpret_cast<u32x4 *>(lds + t * 2048 + i * 1024 + codes_to) = w[slot][t][i];
#pragma unroll
        for (int i = 0; i < XI; ++i) {
            u32x4 v = x[slot][h][i];
            if constexpr (!ORDERED && R == 4) v = u32x4{halves_lo(v.x, v.z), halves_hi(v.x, v.z), halves_lo(v.y, v.w), halves_hi(v.y, v.w)};
            *reinterpret_cast<u32x4 *>(lds_x + x_to[i]) = v;
        }
        wave_fence();
        auto slot_of_x = [&](int at) { return *reinterpret_cast<const u32x4 *>(lds_x + x_from + ((at ^ x_turn) << 4)); };
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            f32x4 dot[RG], sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < RG; ++t) dot[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            uint32_t both[RG];
#pragma unroll
            for (int k0 = 0; k0 < STEPS; ++k0) {
                const int k = c * STEPS + k0;
                u32x4 v;
                if constexpr (R != 2) {
                    v = slot_of_x(4 * k + quarter);
                } else if constexpr (ORDERED) {
                    v = slot_of_x(8 * (k >> 1) + 2 * quarter + (k & 1));
                } else {
                    const u32x4 a = slot_of_x(8 * (k >> 1) + 2 * quarter), b = slot_of_x(8 * (k >> 1) + 2 * quarter + 1);
                    v = k & 1 ? u32x4{halves_lo(a.z, b.z), halves_hi(a.z, b.z), halves_lo(a.w, b.w), halves_hi(a.w, b.w)}
                              : u32x4{halves_lo(a.x, b.x), halves_hi(a.x, b.x), halves_lo(a.y, b.y), halves_hi(a.y, b.y)};
                }
                sum = mfma_tokens(v, ones, sum);
#pragma unroll
                for (int t = 0; t < RG; ++t) {
                    const uint8_t *tile = lds + t * 2048 + codes_from;
                    u32x4 o;
                    if constexpr (R == 4) {
                        const uint32_t d = *reinterpret_cast<const uint32_t *>(tile + (((4 * h + k) ^ codes_turn) << 4) + 4 * quarter);
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] = ((d >> (4 * i)) & mask[0]) | base[0];
                    } else if constexpr (R == 2) {
                        if (!(k & 1)) both[t] = *reinterpret_cast<const uint32_t *>(tile + (((4 * h + (k >> 1)) ^ codes_turn) << 4) + 4 * quarter);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = 4 * (k & 1) + i;
                            o[i] = ((both[t] >> (6 * (j / 3))) & mask[j % 3]) | base[j % 3];
                        }
                    } else {
                        const u32x2 d = *reinterpret_cast<const u32x2 *>(tile + (((4 * h + 2 * k + (quarter >> 1)) ^ codes_turn) << 4) + 8 * (quarter & 1));
#pragma unroll
                        for (int i = 0; i < 4; ++i) {  // (0 .. 255 are bf16 numbers)
                            const float lo = (float)((d[i >> 1] >> (16 * (i & 1))) & 0xFFu), hi = (float)((d[i >> 1] >> (16 * (i & 1) + 8)) & 0xFFu);
                            o[i] = halves_hi(__float_as_uint(lo), __float_as_uint(hi));
                        }
                    }
                    if constexpr (R == 2) dot[t] = mfma_tokens(v, minus[k & 1], dot[t]);
                    dot[t] = mfma_tokens(v, o, dot[t]);
                }
            }
            const int chunk = half * NC + c;
#pragma unroll
            for (int t = 0; t < RG; ++t) {
                const f32pair_t by = lds_params[(t * 4 * NC + chunk) * 16 + li];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[t][i] = __builtin_fmaf(by[0], __builtin_fmaf(by[1], sum[i], dot[t][i]), y[t][i]);
                asm volatile("" : "+v"(y[t]));  // (done here: put off to where y is used, every chunk's sums would stay in registers)
            }
        }
        wave_fence();
    };
    Stretch<XI> s, n;
    if (!next(s)) return;
    fetch_params(s);
#pragma unroll
    for (int j = 0; j < D; ++j) {
        __builtin_amdgcn_sched_barrier(0);  // (in order, as in the loop: a wait counts the requests behind the one it is for)
        fetch(s, j, j);
    }
    __builtin_amdgcn_sched_barrier(0);
    auto body = [&](auto with_next) {
#pragma unroll
        for (int t = 0; t < RG; ++t)
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const float a = bf16_bits_to_float(alpha[t][i]);
                lds_params[(t * 4 * NC + 4 * i + part) * 16 + (lane >> 2)] =
                    f32pair_t{a * step, -__builtin_fmaf(1.0f / step, bf16_bits_to_float(zero[t][i]), kCodeOffset<R>)};
            }
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                // (a row's end, where there may be less, comes last)
                if (decltype(with_next)::value || kHalves * j + h == 0 || s.first + kHalves * j + h < halves) multiply(s, kHalves * j + h, j % D);
                __builtin_amdgcn_sched_barrier(0);  // (keeps the requests of later pieces and what unpacks them out of this one's registers)
            }
            if (j + D < kPieces) {
                fetch(s, j + D, j % D);
            } else if constexpr (decltype(with_next)::value) {
                if (j + D == kPieces) fetch_params(n);
                fetch(n, j + D - kPieces, j % D);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    while (next(n)) {
        body(std::true_type{});
        end(s);
        s = n;
    }
    body(std::false_type{});
    end(s);
}

// Adds up the tiles of the workgroup's waves (part: one place for each wave and tile) into those of the first one.
template <int RG>
__device__ __forceinline__ void join_waves(f32x4 *part, int wave, int waves, f32x4 (&y)[RG]) {
    if (waves == 1) return;
    const int lane = threadIdx.x & 63;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RG; ++t) part[(wave * RG + t) * 64 + lane] = y[t];
    __syncthreads();
    if (wave != 0) return;
    for (int k = 1; k < waves; ++k)
#pragma unroll
        for (int t = 0; t < RG; ++t) y[t] += part[(k * RG + t) * 64 + lane];
}

// What is refused about a plane of `rows` rows and K inputs before a launch.
mq_status grouped_check(const uint8_t *packed, const uint16_t *alpha, const uint16_t *zero, int64_t rows, int64_t K, int64_t group, int r);

}  // namespace mq
