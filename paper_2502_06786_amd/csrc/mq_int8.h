// Internal interface of the layer in 8-bit integers (not part of the public ABI): tokens as int8 codes with a scale and a sum
// each, multiplied with the codes of the weights as they are stored.
#pragma once

#include "mq_gemv.h"
#include "mq_int8_blocks.h"
#include "mq_int8_plan.h"

namespace mq {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
// bf16 outputs side by side at any of their addresses: one store, which the memory pipeline takes apart where it has to
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

constexpr int64_t kInt8MaxK = 131072;     // 127 * 128 * K stays below 2^31
constexpr int64_t kMaxExperts = 1024;
constexpr int64_t kInt8Line = 128;        // of the L2: a stage of 128 k of a row that begins elsewhere takes two of them

// One product: Y[p, n] of T places, place p holding token rows[p] (or p) and belonging to the expert e with
// offsets[e] <= p < offsets[e + 1] (or to the only one).
struct Int8Args {
    const int8_t *Xq;        // [M, K], rows ldq bytes apart
    const float *scale;      // [M]
    const int32_t *sum;      // [M]
    const int32_t *rows;     // [T] or null
    const int32_t *offsets;  // [E + 1] or null (E = 1)
    const uint8_t *codes;    // [E, N, K]
    const float *alpha, *zero;  // [E, N]
    uint16_t *Y;             // [T, N], with a gate [T, N / 2]
    int M, T, N, K, E;
    int ldq;                 // K or more; the library's own rows begin at lines of 128 bytes (kInt8Line)
    int gate;                // 0 none, 1 GELU-tanh, 2 SiLU
    float mult, offset;      // 2^(8-r); what the matrix core's signed reading of a code leaves out (128 at r = 8, otherwise 0)
};

// Codes of r = 8 fill the byte, and the matrix core reads bytes as signed: code ^ 0x80 is code - 128.
template <bool R8>
__device__ __forceinline__ i32x4 signed_codes(i32x4 v) {
    if constexpr (R8) v ^= i32x4{(int)0x80808080u, (int)0x80808080u, (int)0x80808080u, (int)0x80808080u};
    return v;
}

__device__ __forceinline__ i32x4 mfma_i8(const i32x4 &a, const i32x4 &b, const i32x4 &c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// scale (alpha 2^(8-r) (dot + offset sum) - alpha zero sum): the same fp32 steps in every kernel, and `dot` is a sum of whole numbers, so the
// outputs of all forms of the product are the same bits.  (dot below 2^31 and dot + offset sum are rounded to fp32: 2^-24 of themselves.)
// The offset goes back to the sum and not into the zero-point: a channel whose weights are all w has codes of 0 and zero = -w, dot + offset sum is
// then 0 to the last bit, while zero - offset loses what is small beside 128 (w = 3e-5 came out 5 % off).  One instruction more per
// output: 8192 x 28672 x 3584 with a gate 723 -> 725 us, the shorter calls within their spread.  The token's scale last: it may be as small as
// a bf16 subnormal / 127.
__device__ __forceinline__ void channel_factors(const f32x4 &alpha, const f32x4 &zero, float mult, f32x4 &ka, f32x4 &kb) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        ka[e] = alpha[e] * mult;
        kb[e] = alpha[e] * zero[e];
    }
}
// OFFSET false: known to be 0 (the same bits, an instruction less).
template <bool OFFSET = true>
__device__ __forceinline__ float int8_output(int dot, float sum, float scale, float ka, float kb, float offset) {
    const float codes = OFFSET ? __builtin_fmaf(offset, sum, (float)dot) : (float)dot;
    return __builtin_fmaf(ka, codes, -(kb * sum)) * scale;
}

// act(g) u, act(v) = v / (1 + exp(-t)): t = v for SiLU, 2 sqrt(2 / pi) (v + 0.044715 v^3) for GELU in its tanh form.  The gate acts on
// the fp32 outputs: one rounding, to bf16, at the end.  (The reciprocal is the hardware's, 2^-23 of its value off at most.)
__device__ __forceinline__ float gated_value(float g, float u, int gate) {
    const float t = gate == 2 ? g : 1.5957691216057308f * (g + 0.044715f * g * g * g);
    return g * __builtin_amdgcn_rcpf(1.0f + __expf(-t)) * u;
}

// ---- a token's codes: scale = top / 127, code = round(x (127 / top)), top the row's largest magnitude -------------------------------
// The largest magnitude is found on the bf16 bits themselves: their order is that of the magnitudes, infinities and NaN last.
__device__ __forceinline__ uint32_t top_of(uint32_t top2, const u32x4 &v) {   // largest so far of the low and of the high halves
#pragma unroll
    for (int w = 0; w < 4; ++w)
        top2 = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top2), __builtin_bit_cast(u16x2, v[w] & 0x7FFF7FFFu)));
    return top2;
}
__device__ __forceinline__ uint32_t top_of_wave(uint32_t top2) {
    uint32_t top = max(top2 & 0xFFFFu, top2 >> 16);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    return top;
}
struct TokenScale {
    float lift, per, scale;
    bool finite;
};
__device__ __forceinline__ TokenScale token_scale(uint32_t top) {
    const bool finite = top < 0x7F80u;
    const float most = bf16_bits_to_float(top);
    const float lift = most < 0x1p-100f ? 0x1p100f : 1.0f;          // 127 / most would pass the largest fp32 number
    return {lift, finite && top != 0 ? __fdiv_rn(127.0f, most * lift) : 0.0f, finite ? __fdiv_rn(most, 127.0f) : __uint_as_float(0x7FC00000u), finite};
}
// eight values -> eight codes; their sum is added to total
__device__ __forceinline__ u32x2 token_codes(const u32x4 &v, const TokenScale &t, int &total) {
    uint32_t out[2] = {0u, 0u};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t d = t.finite ? v[w] : 0u;  // (infinity times zero is no number)
        const int lo = (int)rintf(bf16_lo(d) * t.lift * t.per), hi = (int)rintf(bf16_hi(d) * t.lift * t.per);
        total += lo + hi;
        out[w >> 1] |= ((uint32_t)(lo & 0xFF) | (uint32_t)(hi & 0xFF) << 8) << (16 * (w & 1));
    }
    return u32x2{out[0], out[1]};
}
__device__ __forceinline__ int sum_of_wave(int total) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    return total;
}

__device__ __forceinline__ Block find_block(const Int8Args &a, int block, int BM) {
    if (!a.offsets) return Block{0, block * BM, min(BM, a.T - block * BM)};
    return find_block(a.T, a.E, block, BM, [&](int e) { return a.offsets[e]; });
}
// the token of a place (rows are data: whatever they hold, tokens stay below M)
__device__ __forceinline__ int token_of(const Int8Args &a, int place) { return a.rows ? min(max(a.rows[place], 0), a.M - 1) : place; }

// four neighbouring outputs (n .. n + 3) of one place, or the two gated ones
__device__ __forceinline__ void store_four(const Int8Args &a, int place, int n, const i32x4 &dot, float scale, float sum, const f32x4 &ka,
                                           const f32x4 &kb) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = int8_output(dot[e], sum, scale, ka[e], kb[e], a.offset);
    // (rows of Y begin at any bf16)
    if (a.gate) {
        const uint32_t o = pack_bf16x2(gated_value(y[0], y[1], a.gate), gated_value(y[2], y[3], a.gate));
        uint16_t *out = a.Y + (int64_t)place * (a.N / 2) + n / 2;
        if (n + 2 < a.N)
            *reinterpret_cast<u32_any *>(out) = o;
        else
            out[0] = (uint16_t)o;
    } else {
        const u32x2 o = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        uint16_t *out = a.Y + (int64_t)place * a.N + n;
        if (n + 3 < a.N) {
            *reinterpret_cast<u32x2_any *>(out) = o;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < a.N) out[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
        }
    }
}

__device__ __forceinline__ void load_factors(const Int8Args &a, int expert, int n, f32x4 &ka, f32x4 &kb) {
    const float *alpha = a.alpha + (int64_t)expert * a.N, *zero = a.zero + (int64_t)expert * a.N;
    f32x4 al, ze;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        al[e] = alpha[min(n + e, a.N - 1)];
        ze[e] = zero[min(n + e, a.N - 1)];
    }
    channel_factors(al, ze, a.mult, ka, kb);
}

// ---- ranges of K ------------------------------------------------------------------------------------------
struct Int8Ranges {
    i32x4 *part;  // [split][tile][wave, rb, tb][lane]
    int splits;
};

// Adds the ranges (whole numbers: in any order) and finishes the outputs: a wave for each block of 16 channels x 16 places of tiles of
// WR x WC waves with RB x TB blocks each.  Dense products only.
template <int RB, int TB, int WR, int WC>
__global__ __launch_bounds__(256) void int8_join_kernel(Int8Args a, int tiles_m, int tiles_n, Int8Ranges s) {
    constexpr int NW = WR * WC, BLOCKS = NW * RB * TB;
    const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15, id = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int tile = id / BLOCKS, wave = id % BLOCKS / (RB * TB), rb = id / TB % RB, tb = id % TB, wr = wave % WR, wc = wave / WR;
    const int tiles = tiles_m * tiles_n;
    if (tile >= tiles) return;
    const int row = tile % tiles_m * (16 * TB * WC) + (wc * TB + tb) * 16 + l16, n = tile / tiles_m * (16 * RB * WR) + (wr * RB + rb) * 16 + 4 * g4;
    if (row >= a.T || n >= a.N) return;
    const i32x4 *from = s.part + (int64_t)id * 64 + lane;
    const int64_t step = (int64_t)tiles * BLOCKS * 64;
    f32x4 ka, kb;
    load_factors(a, 0, n, ka, kb);
    const float scale = a.scale[row], sum = (float)a.sum[row];
    i32x4 dot = {0, 0, 0, 0};
    for (int i = 0; i < s.splits; i += 4) {   // four loads in flight
        i32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = i + j < s.splits ? from[(i + j) * step] : i32x4{0, 0, 0, 0};
        dot += (v[0] + v[1]) + (v[2] + v[3]);
    }
    store_four(a, row, n, dot, scale, sum, ka, kb);
}

template <int RB, int TB, int WR, int WC>
mq_status launch_int8_join(const Int8Args &a, const Int8Ranges &s, hipStream_t st) {
    const int64_t tiles_n = cdiv(a.N, 16 * RB * WR), tiles_m = cdiv(a.T, 16 * TB * WC);
    int8_join_kernel<RB, TB, WR, WC><<<dim3((unsigned)cdiv(tiles_n * tiles_m * WR * WC * RB * TB, 4)), dim3(256), 0, st>>>(a, (int)tiles_m, (int)tiles_n, s);
    return launch_status();
}

mq_status launch_quantize_tokens(const uint16_t *X, int64_t M, int64_t K, int64_t ldx, const int32_t *rows, int64_t X_rows, int8_t *Xq, int64_t ldq,
                                 float *scale, int32_t *sum, hipStream_t st);
mq_status launch_int8_few(const Int8Args &a, hipStream_t st);
// the same on bf16 tokens X [M, K], for up to kInt8SinglePlaces places and kInt8SingleK values a token
mq_status launch_int8_single(const Int8Args &a, const uint16_t *X, hipStream_t st);
// places: of a tile, 32, 64 or 96; part: room for the partial sums of `splits` ranges of K
mq_status launch_int8_mid(const Int8Args &a, int places, int splits, void *part, hipStream_t st);
// form: kInt8Deep128 (which may be cut), kInt8Tile128 or kInt8Tile256
mq_status launch_int8_tiles(const Int8Args &a, Int8Form form, int splits, void *part, hipStream_t st);

}  // namespace mq
