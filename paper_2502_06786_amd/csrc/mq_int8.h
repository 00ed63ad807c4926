// Internal interface of the layer in 8-bit integers (not part of the public ABI): tokens as int8 codes with a scale and a sum
// each, multiplied with the codes of the weights as they are stored.
#pragma once

#include "mq_gemv.h"
#include "mq_int8_plan.h"

namespace mq {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int64_t kInt8MaxK = 131072;     // 127 * 128 * K stays below 2^31
constexpr int64_t kMaxExperts = 1024;

// One product: Y[p, n] of T places, place p holding token rows[p] (or p) and belonging to the expert e with
// offsets[e] <= p < offsets[e + 1] (or to the only one).
struct Int8Args {
    const int8_t *Xq;        // [M, K]
    const float *scale;      // [M]
    const int32_t *sum;      // [M]
    const int32_t *rows;     // [T] or null
    const int32_t *offsets;  // [E + 1] or null (E = 1)
    const uint8_t *codes;    // [E, N, K]
    const float *alpha, *zero;  // [E, N]
    uint16_t *Y;             // [T, N], with a gate [T, N / 2]
    int M, T, N, K, E;
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

// scale (alpha 2^(8-r) dot - alpha (zero - offset) sum): the same fp32 steps in every kernel, and `dot` is a sum of whole numbers, so the
// outputs of all forms of the product are the same bits.  (dot and sum below 2^31 are rounded to fp32: 2^-24 of terms that the
// centring keeps near the size of the result.)  The token's scale last: it may be as small as a bf16 subnormal / 127.
__device__ __forceinline__ void channel_factors(const f32x4 &alpha, const f32x4 &zero, float mult, float offset, f32x4 &ka, f32x4 &kb) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        ka[e] = alpha[e] * mult;
        kb[e] = alpha[e] * (zero[e] - offset);
    }
}
__device__ __forceinline__ float int8_output(int dot, float sum, float scale, float ka, float kb) {
    return __builtin_fmaf(ka, (float)dot, -(kb * sum)) * scale;
}

// act(g) u, act(v) = v / (1 + exp(-t)): t = v for SiLU, 2 sqrt(2 / pi) (v + 0.044715 v^3) for GELU in its tanh form.  The gate acts on
// the fp32 outputs: one rounding, to bf16, at the end.  (The reciprocal is the hardware's, 2^-23 of its value off at most.)
__device__ __forceinline__ float gated_value(float g, float u, int gate) {
    const float t = gate == 2 ? g : 1.5957691216057308f * (g + 0.044715f * g * g * g);
    return g * __builtin_amdgcn_rcpf(1.0f + __expf(-t)) * u;
}

// The `block`-th block of BM places, counted expert by expert: no block holds places of two experts.
struct Block {
    int expert, place, count;  // count = 0: there is no such block
};
__device__ __forceinline__ Block find_block(const Int8Args &a, int block, int BM) {
    if (!a.offsets) return Block{0, block * BM, min(BM, a.T - block * BM)};
    // a lane for each expert: blocks up to and with it by a prefix sum.  (Offsets are data: whatever they hold, places stay below T.)
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int e = e0 + lane;
        int lo = 0, hi = 0;
        if (e < a.E) {
            lo = min(max(a.offsets[e], 0), a.T);
            hi = min(max(a.offsets[e + 1], lo), a.T);
        }
        const int mine = (int)(((uint32_t)(hi - lo) + (uint32_t)BM - 1u) / (uint32_t)BM);
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o, 64);
            if (lane >= o) upto += v;
        }
        const uint64_t past = __ballot(upto > block);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int first = __builtin_amdgcn_readfirstlane(__shfl(upto - mine, at, 64));
            const int place = __builtin_amdgcn_readfirstlane(__shfl(lo, at, 64)) + (block - first) * BM;
            const int end = __builtin_amdgcn_readfirstlane(__shfl(hi, at, 64));
            return Block{e0 + at, place, min(BM, end - place)};
        }
        block -= __builtin_amdgcn_readfirstlane(__shfl(upto, 63, 64));
    }
    return Block{0, 0, 0};
}
// blocks of a launch, at most
inline int64_t block_bound(int64_t T, int64_t E, bool grouped, int BM) { return grouped ? T / BM + (E < T ? E : T) : cdiv(T, BM); }

// the token of a place (rows are data: whatever they hold, tokens stay below M)
__device__ __forceinline__ int token_of(const Int8Args &a, int place) { return a.rows ? min(max(a.rows[place], 0), a.M - 1) : place; }

mq_status launch_quantize_tokens(const uint16_t *X, int64_t M, int64_t K, int64_t ldx, const int32_t *rows, int64_t X_rows, int8_t *Xq,
                                 float *scale, int32_t *sum, hipStream_t st);
mq_status launch_int8_few(const Int8Args &a, hipStream_t st);
// places: of a tile, 32 or 64; part: room for the partial sums of `splits` ranges of K
mq_status launch_int8_mid(const Int8Args &a, int places, int splits, void *part, hipStream_t st);
// places: of a tile, 128 or 256
mq_status launch_int8_tiles(const Int8Args &a, int places, hipStream_t st);

}  // namespace mq
