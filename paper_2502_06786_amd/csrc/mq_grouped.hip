// Matrix-vector products with planes that have a scale and a zero-point for every group of inputs.
#include <algorithm>

#include "mq_grouped.h"

namespace mq {

struct GroupedGemvArgs {
    const uint16_t *x;      // [B, K] bf16
    const uint8_t *packed;  // [N, K R / 8]
    const uint16_t *alpha, *zero;  // [N, groups] bf16
    uint16_t *y;            // [B, N] bf16
    int B, N, K, groups, ks;
    GroupOf group;
};

// waves of a workgroup at most: 16 leave 128 registers to each, 8 256
constexpr int gemv_waves(int R, int C, int RG, int T, int D) {
    return (R == 2 && (T == 16 || RG == 2)) || (R == 4 && C == 32 && RG == 2) ? 8 : 16;
}

// A workgroup takes 16 RG rows, its waves stretches of them in turn; the waves' sums meet in LDS.
// Large planes of four and eight bits are bound by HBM (73728 x 4608, r = 4, B = 1: 35.2 us, 5.1 TB/s; 73728 x 4096, r = 8: 63.1 us, 4.9 TB/s; shorter ones are
// over before that: 28672 x 4096, r = 8: 31.3 us, 4.0 TB/s).  At two bits nothing is full (73728 x 4096, B = 1: 27.5 us, 3.1 TB/s; 28672 x 4096: 13.7 us, 2.7
// TB/s, with the vector unit busy for 0.53 of the cycles, the matrix core for 0.26, LDS for 0.33; waves wait for memory for 0.27 of their time and for
// their turn for 0.44).  Nor with 16 tokens, which come from the L2 once for every 16 RG rows (4096 x 14336, groups of 32, r = 4: 13.1 us, 2.8 TB/s, 159 MB of
// requests to the L2 for a plane of 37 MB; vector unit 0.41, LDS 0.33, matrix core 0.11; waves wait for memory for 0.46 of their time, 2.5 of them to a SIMD).
// Small planes are bound by launch, first lines and end (4096 x 4096, B = 1: 4.6 us, 1.9 TB/s).
template <int R, int C, int RG, int T, int D>
__global__ __launch_bounds__(64 * gemv_waves(R, C, RG, T, D)) void gemv_grouped_kernel(GroupedGemvArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    using G = Grouped<R, C, RG, T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, quarter = lane >> 4;
    const int row0 = (int)blockIdx.x * kGroupedRows * RG, stretches = (a.K + stretch_codes(R) - 1) / stretch_codes(R);
    f32x4 y[RG];
#pragma unroll
    for (int t = 0; t < RG; ++t) y[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    int at = wave;
    grouped_stream<R, C, RG, T, false, D>(
        lds + wave * G::LDS, token_buffer(a.x, 2 * (uint32_t)(a.B * a.K)), a.N - row0, a.K, a.groups, a.group, y,
        [&](Stretch<G::XI> &s) {
            if (at >= stretches) return false;
            s.codes = a.packed + (int64_t)row0 * (a.K / 8 * R);
            s.alpha = a.alpha + (int64_t)row0 * a.groups;
            s.zero = a.zero + (int64_t)row0 * a.groups;
#pragma unroll
            for (int i = 0; i < G::XI; ++i) s.token[i] = 2 * (uint32_t)(min(load_token<G>(i), a.B - 1) * a.K + load_input<G>(i));
            s.first = at * kPieces * kHalves;
            at += a.ks;
            return true;
        },
        [](const Stretch<G::XI> &) {});
    join_waves<RG>(reinterpret_cast<f32x4 *>(lds), wave, a.ks, y);
    if (wave != 0) return;
#pragma unroll
    for (int t = 0; t < RG; ++t) {
        const int row = row0 + 16 * t + li;
        if (row >= a.N) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * quarter + i < a.B) a.y[(int64_t)(4 * quarter + i) * a.N + row] = (uint16_t)float_to_bf16_bits(y[t][i]);
    }
}

mq_status grouped_check(const uint8_t *packed, const uint16_t *alpha, const uint16_t *zero, int64_t rows, int64_t K, int64_t group, int r) {
    if (r != 8 && r != 4 && r != 2) return MQ_ERR_BITS;
    if (K < 1 || K > (1 << 20) || rows < 0 || rows > (1 << 25) || group < 1 || group > K || K % group != 0) return MQ_ERR_SHAPE;
    if (group % group_unit(r) != 0) return MQ_ERR_ALIGN;
    if (rows == 0) return MQ_OK;
    if (!packed || !alpha || !zero) return MQ_ERR_NULL;
    if (!aligned16(packed) || !aligned16(alpha) || !aligned16(zero)) return MQ_ERR_ALIGN;
    return MQ_OK;
}

template <int R, int C, int RG, int T, int D>
static mq_status launch_gemv_grouped_as(GroupedGemvArgs a, hipStream_t st) {
    using G = Grouped<R, C, RG, T>;
    const int64_t stretches = cdiv(a.K, stretch_codes(R)), blocks = cdiv(a.N, kGroupedRows * RG);
    // Waves of a workgroup: 12 on each compute unit where there is no more than a workgroup or two for each (4096 x 14336, B = 16: 11.8 us, with
    // 14 waves instead of 10 12.9), otherwise 24, of which 16 to 20 are there at a time (73728 x 4608, B = 1: 34.9 us, half as many 39.4).
    const int64_t wanted = cdiv((blocks <= 512 ? 12 : 24) * 256, blocks);
    a.ks = (int)std::min<int64_t>({stretches, gemv_waves(R, C, RG, T, D), 163840 / G::LDS, wanted});
    a.ks = (int)cdiv(stretches, cdiv(stretches, a.ks));
    const int lds = a.ks * G::LDS;
    constexpr auto kernel = gemv_grouped_kernel<R, C, RG, T, D>;
    if (lds > 65536 && !allow_lds<kernel>(lds)) return MQ_ERR_DEVICE;
    kernel<<<dim3((unsigned)blocks), dim3(64 * a.ks), lds, st>>>(a);
    return launch_status();
}

template <int R, int C, int T>
static mq_status launch_gemv_grouped(const GroupedGemvArgs &a, hipStream_t st) {
    // (a piece under way beside the one that is multiplied, where registers allow it)
    constexpr int D1 = T > 4 || R == 2 ? 1 : 2, D2 = T > 4 ? 1 : 2;
    if constexpr (gemv_two_tiles_fit(R, C, T))
        if (gemv_tiles(R, C, a.B, a.N) == 2) return launch_gemv_grouped_as<R, C, 2, T, D2>(a, st);
    return launch_gemv_grouped_as<R, C, 1, T, D1>(a, st);
}

}  // namespace mq

extern "C" mq_status mq_gemv_grouped(const uint16_t *x, const uint8_t *packed, const uint16_t *alpha_bf16, const uint16_t *zero_bf16,
                                     int64_t B, int64_t N, int64_t K, int64_t group, int r, uint16_t *y, void *hip_stream) {
    using namespace mq;
    if (B < 1 || B > kGroupedTokens) return MQ_ERR_SHAPE;
    const mq_status s = grouped_check(packed, alpha_bf16, zero_bf16, N, K, group, r);
    if (s != MQ_OK || N == 0) return s;
    if (!x || !y) return MQ_ERR_NULL;
    if (!aligned16(x) || !aligned16(y)) return MQ_ERR_ALIGN;
    const int c = chunk_codes(r, group);
    const GroupedGemvArgs a{x, packed, alpha_bf16, zero_bf16, y, (int)B, (int)N, (int)K, (int)(K / group), 1, group_of(group / c)};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
#define MQ_GROUPED_CASE(R_, C_)                                                    \
    if (r == R_ && c == C_)                                                        \
        return token_class(B) == 4   ? launch_gemv_grouped<R_, C_, 4>(a, st)       \
               : token_class(B) == 8 ? launch_gemv_grouped<R_, C_, 8>(a, st)       \
                                     : launch_gemv_grouped<R_, C_, 16>(a, st);
    MQ_GROUPED_CASE(4, 128) MQ_GROUPED_CASE(4, 64) MQ_GROUPED_CASE(4, 32)
    MQ_GROUPED_CASE(2, 256) MQ_GROUPED_CASE(2, 128) MQ_GROUPED_CASE(2, 64)
    MQ_GROUPED_CASE(8, 64) MQ_GROUPED_CASE(8, 32)
#undef MQ_GROUPED_CASE
    return MQ_ERR_BITS;
}
