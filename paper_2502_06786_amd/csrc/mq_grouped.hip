// Matrix-vector products with planes that have a scale and a zero-point for every group of inputs.
#include "mq_grouped.h"

namespace mq {

struct GroupedGemvArgs {
    const uint16_t *x;      // [B, K] bf16
    const uint8_t *packed;  // [N, K R / 8]
    const uint16_t *alpha, *zero;  // [N, groups] bf16
    uint16_t *y;            // [B, N] bf16
    int B, N, K, groups, chunks, ks;
    GroupOf group;
};

constexpr int kGroupedWaves = 16;
// codes of a row that a wave has under way at a time, as far as its registers go
constexpr int grouped_gemv_span(int c) { return c == 32 ? 256 : 512; }

// A workgroup takes 16 rows (or a few times 16 where rows are short), its waves spans of 512 codes (256 where groups are short) of them in turn: all loads of a span
// leave together, and what hides their latency is the other waves of the compute unit.  The waves' sums meet in LDS.
template <int R, int C>
__global__ __launch_bounds__(64 * kGroupedWaves) void gemv_grouped_kernel(GroupedGemvArgs a) {
    constexpr int SPAN = grouped_gemv_span(C);
    __shared__ f32x4 part[kGroupedWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, quarter = lane >> 4;
    const int tile = wave / a.ks, ks = wave - tile * a.ks, tiles = (int)(blockDim.x >> 6) / a.ks;
    const int row0 = ((int)blockIdx.x * tiles + tile) * kGroupedRows;
    const int row = min(row0 + li, a.N - 1), token = min(li, a.B - 1);
    GroupedLane p;
    p.codes = a.packed + (int64_t)row * (a.K / 8 * R) + quarter * (C * R / 32);
    p.alpha = a.alpha + (int64_t)row * a.groups;
    p.zero = a.zero + (int64_t)row * a.groups;
    p.x = a.x + (int64_t)token * a.K + quarter * (C / 4);
    p.rest = nullptr;
    f32x4 y{0.f, 0.f, 0.f, 0.f};
    if (row0 < a.N)
        for (int c = ks * (SPAN / C); c < a.chunks; c += a.ks * (SPAN / C))
            grouped_span<R, C, SPAN, 1>(p, c, a.chunks, a.group, y);
    if (a.ks > 1) {
        part[wave][lane] = y;
        __syncthreads();
        if (ks != 0) return;
        for (int k = 1; k < a.ks; ++k) y += part[wave + k][lane];
    }
    if (row0 + li >= a.N) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * quarter + i < a.B) a.y[(int64_t)(4 * quarter + i) * a.N + row0 + li] = (uint16_t)float_to_bf16_bits(y[i]);
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

template <int R, int C>
static mq_status launch_gemv_grouped(GroupedGemvArgs a, hipStream_t st) {
    const int spans = (int)cdiv(a.K, grouped_gemv_span(C)), turns = (int)cdiv(spans, kGroupedWaves);
    a.ks = (int)cdiv(spans, turns);
    const int tiles = a.ks >= 4 ? 1 : 4 / a.ks;
    gemv_grouped_kernel<R, C><<<dim3((unsigned)cdiv(a.N, kGroupedRows * tiles)), dim3(64 * a.ks * tiles), 0, st>>>(a);
    return launch_status();
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
    const GroupedGemvArgs a{x, packed, alpha_bf16, zero_bf16, y, (int)B, (int)N, (int)K, (int)(K / group), (int)(K / c), 1, group_of(group / c)};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
#define MQ_GROUPED_CASE(R_, C_) \
    if (r == R_ && c == C_) return launch_gemv_grouped<R_, C_>(a, st);
    MQ_GROUPED_CASE(4, 128) MQ_GROUPED_CASE(4, 64) MQ_GROUPED_CASE(4, 32)
    MQ_GROUPED_CASE(2, 256) MQ_GROUPED_CASE(2, 128) MQ_GROUPED_CASE(2, 64)
    MQ_GROUPED_CASE(8, 64) MQ_GROUPED_CASE(8, 32)
#undef MQ_GROUPED_CASE
    return MQ_ERR_BITS;
}
