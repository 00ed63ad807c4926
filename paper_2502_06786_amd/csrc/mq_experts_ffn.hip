// A feed-forward layer of experts for up to 16 tokens, on planes with a scale and a zero-point for every group of inputs: two launches.
//
// gate / up: a workgroup takes 16 rows of the stacked plane of the expert of one choice (the first of those that chose it; the others
// leave at once) and multiplies them with all tokens: up to 16 tokens are one operand of the matrix core whether they chose this expert
// or not, so none has to be gathered.  Results of tokens that did not are left out where they are stored.
// down: a workgroup takes 16 rows of all chosen experts' down planes, its waves (expert, span) pairs in turn, and adds them with the
// tokens' weights in one order: no expert's output is stored, no atomics.
//
// The gated products go from one launch to the other as two bf16 numbers each (the value rounded, and what that leaves, rounded):
// 16 significant bits.  One bf16 number alone would add an error of its own as large as that of the rounded result.
#include "mq_gemv.h"
#include "mq_grouped.h"

namespace mq {

constexpr int gate_up_span(int c) { return c == 32 ? 256 : 512; }
constexpr int down_span(int r, int c) { return c == 32 || (r == 2 && c == 64) ? 128 : 256; }
constexpr int kFfnTop = 16, kFfnChoices = kGroupedTokens * kFfnTop;

struct ExpertsFfnArgs {
    const uint16_t *x;      // [B, d]
    const int32_t *ids;     // [B, top]
    const float *weight;    // [B, top]
    const uint8_t *gate_up, *down;
    const uint16_t *alpha_gu, *zero_gu, *alpha_dn, *zero_dn;
    uint16_t *y;            // [B, d]
    // in the workspace, a row for every choice
    uint16_t *act, *rest;   // [n, F] gated products in operand order: rounded, what that leaves
    int32_t *expert;        // [n] the expert of the first choice of each expert, -1 in the others
    float *share;           // [n, 16] each token's weight for that expert
    int32_t *row;           // [n, 16] row of act of each token, -1 where it did not choose the expert
    int B, top, n, E, d, F, groups_d, groups_F, ks;
    GroupOf group;
    int silu, residual;
};

// The `width` bits from bit `at` of a mask of 256 bits.
__device__ __forceinline__ uint32_t mask_window(const uint64_t (&m)[4], int at, int width) {
    const int w = at >> 6, sh = at & 63;
    const uint64_t a = w == 0 ? m[0] : w == 1 ? m[1] : w == 2 ? m[2] : m[3];
    const uint64_t b = w == 0 ? m[1] : w == 1 ? m[2] : w == 2 ? m[3] : 0;
    const uint64_t v = sh ? a >> sh | b << (64 - sh) : a;
    return (uint32_t)v & ((1u << width) - 1);
}

template <int R, int C>
__global__ __launch_bounds__(64 * 16) void experts_gate_up_kernel(ExpertsFfnArgs a) {
    constexpr int SPAN = gate_up_span(C);
    __shared__ f32x4 part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, quarter = lane >> 4;
    const int choice = blockIdx.y, e = a.ids[choice];
    bool first = e >= 0 && e < a.E;
    uint64_t same[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = 64 * i + lane;
        same[i] = __ballot(c < a.n && a.ids[min(c, a.n - 1)] == e);
        if (choice >> 6 > i) first = first && same[i] == 0;
        if (choice >> 6 == i) first = first && (same[i] & ((1ull << (choice & 63)) - 1)) == 0;
    }
    const uint32_t mine = li < a.B ? mask_window(same, li * a.top, a.top) : 0;  // which choices of token li are this expert
    const int row_of_act = mine ? li * a.top + __builtin_ctz(mine) : -1;
    if (blockIdx.x == 0 && threadIdx.x < 16) {
        if (threadIdx.x == 0) a.expert[choice] = first ? e : -1;
        if (first) {
            float share = 0.f;
            for (uint32_t m = mine; m; m &= m - 1) share += a.weight[li * a.top + __builtin_ctz(m)];
            a.share[choice * 16 + li] = share;
            a.row[choice * 16 + li] = row_of_act;
        }
    }
    if (!first) return;

    const int tile = wave / a.ks, ks = wave - tile * a.ks, tiles = (int)(blockDim.x >> 6) / a.ks;
    const int row0 = ((int)blockIdx.x * tiles + tile) * kGroupedRows, chunks = a.d / C;
    const int64_t row = (int64_t)e * 2 * a.F + min(row0, 2 * a.F - kGroupedRows) + li;
    GroupedLane p;
    p.codes = a.gate_up + row * (a.d / 8 * R) + quarter * (C * R / 32);
    p.alpha = a.alpha_gu + row * a.groups_d;
    p.zero = a.zero_gu + row * a.groups_d;
    p.x = a.x + (int64_t)min(li, a.B - 1) * a.d + quarter * (C / 4);
    p.rest = nullptr;
    f32x4 y{0.f, 0.f, 0.f, 0.f};
    if (row0 < 2 * a.F)
        for (int c = ks * (SPAN / C); c < chunks; c += a.ks * (SPAN / C)) grouped_span<R, C, SPAN, 1>(p, c, chunks, a.group, y);
    if (a.ks > 1) {
        part[wave][lane] = y;
        __syncthreads();
        if (ks != 0) return;
        for (int k = 1; k < a.ks; ++k) y += part[wave + k][lane];
    }
    if (row0 >= 2 * a.F) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // rows 2 f and 2 f + 1 are neighbouring lanes
        const float other = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(y[i]), 0xB1, 0xF, 0xF, true));
        const int at = __builtin_amdgcn_ds_bpermute((4 * quarter + i) << 2, row_of_act);
        if (li & 1 || at < 0) continue;
        const float v = (a.silu ? silu(y[i]) : gelu_tanh(y[i])) * other;
        const int64_t out = (int64_t)at * a.F + operand_place<R>((row0 + li) >> 1);
        const uint32_t hi = float_to_bf16_bits(v);
        a.act[out] = (uint16_t)hi;
        a.rest[out] = (uint16_t)float_to_bf16_bits(v - bf16_bits_to_float(hi));
    }
}

template <int R, int C>
__global__ __launch_bounds__(64 * 16) void experts_down_kernel(ExpertsFfnArgs a) {
    constexpr int SPAN = down_span(R, C);
    __shared__ f32x4 part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, quarter = lane >> 4, waves = (int)(blockDim.x >> 6);
    const int row0 = (int)blockIdx.x * kGroupedRows, chunks = a.F / C, spans = (chunks + SPAN / C - 1) / (SPAN / C);
    uint64_t chosen[4];
    int experts = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = 64 * i + lane;
        chosen[i] = __ballot(c < a.n && a.expert[min(c, a.n - 1)] >= 0);
        experts += __popcll(chosen[i]);
    }
    f32x4 total{0.f, 0.f, 0.f, 0.f};
    int at = -1, choice = 0;  // the expert reached so far, by its number among the chosen
    for (int item = wave; item < experts * spans; item += waves) {
        const int want = item / spans;
        while (at < want) {
            ++at;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (chosen[i]) {
                    choice = 64 * i + __builtin_ctzll(chosen[i]);
                    chosen[i] &= chosen[i] - 1;
                    break;
                }
        }
        const int e = a.expert[choice];
        const int64_t row = (int64_t)e * a.d + row0 + li;
        const int mine = a.row[choice * 16 + li];
        const int64_t act = (int64_t)(mine >= 0 ? mine : choice) * a.F + quarter * (C / 4);
        GroupedLane p;
        p.codes = a.down + row * (a.F / 8 * R) + quarter * (C * R / 32);
        p.alpha = a.alpha_dn + row * a.groups_F;
        p.zero = a.zero_dn + row * a.groups_F;
        p.x = a.act + act;
        p.rest = a.rest + act;
        const f32x4 share = *reinterpret_cast<const f32x4 *>(a.share + choice * 16 + 4 * quarter);
        const u32x4 rows = *reinterpret_cast<const u32x4 *>(a.row + choice * 16 + 4 * quarter);
        f32x4 o{0.f, 0.f, 0.f, 0.f};
        grouped_span<R, C, SPAN, 2>(p, (item - want * spans) * (SPAN / C), chunks, a.group, o);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((int)rows[i] >= 0) total[i] = __builtin_fmaf(share[i], o[i], total[i]);
    }
    if (waves > 1) {
        part[wave][lane] = total;
        __syncthreads();
        if (wave != 0) return;
        for (int k = 1; k < waves; ++k) total += part[k][lane];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 4 * quarter + i;
        if (t >= a.B) continue;
        const int64_t out = (int64_t)t * a.d + row0 + li;
        if (a.residual) total[i] += bf16_bits_to_float(a.x[out]);
        a.y[out] = (uint16_t)float_to_bf16_bits(total[i]);
    }
}

namespace {

struct ExpertsFfnLayout {
    size_t act, rest, expert, share, row, total;
};

ExpertsFfnLayout experts_ffn_layout(int64_t n, int64_t F) {
    auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
    ExpertsFfnLayout l;
    l.act = 0;
    l.rest = up((size_t)n * F * 2);
    l.expert = l.rest + up((size_t)n * F * 2);
    l.share = l.expert + up((size_t)n * 4);
    l.row = l.share + up((size_t)n * 64);
    l.total = l.row + up((size_t)n * 64);
    return l;
}

template <int R, int C>
void launch_gate_up(ExpertsFfnArgs a, hipStream_t st) {
    const int spans = (int)cdiv(a.d, gate_up_span(C)), turns = (int)cdiv(spans, 16);
    a.ks = (int)cdiv(spans, turns);
    const int tiles = a.ks >= 4 ? 1 : 4 / a.ks;
    experts_gate_up_kernel<R, C><<<dim3((unsigned)cdiv(2 * a.F, kGroupedRows * tiles), a.n), dim3(64 * a.ks * tiles), 0, st>>>(a);
}

template <int R, int C>
void launch_down(const ExpertsFfnArgs &a, hipStream_t st) {
    const int items = a.n * (int)cdiv(a.F, down_span(R, C));
    experts_down_kernel<R, C><<<dim3((unsigned)(a.d / kGroupedRows)), dim3(64 * std::min(16, items)), 0, st>>>(a);
}

}  // namespace

size_t experts_ffn_workspace_bytes(int64_t n, int64_t F) {
    if (n < 1 || n > kFfnChoices || F < 1 || F > (1 << 20)) return 0;
    return experts_ffn_layout(n, F).total + 256;
}

}  // namespace mq

extern "C" mq_status mq_experts_ffn(const uint16_t *x, const mq_ffn_layer *layer, const int32_t *ids, const float *weight, int64_t B, int64_t top,
                                    int64_t E, int64_t d, int64_t F, int64_t group, uint32_t flags, uint16_t *y, void *ws, size_t ws_bytes,
                                    void *hip_stream) {
    using namespace mq;
    if (!layer) return MQ_ERR_NULL;
    const int r = layer->r;
    if (flags & ~(uint32_t)(MQ_FLAG_FFN_SILU | MQ_FLAG_FFN_RESIDUAL)) return MQ_ERR_BITS;
    if (B < 1 || B > kGroupedTokens || top < 1 || top > kFfnTop || E < 1 || E > 1024 || d < 1 || F < 1 || d > (1 << 20) || F > (1 << 20)) return MQ_ERR_SHAPE;
    mq_status s = grouped_check(layer->gate_up, layer->alpha_gu, layer->zero_gu, 2 * F, d, group ? group : d, r);
    if (s == MQ_OK) s = grouped_check(layer->down, layer->alpha_dn, layer->zero_dn, d, F, group ? group : F, r);
    if (s != MQ_OK) return s;
    if (!x || !ids || !weight || !y) return MQ_ERR_NULL;
    if (!aligned16(x) || !aligned16(ids) || !aligned16(weight) || !aligned16(y)) return MQ_ERR_ALIGN;
    const ExpertsFfnLayout l = experts_ffn_layout(B * top, F);
    if (!ws || !aligned16(ws) || ws_bytes < l.total + 256) return MQ_ERR_WORKSPACE;
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
    ExpertsFfnArgs a{x, ids, weight, layer->gate_up, layer->down, layer->alpha_gu, layer->zero_gu, layer->alpha_dn, layer->zero_dn, y,
                     reinterpret_cast<uint16_t *>(base + l.act), reinterpret_cast<uint16_t *>(base + l.rest), reinterpret_cast<int32_t *>(base + l.expert),
                     reinterpret_cast<float *>(base + l.share), reinterpret_cast<int32_t *>(base + l.row), (int)B, (int)top, (int)(B * top), (int)E,
                     (int)d, (int)F, (int)(group ? d / group : 1), (int)(group ? F / group : 1), 1, GroupOf{1, 0}, (flags & MQ_FLAG_FFN_SILU) != 0,
                     (flags & MQ_FLAG_FFN_RESIDUAL) != 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    for (int down = 0; down < 2; ++down) {
        const int64_t g = group ? group : down ? F : d;
        int c = chunk_codes(r, g);
        a.group = group_of(g / c);
#define MQ_EXPERTS_CASE(R_, C_) \
    if (r == R_ && c == C_) down ? launch_down<R_, C_>(a, st) : launch_gate_up<R_, C_>(a, st);
        MQ_EXPERTS_CASE(4, 128) MQ_EXPERTS_CASE(4, 64) MQ_EXPERTS_CASE(4, 32)
        MQ_EXPERTS_CASE(2, 256) MQ_EXPERTS_CASE(2, 128) MQ_EXPERTS_CASE(2, 64)
        MQ_EXPERTS_CASE(8, 64) MQ_EXPERTS_CASE(8, 32)
#undef MQ_EXPERTS_CASE
        s = launch_status();
        if (s != MQ_OK) return s;
    }
    return MQ_OK;
}
