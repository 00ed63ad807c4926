// A feed-forward layer of experts for up to 16 tokens, on planes with a scale and a zero-point for every group of inputs: two launches.
//
// gate / up: a workgroup takes rows of the stacked plane of the expert of one choice (the first of those that chose it; the others leave at
// once) and multiplies them with the tokens that chose it, up to 16 of them side by side, so each expert's plane is read once.
// down: a workgroup takes rows of all chosen experts' down planes, its waves (tokens of an expert, stretch) pairs in turn, and adds them with
// the tokens' weights in an order that the sizes and the choices fix.  Where there are few rows, several workgroups share the pairs of the
// same rows, and the last one to arrive adds their sums, in the order of the workgroups.
//
// The gated products go from one launch to the other as two bf16 numbers each (the value rounded, and what that leaves, rounded): 16
// significant bits.  One bf16 number alone would add an error of its own as large as that of the rounded result.  The two are two tokens of
// the product, whose results are added at its end.
#include <algorithm>

#include "mq_gemv.h"
#include "mq_grouped.h"

namespace mq {

// waves of a workgroup at most: 8 leave 256 registers to each, 12 168 (16 leave 128, which spill: 16 tokens x 2 of 8, 4096 x 14336, r = 4:
// 189 us, with 12 171)
constexpr int kGateUpWaves = 8;
constexpr int down_waves(int R) { return R == 2 ? 8 : 12; }
constexpr int kFfnTop = 16, kFfnChoices = kGroupedTokens * kFfnTop;

struct ExpertsFfnArgs {
    const uint16_t *x;      // [B, d]
    const int32_t *ids;     // [B, top]
    const float *weight;    // [B, top]
    const uint8_t *gate_up, *down;
    const uint16_t *alpha_gu, *zero_gu, *alpha_dn, *zero_dn;
    uint16_t *y;            // [B, d]
    // in the workspace
    uint16_t *act, *rest;   // [n, F] a choice's gated products in operand order: rounded, what that leaves
    // [2 n] up to 8 tokens of an expert each: of the expert that choice c is the first to choose, tokens 0 .. 7 of it in entry c, the others in entry n + c
    int32_t *count, *expert;
    uint8_t *token;         // [2 n, 8]
    int32_t *row;           // [2 n, 8] rows of act
    float *share;           // [2 n, 8] weights
    float *part;            // [tiles of rows][splits][B, rows] sums of workgroups that share rows
    uint32_t *arrived;      // [tiles of rows] how many of them have left theirs; cleared by the first launch
    int B, top, n, E, d, F, groups_d, groups_F, ks, splits;
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

// lane `to` gets v (lanes that send to the same one: any of theirs)
__device__ __forceinline__ int send_to(int to, int v) { return __builtin_amdgcn_ds_permute(to << 2, v); }
__device__ __forceinline__ int take_from(int from, int v) { return __builtin_amdgcn_ds_bpermute(from << 2, v); }

// MOST: tokens that an expert may have, 4, 8 or 16.  Experts with up to 4 load no more than 4 (16 tokens x 2 of 8, 4096 x 14336, r = 4: 168 us,
// otherwise 178; x 4 of 128, 2048 x 1408: 50 and 54.5).
// At four and eight bits bound by HBM where experts are large (the first of these layers: 7 or 8 experts, 437 or 499 MB, in 92 to 112 us by card, 4.5 to 5.0 TB/s;
// at eight bits 0.85 or 0.97 GB in 170 to 200 us, 4.9 to 5.0), by the start of a workgroup (who chose what, first lines, 2 to 3 us) where they are
// small (one token x 8 of 64, 2048 x 1024: 18 MB in 7.8 us).  At two bits nothing is full (5 tokens x 2 of 8, 2304 x 9216: 26 to 36 us, 2.4 TB/s; vector
// unit busy for 0.57 of the cycles, matrix core for 0.25, LDS for 0.34; about 45 instructions to 1024 codes and a load, 10 of them unpack; waves wait for
// memory for 0.42 of their time), and one token takes longer than at four bits (x 2 of 8, 4096 x 14336, groups of 64: 33.5 us, at four bits with groups of 128
// 28.8; vector unit 0.66).
template <int R, int C, int RG, int MOST, int D>
__global__ __launch_bounds__(64 * kGateUpWaves) void experts_gate_up_kernel(ExpertsFfnArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, quarter = lane >> 4;
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
    if (choice == 0)
        for (int i = (int)(blockIdx.x * blockDim.x + threadIdx.x); i < a.d / kGroupedRows; i += (int)(gridDim.x * blockDim.x)) a.arrived[i] = 0;
    const uint32_t mine = li < a.B ? mask_window(same, li * a.top, a.top) : 0;  // which choices of token li are this expert
    const uint64_t who = __ballot(mine != 0 && lane < 16);
    const int count = __popcll(who);
    if (blockIdx.x == 0 && threadIdx.x < 2) {
        a.count[threadIdx.x * a.n + choice] = first ? (threadIdx.x ? max(count - 8, 0) : min(count, 8)) : 0;
        a.expert[threadIdx.x * a.n + choice] = e;
    }
    if (!first) return;
    // lane p gets the expert's token p and the row of act for it
    const int place = mine != 0 && lane < 16 ? __popcll(who & ((1ull << lane) - 1)) : 63;
    const int token = send_to(place, li), row_of_act = send_to(place, mine ? li * a.top + __builtin_ctz(mine) : 0);
    if (blockIdx.x == 0 && wave == 0) {
        float share = 0.f;
        if (lane < 16)
            for (uint32_t m = mine; m; m &= m - 1) share += a.weight[li * a.top + __builtin_ctz(m)];
        share = __int_as_float(send_to(place, __float_as_int(share)));
        if (lane < count) {
            const int at = (choice + (lane >> 3) * a.n) * 8 + (lane & 7);
            a.token[at] = (uint8_t)token;
            a.row[at] = row_of_act;
            a.share[at] = share;
        }
    }

    const int row0 = (int)blockIdx.x * kGroupedRows * RG, stretches = (a.d + stretch_codes(R) - 1) / stretch_codes(R);
    const int64_t first_row = (int64_t)e * 2 * a.F + row0;
    f32x4 y[RG];
#pragma unroll
    for (int t = 0; t < RG; ++t) y[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto products = [&](auto tokens, auto ahead) {
        constexpr int T = decltype(tokens)::value;
        using G = Grouped<R, C, RG, T>;
        int at = wave;
        uint32_t begin[G::XI];
#pragma unroll
        for (int i = 0; i < G::XI; ++i) begin[i] = 2 * (uint32_t)(take_from(min(load_token<G>(i), count - 1), token) * a.d + load_input<G>(i));
        grouped_stream<R, C, RG, T, false, decltype(ahead)::value>(
            lds + wave * Grouped<R, C, RG, MOST>::LDS, token_buffer(a.x, 2 * (uint32_t)(a.B * a.d)), 2 * a.F - row0, a.d, a.groups_d, a.group, y,
            [&](Stretch<G::XI> &s) {
                if (at >= stretches) return false;
                s.codes = a.gate_up + first_row * (a.d / 8 * R);
                s.alpha = a.alpha_gu + first_row * a.groups_d;
                s.zero = a.zero_gu + first_row * a.groups_d;
#pragma unroll
                for (int i = 0; i < G::XI; ++i) s.token[i] = begin[i];
                s.first = at * kPieces * kHalves;
                at += a.ks;
                return true;
            },
            [](const Stretch<G::XI> &) {});
    };
    if (MOST == 4 || count <= 4)
        products(std::integral_constant<int, 4>{}, std::integral_constant<int, D>{});
    else
        products(std::integral_constant<int, MOST>{}, std::integral_constant<int, 1>{});
    join_waves<RG>(reinterpret_cast<f32x4 *>(lds), wave, a.ks, y);
    if (wave == 0)
#pragma unroll
        for (int t = 0; t < RG; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // rows 2 f and 2 f + 1 are neighbouring lanes
                const float other = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(y[t][i]), 0xB1, 0xF, 0xF, true));
                const int mine = 4 * quarter + i, to = take_from(mine, row_of_act), row = row0 + 16 * t + li;
                if (li & 1 || mine >= count || row >= 2 * a.F) continue;
                const float v = (a.silu ? silu(y[t][i]) : gelu_tanh(y[t][i])) * other;
                const int64_t out = (int64_t)to * a.F + operand_place<R>(row >> 1);
                const uint32_t hi = float_to_bf16_bits(v);
                a.act[out] = (uint16_t)hi;
                a.rest[out] = (uint16_t)float_to_bf16_bits(v - bf16_bits_to_float(hi));
            }
}

// LDS of the down kernel: for each wave its part of the products and 16 tokens x 16 RG rows of sums; the entries in use.
template <int R, int C, int RG, int MOST>
struct DownLds {
    static constexpr int STREAM = Grouped<R, C, RG, 2 * MOST>::LDS, WAVE = STREAM + 1024 * RG, LIST = 2 * kFfnChoices * 8 + 16;
};

// MOST: tokens of an entry, 4 or 8.  blockIdx.y: which of the workgroups that share the rows
// One workgroup to a compute unit, three waves to a SIMD: bound by waiting (16 tokens x 2 of 8, 4096 x 14336, r = 4: 250 MB in 62 to 77 us, 3.2 to 3.7 TB/s, 654 MB of
// requests to the L2, the vector unit busy for 0.46 of the cycles, LDS for 0.46, the matrix core for 0.18, waves waiting for memory for 0.39 of their time;
// 16 x 4 of 128, 2048 x 1408: 0.34, 0.32, 0.12 and 0.39), for small layers by start and end (one token x 8 of 64, 2048 x 1024: 9 MB in 7.0 us).
template <int R, int C, int RG, int MOST, int D>
__global__ __launch_bounds__(64 * down_waves(R)) void experts_down_kernel(ExpertsFfnArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    using Lds = DownLds<R, C, RG, MOST>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, quarter = lane >> 4;
    const int waves = (int)(blockDim.x >> 6), row0 = (int)blockIdx.x * kGroupedRows * RG, stretches = (a.F + stretch_codes(R) - 1) / stretch_codes(R);
    uint8_t *const mine = lds + Lds::LIST + wave * Lds::WAVE;
    float *const sums = reinterpret_cast<float *>(mine + Lds::STREAM);  // [token][row]
    // (entry, tokens << 16; expert): entries of up to 4 tokens from the front, of more from the back
    u32x2 *const list = reinterpret_cast<u32x2 *>(lds);
    int *const totals = reinterpret_cast<int *>(lds + Lds::LIST - 16);
    const int entries = MOST == 4 ? a.n : 2 * a.n;  // (4 tokens fill no second entry)
    if (wave == 0) {
        int few = 0, more = 0;
        for (int at = 0; at < entries; at += 64) {
            const int entry = at + lane, count = entry < entries ? a.count[entry] : 0, expert = a.expert[min(entry, entries - 1)];
            const u32x2 word = {(uint32_t)entry | (uint32_t)count << 16, (uint32_t)expert};
            const uint64_t f = __ballot(count > 0 && count <= 4), m = __ballot(count > 4), below = (1ull << lane) - 1;
            if (count > 4)
                list[2 * kFfnChoices - 1 - more - __popcll(m & below)] = word;
            else if (count > 0)
                list[few + __popcll(f & below)] = word;
            few += __popcll(f);
            more += __popcll(m);
        }
        if (lane == 0) totals[0] = few, totals[1] = more;
    }
#pragma unroll
    for (int t = 0; t < RG; ++t) *reinterpret_cast<f32x4 *>(sums + (t * 64 + lane) * 4) = f32x4{0.f, 0.f, 0.f, 0.f};
    __syncthreads();
    f32x4 y[RG];
#pragma unroll
    for (int t = 0; t < RG; ++t) y[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int few = totals[0], more = totals[1], step = waves * a.splits, first = (int)blockIdx.y + wave * a.splits;
    const uint32_t rest = (uint32_t)(a.rest - a.act);
    // up to TOKENS tokens of an entry: as many rounded values, then as many rests
    auto products = [&](auto tokens, auto ahead, int items, auto entry_of, int start) {
        constexpr int TOKENS = decltype(tokens)::value;
        using G = Grouped<R, C, RG, 2 * TOKENS>;
        int item = start;
        grouped_stream<R, C, RG, 2 * TOKENS, true, decltype(ahead)::value>(
            mine, token_buffer(a.act, 2 * (rest + (uint32_t)(a.n * a.F))), a.d - row0, a.F, a.groups_F, a.group, y,
            [&](Stretch<G::XI> &s) {
                if (item >= items) return false;
                const int which = item / stretches;
                const u32x2 word = entry_of(which);
                const int packed = __builtin_amdgcn_readfirstlane((int)word[0]), entry = packed & 0xFFFF;
                const int64_t first_row = (int64_t)__builtin_amdgcn_readfirstlane((int)word[1]) * a.d + row0;
                s.count = packed >> 16;
                s.codes = a.down + first_row * (a.F / 8 * R);
                s.alpha = a.alpha_dn + first_row * a.groups_F;
                s.zero = a.zero_dn + first_row * a.groups_F;
#pragma unroll
                for (int i = 0; i < G::XI; ++i) {
                    const int t = load_token<G>(i) % (2 * TOKENS);
                    s.token[i] = 2 * ((uint32_t)a.row[entry * 8 + min(t % TOKENS, s.count - 1)] * (uint32_t)a.F + (t < TOKENS ? 0u : rest) + load_input<G>(i));
                }
                s.first = (item - which * stretches) * kPieces * kHalves;
                s.tokens = *reinterpret_cast<const uint32_t *>(a.token + entry * 8 + 4 * (quarter & 1));
                s.share = *reinterpret_cast<const f32x4 *>(a.share + entry * 8 + 4 * (quarter & 1));
                item += step;
                return true;
            },
            [&](const Stretch<G::XI> &s) {
#pragma unroll
                for (int t = 0; t < RG; ++t) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = y[t][i] + __int_as_float(take_from((lane + 16 * (TOKENS / 4)) & 63, __float_as_int(y[t][i])));
                        if (4 * quarter + i >= s.count) continue;
                        float *sum = sums + (int)(s.tokens >> (8 * i) & 15) * (16 * RG) + 16 * t + li;
                        *sum = __builtin_fmaf(s.share[i], v, *sum);
                    }
                    y[t] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            });
    };
    products(std::integral_constant<int, 4>{}, std::integral_constant<int, D>{}, few * stretches, [&](int i) { return list[i]; }, first);
    if constexpr (MOST > 4)  // (the waves that have done an item less go first)
        products(std::integral_constant<int, MOST>{}, std::integral_constant<int, 1>{}, more * stretches,
                 [&](int i) { return list[2 * kFfnChoices - 1 - i]; }, (first + step - few * stretches % step) % step);
    __syncthreads();
    const int outputs = a.B * 16 * RG;
    float *const part = a.part + (int64_t)blockIdx.x * a.splits * outputs;
    auto finish = [&](int i, float total) {
        const int b = i / (16 * RG), row = row0 + i % (16 * RG);
        if (row >= a.d) return;
        const int64_t out = (int64_t)b * a.d + row;
        if (a.residual) total += bf16_bits_to_float(a.x[out]);
        a.y[out] = (uint16_t)float_to_bf16_bits(total);
    };
    for (int i = threadIdx.x; i < outputs; i += (int)blockDim.x) {
        float total = 0.f;
        for (int w = 0; w < waves; ++w) total += *reinterpret_cast<const float *>(lds + Lds::LIST + w * Lds::WAVE + Lds::STREAM + i * 4);
        if (a.splits == 1)
            finish(i, total);
        else  // (past the caches that XCDs do not share)
            __hip_atomic_store(part + blockIdx.y * outputs + i, total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (a.splits == 1) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // each wave's sums are there before the workgroup is counted
    __syncthreads();
    if (threadIdx.x == 0) totals[2] = (int)__hip_atomic_fetch_add(a.arrived + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (totals[2] != a.splits - 1) return;
    for (int i = threadIdx.x; i < outputs; i += (int)blockDim.x) {
        float total = 0.f;
        for (int k = 0; k < a.splits; ++k) total += __hip_atomic_load(part + k * outputs + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        finish(i, total);
    }
}

namespace {

struct ExpertsFfnLayout {
    size_t act, rest, count, expert, token, row, share, part, arrived, total;
};

ExpertsFfnLayout experts_ffn_layout(int64_t n, int64_t F, int64_t d) {
    auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
    ExpertsFfnLayout l;
    l.act = 0;
    l.rest = up((size_t)n * F * 2);
    l.count = l.rest + up((size_t)n * F * 2);
    l.expert = l.count + up((size_t)n * 8);
    l.token = l.expert + up((size_t)n * 8);
    l.row = l.token + up((size_t)n * 16);
    l.share = l.row + up((size_t)n * 64);
    l.part = l.share + up((size_t)n * 64);
    l.arrived = l.part + up((size_t)std::min<int64_t>(n, kGroupedTokens) * d * 4 * kDownSplits);
    l.total = l.arrived + up((size_t)d / kGroupedRows * 4);
    return l;
}

template <int R, int C, int RG, int MOST, int D>
mq_status launch_gate_up_as(ExpertsFfnArgs a, hipStream_t st) {
    constexpr int LDS = Grouped<R, C, RG, MOST>::LDS;
    const int64_t stretches = cdiv(a.d, stretch_codes(R)), blocks = cdiv(2 * a.F, kGroupedRows * RG);
    // (waves as for the product alone: 24 for each compute unit)
    a.ks = (int)std::min<int64_t>({stretches, kGateUpWaves, 163840 / LDS, cdiv(24 * 256, blocks * std::min(a.n, a.E))});
    a.ks = (int)cdiv(stretches, cdiv(stretches, a.ks));
    const int lds = a.ks * LDS;
    constexpr auto kernel = experts_gate_up_kernel<R, C, RG, MOST, D>;
    if (lds > 65536 && !allow_lds<kernel>(lds)) return MQ_ERR_DEVICE;
    kernel<<<dim3((unsigned)blocks, a.n), dim3(64 * a.ks), lds, st>>>(a);
    return launch_status();
}
template <int R, int C, int RG, int MOST, int D>
mq_status launch_down_as(ExpertsFfnArgs a, hipStream_t st) {
    using Lds = DownLds<R, C, RG, MOST>;
    const int64_t items = cdiv(a.F, stretch_codes(R)) * std::min(a.n, a.E), blocks = cdiv(a.d, kGroupedRows * RG);
    a.splits = down_splits(R, a.d, a.F, std::min(a.n, a.E), RG);
    const int waves = (int)std::min<int64_t>({cdiv(items, a.splits), down_waves(R), (163840 - Lds::LIST) / Lds::WAVE});
    const int lds = Lds::LIST + waves * Lds::WAVE;
    constexpr auto kernel = experts_down_kernel<R, C, RG, MOST, D>;
    if (lds > 65536 && !allow_lds<kernel>(lds)) return MQ_ERR_DEVICE;
    kernel<<<dim3((unsigned)blocks, a.splits), dim3(64 * waves), lds, st>>>(a);
    return launch_status();
}
template <int R, int C, int MOST>
mq_status launch_gate_up(const ExpertsFfnArgs &a, hipStream_t st) {
    // A piece under way beside the one that is multiplied (one token x 2 of 8, 4096 x 14336: 47.2 us, without 49.7), but at two bits, which want
    // registers for more waves (5 tokens x 2 of 8, 2304 x 9216: 55.0, with it 58.3).
    constexpr int D = R == 2 ? 1 : 2;
    if (gate_up_tiles(a.F, std::min(a.n, a.E)) == 2) return launch_gate_up_as<R, C, 2, MOST, D>(a, st);
    return launch_gate_up_as<R, C, 1, MOST, D>(a, st);
}
template <int R, int C, int MOST>
mq_status launch_down(const ExpertsFfnArgs &a, hipStream_t st) {
    // A piece under way helps small layers (2 tokens x 4 of 64, 2048 x 768: 13.2 us, without 14.0), at two bits it makes no odds (16 tokens x 2 of 8,
    // 4096 x 14336: 155.8, without 153.9; 5 tokens x 2 of 8, 2304 x 9216: 53.6 and 55.2), groups of 32 at four bits leave no registers for it.
    constexpr int D = R == 2 || (R == 4 && C == 32) ? 1 : 2;
    if (down_tiles(R, a.d, a.F, std::min(a.n, a.E)) == 2) return launch_down_as<R, C, 2, MOST, D>(a, st);
    return launch_down_as<R, C, 1, MOST, D>(a, st);
}
template <int R, int C>
mq_status launch_half(const ExpertsFfnArgs &a, bool down, hipStream_t st) {
    if (a.B <= 4) return down ? launch_down<R, C, 4>(a, st) : launch_gate_up<R, C, 4>(a, st);
    return down ? launch_down<R, C, 8>(a, st) : a.B <= 8 ? launch_gate_up<R, C, 8>(a, st) : launch_gate_up<R, C, 16>(a, st);
}

}  // namespace

size_t experts_ffn_workspace_bytes(int64_t n, int64_t F, int64_t d) {
    if (n < 1 || n > kFfnChoices || F < 1 || F > (1 << 20) || d < 1 || d > (1 << 20)) return 0;
    return experts_ffn_layout(n, F, d).total + 256;
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
    const ExpertsFfnLayout l = experts_ffn_layout(B * top, F, d);
    if (!ws || !aligned16(ws) || ws_bytes < l.total + 256) return MQ_ERR_WORKSPACE;
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
    ExpertsFfnArgs a{x, ids, weight, layer->gate_up, layer->down, layer->alpha_gu, layer->zero_gu, layer->alpha_dn, layer->zero_dn, y,
                     reinterpret_cast<uint16_t *>(base + l.act), reinterpret_cast<uint16_t *>(base + l.rest), reinterpret_cast<int32_t *>(base + l.count),
                     reinterpret_cast<int32_t *>(base + l.expert), base + l.token, reinterpret_cast<int32_t *>(base + l.row),
                     reinterpret_cast<float *>(base + l.share), reinterpret_cast<float *>(base + l.part), reinterpret_cast<uint32_t *>(base + l.arrived),
                     (int)B, (int)top, (int)(B * top), (int)E, (int)d, (int)F, (int)(group ? d / group : 1), (int)(group ? F / group : 1), 1, 1, GroupOf{0, 0}, (flags & MQ_FLAG_FFN_SILU) != 0,
                     (flags & MQ_FLAG_FFN_RESIDUAL) != 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    for (int down = 0; down < 2; ++down) {
        const int64_t g = group ? group : down ? F : d;
        int c = chunk_codes(r, g);
        a.group = group_of(g / c);
#define MQ_EXPERTS_CASE(R_, C_) \
    if (r == R_ && c == C_) s = launch_half<R_, C_>(a, down, st);
        MQ_EXPERTS_CASE(4, 128) MQ_EXPERTS_CASE(4, 64) MQ_EXPERTS_CASE(4, 32)
        MQ_EXPERTS_CASE(2, 256) MQ_EXPERTS_CASE(2, 128) MQ_EXPERTS_CASE(2, 64)
        MQ_EXPERTS_CASE(8, 64) MQ_EXPERTS_CASE(8, 32)
#undef MQ_EXPERTS_CASE
        if (s != MQ_OK) return s;
    }
    return MQ_OK;
}
