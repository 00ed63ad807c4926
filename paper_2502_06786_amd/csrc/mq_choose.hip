// A router's choice of experts and its gradient.
#include "mq_common.h"

namespace mq {

struct ChooseArgs {
    const float *scores;  // [M, ld]
    int64_t ld;
    int32_t *ids;         // [M, top]
    float *weight;        // [M, top]
    int M, E, top, renormalize;
};

struct ChooseBwdArgs {
    const float *scores;
    int64_t ld;
    const int32_t *ids;
    const float *weight, *dweight;
    float *dscores;  // [M, E]
    int M, E, top, renormalize;
};

// Over the LPT neighbouring lanes of a token; every lane gets the result, in the same bits.
template <int LPT, typename Op>
__device__ __forceinline__ int token_reduce(int v, Op op) {
    // (all lanes of a row take part, so nothing stands in for one that does not: the move joins the operation that uses it)
    auto dpp = [](int x, auto ctrl) { return __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, 0xF, 0xF, true); };
    if constexpr (LPT >= 2) v = op(v, dpp(v, std::integral_constant<int, 0xB1>{}));   // the neighbour
    if constexpr (LPT >= 4) v = op(v, dpp(v, std::integral_constant<int, 0x4E>{}));   // the other pair
    if constexpr (LPT >= 8) v = op(v, dpp(v, std::integral_constant<int, 0x141>{}));  // the other four (half row mirrored)
    if constexpr (LPT >= 16) v = op(v, dpp(v, std::integral_constant<int, 0x140>{})); // the other eight (row mirrored)
    if constexpr (LPT >= 32) v = op(v, __shfl_xor(v, 16, 64));
    if constexpr (LPT >= 64) v = op(v, __shfl_xor(v, 32, 64));
    return v;
}
template <int LPT>
__device__ __forceinline__ int token_max(int v) {
    return token_reduce<LPT>(v, [](int a, int b) { return max(a, b); });
}
template <int LPT>
__device__ __forceinline__ int token_min(int v) {
    return token_reduce<LPT>(v, [](int a, int b) { return min(a, b); });
}
template <int LPT>
__device__ __forceinline__ float token_sum(float v) {
    return __int_as_float(token_reduce<LPT>(__float_as_int(v), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}

// Scores in whole numbers of the same order (zeros of both signs are one score), which compare without regard to NaN.
__device__ __forceinline__ int order_of(float v) {
    const int b = __float_as_int(v + 0.0f);
    return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float score_of(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7FFFFFFF)); }
constexpr int kNone = (int)0x807FFFFFu;  // of -inf

// Expert of value v of lane l of a token: neighbouring lanes hold neighbouring fours.  Ascending in v.
template <int LPT>
__device__ __forceinline__ int expert_of(int v, int l) {
    return v / 4 * (4 * LPT) + l * 4 + v % 4;
}

// A token's scores, -inf behind the last.  NaN counts as +inf: it is chosen first, and the softmax turns the token's weights into NaN.
template <int LPT, int V, int VEC>
__device__ __forceinline__ void load_scores(const float *row, int E, int l, float (&s)[V]) {
#pragma unroll
    for (int v = 0; v < V; v += VEC) {
        const int e = expert_of<LPT>(v, l);
        if constexpr (VEC == 4) {
            f32x4 d = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (e < E) d = *reinterpret_cast<const f32x4 *>(row + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[v + i] = d[i];
        } else {
            s[v] = e < E ? row[e] : -INFINITY;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = s[v] != s[v] ? INFINITY : s[v];
}

// how many of a token's choices a lane keeps: choice j is lane j % LPT's
template <int LPT, int V>
constexpr int kKept = LPT * V < 32 ? V : LPT < 32 ? 32 / LPT : 1;

// `top` times the largest score is taken: the largest over the token's lanes, then the lowest of the experts that have it.  Bound by the vector unit:
// about 90 instructions to a round of the eight tokens that a wave has at E = 128 (65531 x 128, 8 of them: 14.7 us, 2.6 TB/s; to take a score out by the
// comparison that found it, where a wave has no equal ones, costs as much as it saves: 16.3, with 15.8 for this in the same run).
// LPT lanes to a token, V values to a lane, VEC of them to a load.
template <int LPT, int V, int VEC>
__global__ __launch_bounds__(256) void choose_kernel(ChooseArgs a) {
    constexpr int KEPT = kKept<LPT, V>;
    const int l = threadIdx.x % LPT;
    const int64_t m = (int64_t)blockIdx.x * (256 / LPT) + threadIdx.x / LPT;
    if (m >= a.M) return;
    float s[V], total = 0.f;
    int o[V];
    load_scores<LPT, V, VEC>(a.scores + m * a.ld, a.E, l, s);
    int most = kNone;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        o[v] = order_of(s[v]);
        most = max(most, o[v]);
    }
    most = token_max<LPT>(most);
    const float base = most == kNone ? 0.f : score_of(most);  // (no expert at all)
    if (!a.renormalize) {
#pragma unroll
        for (int v = 0; v < V; ++v) total += expf(s[v] - base);
        total = token_sum<LPT>(total);
    }
    int id[KEPT], w[KEPT];
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
        id[k] = -1;
        w[k] = kNone;
        for (int j = 0; j < LPT && k * LPT + j < a.top; ++j) {
            int best = o[0];
#pragma unroll
            for (int v = 1; v < V; ++v) best = max(best, o[v]);
            best = token_max<LPT>(best);
            int which = V;
#pragma unroll
            for (int v = V - 1; v >= 0; --v) which = o[v] == best ? v : which;
            const int mine = which < V ? expert_of<LPT>(which, l) : 0x7FFFFFFF, e = token_min<LPT>(mine);
            which = mine == e ? which : V;
#pragma unroll
            for (int v = 0; v < V; ++v) o[v] = which == v ? kNone : o[v];
            if (l == j && best != kNone) {
                id[k] = e;
                w[k] = best;
            }
        }
    }
    float p[KEPT], sum = 0.f;
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
        p[k] = id[k] < 0 ? 0.f : expf(score_of(w[k]) - base);
        sum += p[k];
    }
    if (a.renormalize) total = token_sum<LPT>(sum);
#pragma unroll
    for (int k = 0; k < KEPT; ++k)
        if (k * LPT + l < a.top) {
            a.ids[m * a.top + k * LPT + l] = id[k];
            a.weight[m * a.top + k * LPT + l] = id[k] < 0 ? 0.f : p[k] / total;
        }
}

// A lane has the choices l, l + LPT, ... of its token; each goes round all its lanes, which add it to the expert it is of.  Bound by memory (65531 x 64, 6
// choices: 8.9 us, 4.3 TB/s).
template <int LPT, int V, int VEC>
__global__ __launch_bounds__(256) void choose_bwd_kernel(ChooseBwdArgs a) {
    constexpr int KEPT = kKept<LPT, V>;
    const int l = threadIdx.x % LPT;
    const int64_t m = (int64_t)blockIdx.x * (256 / LPT) + threadIdx.x / LPT;
    if (m >= a.M) return;
    int id[KEPT];
    float w[KEPT], g[KEPT];
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
        const int64_t at = m * a.top + k * LPT + l;
        const bool there = k * LPT + l < a.top;
        id[k] = there ? a.ids[at] : -1;
        w[k] = there ? a.weight[at] : 0.f;
        g[k] = there ? a.dweight[at] : 0.f;
    }
    float p[V], up[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = up[v] = 0.f;
    if (!a.renormalize) load_scores<LPT, V, VEC>(a.scores + m * a.ld, a.E, l, p);
    float mean = 0.f;
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
        if (id[k] < 0 || id[k] >= a.E) id[k] = -1, w[k] = g[k] = 0.f;  // (what stands beside no choice may be anything)
        mean = __builtin_fmaf(w[k], g[k], mean);
    }
    mean = token_sum<LPT>(mean);
    if (!a.renormalize) {
        int most = kNone;
        float total = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) most = max(most, order_of(p[v]));
        most = token_max<LPT>(most);
        const float base = most == kNone ? 0.f : score_of(most);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] = expf(p[v] - base);
            total += p[v];
        }
        total = token_sum<LPT>(total);
        // (one quotient for all experts: half a step of fp32 more than a quotient for each, which took 10.5 us instead of 9.6 for 65531 x 64)
        const float scale = total == 0.f ? 0.f : 1.0f / total;
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] *= scale;
    }
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
        const float mine = a.renormalize ? w[k] * (g[k] - mean) : g[k];
        for (int j = 0; j < LPT && k * LPT + j < a.top; ++j) {
            const int e = LPT == 1 ? id[k] : __shfl(id[k], j, LPT);
            const float d = LPT == 1 ? mine : __shfl(mine, j, LPT);
#pragma unroll
            for (int v = 0; v < V; ++v) up[v] += expert_of<LPT>(v, l) == e ? d : 0.f;
        }
    }
    float *out = a.dscores + m * a.E;
#pragma unroll
    for (int v = 0; v < V; v += VEC) {
        const int e = expert_of<LPT>(v, l);
        if (e >= a.E) continue;
        if constexpr (VEC == 4) {
            f32x4 d;
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = a.renormalize ? up[v + i] : p[v + i] * (up[v + i] - mean);
            *reinterpret_cast<f32x4 *>(out + e) = d;
        } else {
            out[e] = a.renormalize ? up[v] : p[v] * (up[v] - mean);
        }
    }
}

// f(lanes to a token, values to a lane, values to a load) for E experts; vec: rows are whole 16-byte pieces.  The choice takes as many steps
// between lanes whatever a lane holds, so fewer lanes with more values each are quicker, down to where a wave's registers are full; the gradient, which
// is bound by memory, wants short loops.  us with half as many lanes, with these, with twice as many, 8 choices out of the softmax over all:
//   choice     65536 x 64   11.9, 11.6, 25.1    65536 x 128   19.1, 18.1, 24.9    65536 x 256   29.9, 30.7, 45.6
//   gradient   65536 x 64   10.9, 10.4, 16.4    65536 x 128   17.1, 15.3, 16.5    65536 x 256   28.3, 27.7, 31.2
// Beyond, 32 lanes instead of 64 would be quicker for the choice: 30000 x 300 27.9 and 33.5, x 512 27.9 and 33.0, 20000 x 1024 34.6 and 37.6 (16 lanes with
// 32 values: 28.5 and 29.3 for the first two), for the gradient with up to 300 (20.7 and 22.1; x 512 26.4 and 25.6, x 1024 36.2 and 32.3).
template <bool CHOICE, typename F>
static void by_experts(int E, bool vec, F f) {
    auto with = [&](auto lanes, auto values) {
        return vec ? f(lanes, values, std::integral_constant<int, 4>{}) : f(lanes, values, std::integral_constant<int, 1>{});
    };
#define MQ_CHOOSE_CASE(L_, V_) \
    if (E <= L_ * V_) return with(std::integral_constant<int, L_>{}, std::integral_constant<int, V_>{});
    MQ_CHOOSE_CASE(1, 8) MQ_CHOOSE_CASE(4, 4) MQ_CHOOSE_CASE(8, 4)
    if constexpr (CHOICE) {
        MQ_CHOOSE_CASE(8, 8) MQ_CHOOSE_CASE(8, 16) MQ_CHOOSE_CASE(16, 16)
    } else {
        MQ_CHOOSE_CASE(16, 4) MQ_CHOOSE_CASE(16, 8) MQ_CHOOSE_CASE(32, 8)
    }
    MQ_CHOOSE_CASE(64, 8) MQ_CHOOSE_CASE(64, 16)
#undef MQ_CHOOSE_CASE
}

constexpr int kChooseExperts = 1024, kChooseTop = 32, kChooseTokens = 1 << 25;

static mq_status choose_check(const float *scores, int64_t M, int64_t E, int64_t ld, int64_t top, uint32_t flags) {
    if (flags & ~(uint32_t)MQ_FLAG_RENORMALIZE) return MQ_ERR_BITS;
    if (M < 0 || M > kChooseTokens || E < 1 || E > kChooseExperts || ld < E || top < 1 || top > kChooseTop || top > E) return MQ_ERR_SHAPE;
    if (M > 0 && ld > (int64_t)0x3FFFFFFFFFFFFFFF / 4 / M) return MQ_ERR_SHAPE;
    if (M > 0 && !scores) return MQ_ERR_NULL;
    return reinterpret_cast<uintptr_t>(scores) % 4 == 0 ? MQ_OK : MQ_ERR_ALIGN;
}

}  // namespace mq

extern "C" mq_status mq_experts_choose(const float *scores, int64_t M, int64_t E, int64_t ld, int64_t top, uint32_t flags, int32_t *ids,
                                       float *weight, void *hip_stream) {
    using namespace mq;
    const mq_status s = choose_check(scores, M, E, ld, top, flags);
    if (s != MQ_OK || M == 0) return s;
    if (!ids || !weight) return MQ_ERR_NULL;
    if (!aligned16(ids) || !aligned16(weight)) return MQ_ERR_ALIGN;
    const ChooseArgs a{scores, ld, ids, weight, (int)M, (int)E, (int)top, (flags & MQ_FLAG_RENORMALIZE) != 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    by_experts<true>((int)E, E % 4 == 0 && ld % 4 == 0 && aligned16(scores), [&](auto L, auto V, auto Vec) {
        constexpr int per = 256 / decltype(L)::value;
        choose_kernel<decltype(L)::value, decltype(V)::value, decltype(Vec)::value><<<dim3((unsigned)cdiv(M, per)), dim3(256), 0, st>>>(a);
    });
    return launch_status();
}

extern "C" mq_status mq_experts_choose_bwd(const float *scores, int64_t ld, const int32_t *ids, const float *weight, const float *dweight,
                                           int64_t M, int64_t E, int64_t top, uint32_t flags, float *dscores, void *hip_stream) {
    using namespace mq;
    const mq_status s = choose_check(scores, M, E, ld, top, flags);
    if (s != MQ_OK || M == 0) return s;
    if (!ids || !weight || !dweight || !dscores) return MQ_ERR_NULL;
    if (!aligned16(ids) || !aligned16(weight) || !aligned16(dweight) || !aligned16(dscores)) return MQ_ERR_ALIGN;
    const ChooseBwdArgs a{scores, ld, ids, weight, dweight, dscores, (int)M, (int)E, (int)top, (flags & MQ_FLAG_RENORMALIZE) != 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    by_experts<false>((int)E, E % 4 == 0 && ld % 4 == 0 && aligned16(scores), [&](auto L, auto V, auto Vec) {
        constexpr int per = 256 / decltype(L)::value;
        choose_bwd_kernel<decltype(L)::value, decltype(V)::value, decltype(Vec)::value><<<dim3((unsigned)cdiv(M, per)), dim3(256), 0, st>>>(a);
    });
    return launch_status();
}
