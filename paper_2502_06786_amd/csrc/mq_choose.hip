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
    auto dpp = [](int x, auto ctrl) { return __builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xF, 0xF, false); };
    if constexpr (LPT >= 2) v = op(v, dpp(v, std::integral_constant<int, 0xB1>{}));   // the neighbour
    if constexpr (LPT >= 4) v = op(v, dpp(v, std::integral_constant<int, 0x4E>{}));   // the other pair
    if constexpr (LPT >= 8) v = op(v, dpp(v, std::integral_constant<int, 0x141>{}));  // the other four (half row mirrored)
    if constexpr (LPT >= 16) v = op(v, dpp(v, std::integral_constant<int, 0x140>{})); // the other eight (row mirrored)
    if constexpr (LPT >= 32) v = op(v, __shfl_xor(v, 16, 64));
    if constexpr (LPT >= 64) v = op(v, __shfl_xor(v, 32, 64));
    return v;
}
template <int LPT>
__device__ __forceinline__ float token_max(float v) {
    return __int_as_float(token_reduce<LPT>(__float_as_int(v), [](int a, int b) { return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b))); }));
}
template <int LPT>
__device__ __forceinline__ float token_sum(float v) {
    return __int_as_float(token_reduce<LPT>(__float_as_int(v), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}
template <int LPT>
__device__ __forceinline__ int token_min(int v) {
    return token_reduce<LPT>(v, [](int a, int b) { return min(a, b); });
}

// A token's scores: expert v LPT + l in value v of its lane l; -inf behind the last.  NaN counts as +inf: it is chosen first, and the
// softmax turns the token's weights into NaN.
template <int LPT, int V>
__device__ __forceinline__ void load_scores(const float *row, int E, int l, float (&s)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = v * LPT + l < E ? row[v * LPT + l] : -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = s[v] != s[v] ? INFINITY : s[v];
}

// The largest score is taken `top` times: the largest value over the token's lanes, then the lowest of the experts that have it.
// LPT lanes to a token, V values to a lane.  A lane keeps the choices l, l + LPT, ... and writes them at the end.
template <int LPT, int V>
__global__ __launch_bounds__(256) void choose_kernel(ChooseArgs a) {
    constexpr int KEPT = (LPT * V < 32 ? LPT * V : 32) / LPT > 0 ? (LPT * V < 32 ? LPT * V : 32) / LPT : 1;
    const int l = threadIdx.x % LPT;
    const int64_t m = (int64_t)blockIdx.x * (256 / LPT) + threadIdx.x / LPT;
    if (m >= a.M) return;
    float s[V], total = 0.f;
    load_scores<LPT, V>(a.scores + m * a.ld, a.E, l, s);
    float most = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) most = fmaxf(most, s[v]);
    most = token_max<LPT>(most);
    const float base = most == -INFINITY ? 0.f : most;  // (no expert at all)
    if (!a.renormalize) {
#pragma unroll
        for (int v = 0; v < V; ++v) total += expf(s[v] - base);
        total = token_sum<LPT>(total);
    }
    int id[KEPT];
    float w[KEPT];
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
        id[k] = -1;
        w[k] = 0.f;
        for (int j = 0; j < LPT && k * LPT + j < a.top; ++j) {
            float best = s[0];
#pragma unroll
            for (int v = 1; v < V; ++v) best = fmaxf(best, s[v]);
            best = token_max<LPT>(best);
            int e = 0x7FFFFFFF;
#pragma unroll
            for (int v = V - 1; v >= 0; --v) e = s[v] == best ? v * LPT + l : e;
            e = token_min<LPT>(e);
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] = v * LPT + l == e ? -INFINITY : s[v];
            const float p = expf(best - base);
            if (a.renormalize && best != -INFINITY) total += p;
            if (l == j && best != -INFINITY) {
                id[k] = e;
                w[k] = p;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < KEPT; ++k)
        if (k * LPT + l < a.top) {
            a.ids[m * a.top + k * LPT + l] = id[k];
            a.weight[m * a.top + k * LPT + l] = id[k] < 0 ? 0.f : w[k] / total;
        }
}

template <int LPT, int V>
__global__ __launch_bounds__(256) void choose_bwd_kernel(ChooseBwdArgs a) {
    const int l = threadIdx.x % LPT;
    const int64_t m = (int64_t)blockIdx.x * (256 / LPT) + threadIdx.x / LPT;
    if (m >= a.M) return;
    const int32_t *ids = a.ids + m * a.top;
    const float *weight = a.weight + m * a.top, *dweight = a.dweight + m * a.top;
    float p[V], up[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = up[v] = 0.f;
    if (!a.renormalize) {
        load_scores<LPT, V>(a.scores + m * a.ld, a.E, l, p);
        float most = -INFINITY, total = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) most = fmaxf(most, p[v]);
        most = token_max<LPT>(most);
        const float base = most == -INFINITY ? 0.f : most;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] = expf(p[v] - base);
            total += p[v];
        }
        total = token_sum<LPT>(total);
        const float scale = total == 0.f ? 0.f : 1.0f / total;
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] *= scale;
    }
    float mean = 0.f;
    for (int j = 0; j < a.top; ++j) {
        const int e = ids[j];
        if (e >= 0 && e < a.E) mean = __builtin_fmaf(weight[j], dweight[j], mean);
    }
    for (int j = 0; j < a.top; ++j) {
        const int e = ids[j];
        if (e < 0 || e >= a.E) continue;
        const float g = a.renormalize ? weight[j] * (dweight[j] - mean) : dweight[j];
#pragma unroll
        for (int v = 0; v < V; ++v) up[v] += v * LPT + l == e ? g : 0.f;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v * LPT + l < a.E) a.dscores[m * a.E + v * LPT + l] = a.renormalize ? up[v] : p[v] * (up[v] - mean);
}

// f(lanes to a token, values to a lane) for E experts
template <typename F>
static void by_experts(int E, F f) {
#define MQ_CHOOSE_CASE(L_, V_) \
    if (E <= L_ * V_) return f(std::integral_constant<int, L_>{}, std::integral_constant<int, V_>{});
    MQ_CHOOSE_CASE(1, 8) MQ_CHOOSE_CASE(4, 4) MQ_CHOOSE_CASE(8, 4) MQ_CHOOSE_CASE(16, 4) MQ_CHOOSE_CASE(16, 8)
    MQ_CHOOSE_CASE(32, 8) MQ_CHOOSE_CASE(64, 8) MQ_CHOOSE_CASE(64, 16)
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
    by_experts((int)E, [&](auto L, auto V) {
        constexpr int per = 256 / decltype(L)::value;
        choose_kernel<decltype(L)::value, decltype(V)::value><<<dim3((unsigned)cdiv(M, per)), dim3(256), 0, st>>>(a);
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
    by_experts((int)E, [&](auto L, auto V) {
        constexpr int per = 256 / decltype(L)::value;
        choose_bwd_kernel<decltype(L)::value, decltype(V)::value><<<dim3((unsigned)cdiv(M, per)), dim3(256), 0, st>>>(a);
    });
    return launch_status();
}
