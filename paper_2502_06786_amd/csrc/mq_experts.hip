// Around the products by expert: the router's choices grouped by expert, and the weighted sum of the experts' outputs.
#include "mq_int8.h"

namespace mq {

// ============================================================================================
// grouping
// ============================================================================================
// A stable counting sort with E + 1 buckets, the last one for choices of no expert.  A workgroup takes kRouteChunk choices, a wave 64 of them
// at a time.  Lanes with the same bucket find each other by comparing a bit of the bucket at a time; the first of them leaves their
// number in count[64 choices][bucket], and sums over the earlier counts give every choice its place: no atomics, one order.  Bound by the steps
// that follow each other: 3.6 us for the two choices of a token, 8.2 us for 3330 of 64, 14 us in two launches for 8198 of 8.  Every workgroup adds up
// the counts of all chunks, which grows with their square but stays small for long: 262144 choices of 64 31 us, 1048576 76 us, 4194304 420 us.
constexpr int kRouteThreads = 1024, kRouteSteps = 4, kRouteChunk = kRouteThreads * kRouteSteps;

struct RouteArgs {
    const int32_t *ids;   // [n]
    int32_t *offsets, *rows, *place;
    int32_t *chunk_counts;  // [chunks][E + 1]
    int n, top, E, chunks;
};

// PLACES false: only the counts of the chunk, into chunk_counts (launches of more than one chunk need them first).
template <bool PLACES>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int buckets = a.E + 1, padded = (buckets + 1) & ~1;
    constexpr int GROUPS = kRouteChunk / 64;
    uint16_t *count = reinterpret_cast<uint16_t *>(smem);                        // [GROUPS][padded]
    int32_t *base = reinterpret_cast<int32_t *>(smem + GROUPS * padded * 2);     // [padded] first place of this chunk's choices
    int32_t *total = base + padded;                                              // [padded]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * kRouteChunk;

    const int groups = min(GROUPS, (a.n - first + 63) / 64);   // that there are choices for
    for (int i = threadIdx.x; i < (groups * padded + 1) / 2; i += kRouteThreads) reinterpret_cast<uint32_t *>(smem)[i] = 0;
    __syncthreads();
    int bucket[kRouteSteps], rank[kRouteSteps];
#pragma unroll
    for (int s = 0; s < kRouteSteps; ++s) {
        const int i = first + s * kRouteThreads + (int)threadIdx.x;
        bucket[s] = -1;   // past the end: a bucket of its own that nobody counts
        if (i < a.n) {
            const int id = a.ids[i];
            bucket[s] = id >= 0 && id < a.E ? id : a.E;
        }
    }
#pragma unroll
    for (int s = 0; s < kRouteSteps; ++s) {
        uint64_t same = __ballot(bucket[s] >= 0);
        for (int bit = 0; (1 << bit) < buckets; ++bit) {
            const bool set = bucket[s] >> bit & 1;
            const uint64_t with = __ballot(set);
            same &= set ? with : ~with;
        }
        rank[s] = __popcll(same & ((1ull << lane) - 1));
        if (bucket[s] >= 0 && rank[s] == 0) count[(s * (kRouteThreads / 64) + wave) * padded + bucket[s]] = (uint16_t)__popcll(same);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < buckets; b += kRouteThreads) {
        int sum = 0;
        for (int g0 = 0; g0 < groups; g0 += 8) {   // eight counts on their way at a time
            int c[8];
#pragma unroll
            for (int g = 0; g < 8; ++g) c[g] = g0 + g < groups ? count[(g0 + g) * padded + b] : 0;
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                if (g0 + g < groups) count[(g0 + g) * padded + b] = (uint16_t)sum;
                sum += c[g];
            }
        }
        if constexpr (PLACES) {
            int before = 0, all = sum;
            if (a.chunks > 1) {
                all = 0;
                for (int c = 0; c < a.chunks; ++c) {
                    const int v = a.chunk_counts[(int64_t)c * buckets + b];
                    before += c < (int)blockIdx.x ? v : 0;
                    all += v;
                }
            }
            base[b] = before;
            total[b] = all;
        } else {
            a.chunk_counts[(int64_t)blockIdx.x * buckets + b] = sum;
        }
    }
    if constexpr (PLACES) {
        __syncthreads();
        if (wave == 0) {  // prefix sums of the totals, 64 buckets at a time
            int carry = 0;
            for (int b0 = 0; b0 < buckets; b0 += 64) {
                const int b = b0 + lane, mine = b < buckets ? total[b] : 0;
                int upto = mine;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int v = __shfl_up(upto, o, 64);
                    if (lane >= o) upto += v;
                }
                if (b < buckets) {
                    base[b] += carry + upto - mine;
                    if (blockIdx.x == 0) a.offsets[b] = carry + upto - mine;
                }
                carry += __shfl(upto, 63, 64);
            }
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kRouteSteps; ++s) {
            if (bucket[s] < 0) continue;
            const int i = first + s * kRouteThreads + (int)threadIdx.x;
            const int p = base[bucket[s]] + count[(s * (kRouteThreads / 64) + wave) * padded + bucket[s]] + rank[s];
            a.rows[p] = bucket[s] < a.E ? i / a.top : -1;
            a.place[i] = bucket[s] < a.E ? p : -1;
        }
    }
}

// ============================================================================================
// weighted sum
// ============================================================================================
struct CombineArgs {
    const uint16_t *Y;
    const int32_t *place;
    const float *weight;
    uint16_t *out;
    uint32_t N;
    int top, T;
};

// Bound by memory: 4099 tokens of 4096 outputs, two rows each, 18 us (5.6 TB/s).
// Workgroup = up to 128 chunks of one token's row: the places and weights are the same for all its lanes.  V: values per thread, 8 where rows
// are whole 16-byte chunks, otherwise 1.
template <int V>
__global__ __launch_bounds__(128) void combine_kernel(CombineArgs a, uint32_t parts) {
    const uint32_t m = blockIdx.x / parts, n = ((blockIdx.x - m * parts) * 128 + threadIdx.x) * V;
    if (n >= a.N) return;
    const int32_t *place = a.place + (int64_t)m * a.top;
    const float *weight = a.weight + (int64_t)m * a.top;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.f;
    for (int j0 = 0; j0 < a.top; j0 += 4) {   // four rows on their way at a time
        int p[4];
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p[j] = j0 + j < a.top ? place[j0 + j] : -1;
            w[j] = j0 + j < a.top ? weight[j0 + j] : 0.f;
        }
        u32x4 d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            d[j] = u32x4{0u, 0u, 0u, 0u};
            if (p[j] < 0 || p[j] >= a.T) continue;
            const uint16_t *y = a.Y + (int64_t)p[j] * a.N + n;
            if constexpr (V == 8)
                d[j] = *reinterpret_cast<const u32x4 *>(y);
            else
                d[j][0] = *y;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (p[j] < 0 || p[j] >= a.T) continue;   // (its weight may be anything)
            if constexpr (V == 8) {
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    sum[2 * v] = __builtin_fmaf(w[j], bf16_lo(d[j][v]), sum[2 * v]);
                    sum[2 * v + 1] = __builtin_fmaf(w[j], bf16_hi(d[j][v]), sum[2 * v + 1]);
                }
            } else {
                sum[0] = __builtin_fmaf(w[j], bf16_bits_to_float(d[j][0]), sum[0]);
            }
        }
    }
    uint16_t *out = a.out + (int64_t)m * a.N + n;
    if constexpr (V == 8)
        *reinterpret_cast<u32x4 *>(out) = u32x4{pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3]), pack_bf16x2(sum[4], sum[5]),
                                                pack_bf16x2(sum[6], sum[7])};
    else
        *out = (uint16_t)float_to_bf16_bits(sum[0]);
}

namespace {

int route_lds(int64_t E) {
    const int padded = (int)((E + 2) & ~(int64_t)1);
    return kRouteChunk / 64 * padded * 2 + 2 * padded * 4;
}

template <bool PLACES>
mq_status launch_route(const RouteArgs &a, hipStream_t st) {
    const int lds = route_lds(a.E);
    if (!allow_lds<route_kernel<PLACES>>(lds)) return MQ_ERR_DEVICE;
    route_kernel<PLACES><<<dim3((unsigned)a.chunks), dim3(kRouteThreads), lds, st>>>(a);
    return launch_status();
}

}  // namespace

size_t route_workspace_bytes(int64_t n, int64_t E) {
    if (E < 1 || E > kMaxExperts || n < 0 || n > 0x7FFFFF00) return 0;
    return (size_t)cdiv(n, kRouteChunk) * (size_t)(E + 1) * 4 + 256;
}

}  // namespace mq

extern "C" mq_status mq_experts_route(const int32_t *ids, int64_t M, int64_t top, int64_t E, int32_t *offsets, int32_t *rows, int32_t *place,
                                      void *ws, size_t ws_bytes, void *hip_stream) {
    using namespace mq;
    if (M < 0 || top < 1 || E < 1 || E > kMaxExperts || top > kMaxExperts || M > 0x7FFFFF00 / top) return MQ_ERR_SHAPE;
    if (!offsets || (M > 0 && (!ids || !rows || !place))) return MQ_ERR_NULL;
    if (!aligned16(ids) || !aligned16(offsets) || !aligned16(rows) || !aligned16(place)) return MQ_ERR_ALIGN;
    RouteArgs a{ids, offsets, rows, place, nullptr, (int)(M * top), (int)top, (int)E, (int)(M == 0 ? 1 : cdiv(M * top, kRouteChunk))};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (a.chunks > 1) {
        if (!ws || !aligned16(ws) || ws_bytes < route_workspace_bytes(a.n, E)) return MQ_ERR_WORKSPACE;
        a.chunk_counts = reinterpret_cast<int32_t *>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
        const mq_status s = launch_route<false>(a, st);
        if (s != MQ_OK) return s;
    }
    return launch_route<true>(a, st);
}

extern "C" mq_status mq_experts_combine(const uint16_t *Y, const int32_t *place, const float *weight, int64_t T, int64_t M, int64_t top,
                                        int64_t N, uint16_t *out, void *hip_stream) {
    using namespace mq;
    if (M < 0 || N < 0 || T < 0 || top < 1 || top > kMaxExperts || M > 0x7FFFFF00 || N > 0x7FFFFF00 || T > 0x7FFFFF00) return MQ_ERR_SHAPE;
    if (M == 0 || N == 0) return MQ_OK;
    if ((T > 0 && !Y) || !place || !weight || !out) return MQ_ERR_NULL;
    if (!aligned16(Y) || !aligned16(place) || !aligned16(weight) || !aligned16(out)) return MQ_ERR_ALIGN;
    const CombineArgs a{Y, place, weight, out, (uint32_t)N, (int)top, (int)T};
    const int V = N % 8 == 0 ? 8 : 1;
    const int64_t parts = cdiv(N / V, 128), blocks = M * parts;
    if (blocks > 0x1FFFFFF) return MQ_ERR_SHAPE;   // (a launch has less than 2^32 threads)
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (V == 8)
        combine_kernel<8><<<dim3((unsigned)blocks), dim3(128), 0, st>>>(a, (uint32_t)parts);
    else
        combine_kernel<1><<<dim3((unsigned)blocks), dim3(128), 0, st>>>(a, (uint32_t)parts);
    return launch_status();
}
