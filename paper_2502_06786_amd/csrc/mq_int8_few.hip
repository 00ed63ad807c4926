// The product in 8-bit integers for few tokens: bound by the codes' way out of memory.  Every code is used by one workgroup, so LDS would only
// add a stop on its way, and 16 channels to a workgroup give the most of them.
#include <algorithm>

#include "mq_int8.h"
#include "mq_linear.h"

namespace mq {

// Workgroup = up to 16 places x 16 channels of one expert; its NW waves take turns along K, 128 bytes of every row at a time, and add
// their sums (whole numbers) in LDS.  Operands go straight from memory to registers, DEEP turns ahead.  Rows of the matrix-core product are
// channels, columns places: lane (l16, g4) ends up with channels 4 g4 .. 4 g4 + 3 of place l16.
template <bool R8, int NW, int DEEP>
__global__ __launch_bounds__(64 * NW) void int8_few_kernel(Int8Args a, int tiles_n, int blocks) {
    __shared__ i32x4 part[NW][64];
    const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lid = xcd_contiguous_id(blockIdx.x, gridDim.x);   // (blocks of one expert follow each other: its codes are in that L2)
    const Block b = find_block(a, (int)(lid % (uint32_t)blocks), 16);
    if (b.count <= 0) return;
    const int n0 = (int)(lid / (uint32_t)blocks) * 16;

    const __amdgpu_buffer_rsrc_t rC = make_rsrc(a.codes + ((int64_t)b.expert * a.N + n0) * a.K, (uint64_t)(a.N - n0) * a.K);
    const int base = a.rows ? 0 : b.place;   // (gathered tokens lie within 2 GiB: quantize_and_multiply)
    const __amdgpu_buffer_rsrc_t rX = make_rsrc(a.Xq + (int64_t)base * a.ldq, (uint64_t)(a.M - base) * a.ldq);
    const int m = token_of(a, b.place + min(l16, b.count - 1));
    // (a lane takes 32 neighbouring bytes of a row, so that the four of a row take a line; both operands in that order)
    const uint32_t coff = (uint32_t)l16 * (uint32_t)a.K + 32u * g4, xoff = (uint32_t)(m - base) * (uint32_t)a.ldq + 32u * g4;
    i32x4 c[DEEP][2], x[DEEP][2];
    auto load = [&](int slot, int k0) {   // past the end of the rows: out of range, zeros
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + 16 * h;
            const bool in = k + 32 * g4 < a.K;
            c[slot][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rC, in ? coff + (uint32_t)k : kOOB, 0, 0));
            x[slot][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rX, in ? xoff + (uint32_t)k : kOOB, 0, 0));
        }
    };
    constexpr int TURN = 128 * NW;
    int k0 = wave * 128;
#pragma unroll
    for (int u = 0; u < DEEP; ++u) load(u, k0 + u * TURN);

    // what the outputs need, requested behind the first operands
    const int n = n0 + 4 * g4;
    float alpha[4], zero[4], scale = 0.f;
    int total = 0;
    if (wave == 0) {
        const int64_t first = (int64_t)b.expert * a.N;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            alpha[e] = a.alpha[first + min(n + e, a.N - 1)];
            zero[e] = a.zero[first + min(n + e, a.N - 1)];
        }
        scale = a.scale[m];
        total = a.sum[m];
    }
    i32x4 acc = {0, 0, 0, 0};
    for (; k0 < a.K; k0 += DEEP * TURN)
#pragma unroll
        for (int u = 0; u < DEEP; ++u) {
#pragma unroll
            for (int h = 0; h < 2; ++h) acc = mfma_i8(signed_codes<R8>(c[u][h]), x[u][h], acc);
            if (k0 + DEEP * TURN < a.K) load(u, k0 + (DEEP + u) * TURN);
        }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave > 0 || l16 >= b.count || n >= a.N) return;
    f32x4 ka, kb;
    channel_factors(f32x4{alpha[0], alpha[1], alpha[2], alpha[3]}, f32x4{zero[0], zero[1], zero[2], zero[3]}, a.mult, ka, kb);
#pragma unroll
    for (int w = 1; w < NW; ++w) acc += part[w][lane];
    store_four(a, b.place + l16, n, acc, scale, (float)total, ka, kb);
}

// The same on bf16 tokens, which every workgroup quantizes for itself into LDS while its first codes are on their way: up to
// kInt8SinglePlaces places in all.  Workgroup = 16 RB channels, NW waves.  Bound by latency (launch, first lines and the quantizer in turn take about
// 3.5 us), then by the codes: one token through 4096 x 4096 6.8 us (16.8 MB), 18432 x 2304 for each of two experts 21.8 us (85 MB).
template <bool R8, int NW, int RB, int DEEP>
__global__ __launch_bounds__(64 * NW) void int8_single_kernel(Int8Args a, const uint16_t *__restrict__ X, int tiles_n, int blocks) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];   // codes [count][K + 16]
    constexpr int V = kInt8SingleK / (8 * 64 * NW);
    __shared__ i32x4 part[NW][RB][64];
    __shared__ uint32_t tops[NW];
    __shared__ int32_t sums[kInt8SinglePlaces][NW];
    __shared__ float scales[kInt8SinglePlaces];
    const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lid = xcd_contiguous_id(blockIdx.x, gridDim.x);
    const Block b = find_block(a, (int)(lid % (uint32_t)blocks), 16);
    if (b.count <= 0) return;
    const int n0 = (int)(lid / (uint32_t)blocks) * 16 * RB;

    const __amdgpu_buffer_rsrc_t rC = make_rsrc(a.codes + ((int64_t)b.expert * a.N + n0) * a.K, (uint64_t)(a.N - n0) * a.K);
    const uint32_t coff = (uint32_t)l16 * (uint32_t)a.K + 32u * g4;
    i32x4 c[DEEP][RB][2];
    auto load = [&](int slot, int k0) {   // past the end of the rows: out of range, zeros
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + 16 * h;
                const bool in = k + 32 * g4 < a.K;
                c[slot][rb][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                               rC, in ? coff + (uint32_t)(16 * rb) * (uint32_t)a.K + (uint32_t)k : kOOB, 0, 0));
            }
    };
    constexpr int TURN = 128 * NW;
    int k0 = wave * 128;
#pragma unroll
    for (int u = 0; u < DEEP; ++u) load(u, k0 + u * TURN);

    // what the outputs need, requested behind the first codes
    const int n = n0 + 16 * wave + 4 * g4;
    float alpha[4], zero[4];
    if (wave < RB) {
        const int64_t first = (int64_t)b.expert * a.N;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            alpha[e] = a.alpha[first + min(n + e, a.N - 1)];
            zero[e] = a.zero[first + min(n + e, a.N - 1)];
        }
    }
    const int row_bytes = a.K + 16;
    for (int j = 0; j < b.count; ++j) {
        const u32x4 *src = reinterpret_cast<const u32x4 *>(X + (int64_t)token_of(a, b.place + j) * a.K);
        u32x4 v[V];
        uint32_t top2 = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[i] = u32x4{0u, 0u, 0u, 0u};
            if ((int)(threadIdx.x + i * 64 * NW) * 8 < a.K) v[i] = src[threadIdx.x + i * 64 * NW];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) top2 = top_of(top2, v[i]);
        uint32_t top = top_of_wave(top2);
        if (j > 0) __syncthreads();   // (tops of the token before have been read)
        if (lane == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) top = max(top, tops[w]);
        const TokenScale ts = token_scale(top);
        int total = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int chunk = threadIdx.x + i * 64 * NW;
            if (chunk * 8 >= a.K) break;
            *reinterpret_cast<u32x2 *>(smem + j * row_bytes + chunk * 8) = token_codes(v[i], ts, total);
        }
        total = sum_of_wave(total);
        if (lane == 0) sums[j][wave] = total;
        if (threadIdx.x == 0) scales[j] = ts.scale;
    }
    __syncthreads();

    i32x4 acc[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) acc[rb] = i32x4{0, 0, 0, 0};
    const int row = min(l16, b.count - 1);
    for (; k0 < a.K; k0 += DEEP * TURN)
#pragma unroll
        for (int u = 0; u < DEEP; ++u) {
            const int k = k0 + u * TURN + 32 * g4;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                i32x4 x = {0, 0, 0, 0};
                if (k + 16 * h < a.K) x = *reinterpret_cast<const i32x4 *>(smem + row * row_bytes + k + 16 * h);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) acc[rb] = mfma_i8(signed_codes<R8>(c[u][rb][h]), x, acc[rb]);
            }
            if (k0 + DEEP * TURN < a.K) load(u, k0 + (DEEP + u) * TURN);
        }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) part[wave][rb][lane] = acc[rb];
    __syncthreads();
    if (wave >= RB || l16 >= b.count || n >= a.N) return;
    f32x4 ka, kb;
    channel_factors(f32x4{alpha[0], alpha[1], alpha[2], alpha[3]}, f32x4{zero[0], zero[1], zero[2], zero[3]}, a.mult, ka, kb);
    i32x4 dot = {0, 0, 0, 0};
    int total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        dot += part[w][wave][lane];
        total += sums[l16][w];
    }
    store_four(a, b.place + l16, n, dot, scales[l16], (float)total, ka, kb);
}

namespace {

template <int NW, int DEEP>
mq_status launch_few(const Int8Args &a, hipStream_t st) {
    const int64_t tiles_n = cdiv(a.N, 16), grid_size = int8_grid(kInt8Few, a.T, a.N, a.offsets ? a.E : 0, 1), blocks = grid_size / tiles_n;
    const dim3 grid((unsigned)grid_size), threads(64 * NW);
    static_assert(NW <= 4, "");
    if (a.offset != 0.f)
        int8_few_kernel<true, NW, DEEP><<<grid, threads, 0, st>>>(a, (int)tiles_n, (int)blocks);
    else
        int8_few_kernel<false, NW, DEEP><<<grid, threads, 0, st>>>(a, (int)tiles_n, (int)blocks);
    return launch_status();
}

template <int NW, int RB, int DEEP>
mq_status launch_single(const Int8Args &a, const uint16_t *X, hipStream_t st) {
    const int64_t tiles_n = cdiv(a.N, 16 * RB), blocks = a.offsets ? std::min(a.T, a.E) : 1;   // (an expert has one block at most)
    const int lds = a.T * (a.K + 16);
    const dim3 grid((unsigned)(tiles_n * blocks));
    if (!(a.offset != 0.f ? allow_lds<int8_single_kernel<true, NW, RB, DEEP>>(lds) : allow_lds<int8_single_kernel<false, NW, RB, DEEP>>(lds))) return MQ_ERR_DEVICE;
    if (a.offset != 0.f)
        int8_single_kernel<true, NW, RB, DEEP><<<grid, dim3(64 * NW), lds, st>>>(a, X, (int)tiles_n, (int)blocks);
    else
        int8_single_kernel<false, NW, RB, DEEP><<<grid, dim3(64 * NW), lds, st>>>(a, X, (int)tiles_n, (int)blocks);
    return launch_status();
}

}  // namespace

// Eight waves to 16 channels: with a workgroup or two to a compute unit four would not have enough codes on their way (4096 x 4096 7.8 -> 6.8 us,
// 4096 x 14336 16.8 -> 15.9, 2304 x 9216 11.2 -> 10.5).  Four turns ahead where the rows are long enough and two workgroups fit a compute unit
// (8192 x 8192 15.6 us, with two turns 16.7); with more workgroups the registers of two let three of them in (10028 x 2320 9.5 us, with four turns
// 12.0).  With 32 channels there are several (28672 x 4096 26.4 us, with eight waves 28.2).
mq_status launch_int8_single(const Int8Args &a, const uint16_t *X, hipStream_t st) {
    const int64_t E = a.offsets ? a.E : 0, tiles = cdiv(a.N, 16) * (E == 0 ? 1 : std::min(a.T, a.E));
    if (int8_single_wide(a.T, a.N, E)) return launch_single<4, 2, 2>(a, X, st);
    return tiles <= 512 && a.K > 2048 ? launch_single<8, 1, 4>(a, X, st) : launch_single<8, 1, 2>(a, X, st);
}

mq_status launch_int8_few(const Int8Args &a, hipStream_t st) { return launch_few<4, 8>(a, st); }

}  // namespace mq
