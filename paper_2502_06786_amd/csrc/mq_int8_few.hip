// The product in 8-bit integers for few tokens: bound by the codes' way out of memory.
#include <type_traits>

#include "mq_int8.h"
#include "mq_linear.h"

namespace mq {

// Workgroup = up to 16 TB places x 16 RB channels of one expert; its NW waves take turns along K, 128 bytes of every row at a time, and
// add their sums (whole numbers) in LDS.  Operands go straight from memory to registers, U turns at once.  Rows of the matrix-core product
// are channels, columns places: lane (l16, g4) ends up with channels 4 g4 .. 4 g4 + 3 of place l16.
template <bool R8, int RB, int TB, int NW, int U>
__global__ __launch_bounds__(64 * NW) void int8_few_kernel(Int8Args a, int tiles_n, int blocks) {
    __shared__ i32x4 part[NW][RB * TB][64];
    const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lid = xcd_contiguous_id(blockIdx.x, gridDim.x);   // (blocks of one expert follow each other: its codes are in that L2)
    const Block b = find_block(a, (int)(lid % (uint32_t)blocks), 16 * TB);
    if (b.count <= 0) return;
    const int n0 = (int)(lid / (uint32_t)blocks) * 16 * RB;

    const __amdgpu_buffer_rsrc_t rC = make_rsrc(a.codes + ((int64_t)b.expert * a.N + n0) * a.K, (uint64_t)(a.N - n0) * a.K);
    const int64_t base = a.rows ? 0 : b.place;   // (gathered tokens lie within 2 GiB)
    const __amdgpu_buffer_rsrc_t rX = make_rsrc(a.Xq + base * a.K, (uint64_t)(a.M - base) * a.K);
    // (a lane takes 32 neighbouring bytes of a row, so that the four of a row take a line; both operands in that order)
    const uint32_t coff = (uint32_t)l16 * (uint32_t)a.K + 32u * g4;
    uint32_t xoff[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb)
        xoff[tb] = (uint32_t)(token_of(a, b.place + min(16 * tb + l16, b.count - 1)) - (int)base) * (uint32_t)a.K + 32u * g4;

    i32x4 acc[RB][TB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = i32x4{0, 0, 0, 0};
    auto turns = [&](auto inside_tag, int k0) {   // U turns from k0 on
        constexpr bool INSIDE = decltype(inside_tag)::value;
        i32x4 c[U][RB][2], x[U][TB][2];
        auto load = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off, int k, int half) {
            // past the end of the rows: out of range, zeros
            if constexpr (INSIDE) return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 16u * half, k, 0));
            const bool in = k + 32 * g4 + 16 * half < a.K;
            return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, in ? off + (uint32_t)k + 16u * half : kOOB, 0, 0));
        };
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int h = 0; h < 2; ++h) c[u][rb][h] = load(rC, coff + (uint32_t)(16 * rb) * (uint32_t)a.K, k0 + u * 128 * NW, h);
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                for (int h = 0; h < 2; ++h) x[u][tb][h] = load(rX, xoff[tb], k0 + u * 128 * NW, h);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const i32x4 w = signed_codes<R8>(c[u][rb][h]);
#pragma unroll
                    for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = mfma_i8(w, x[u][tb][h], acc[rb][tb]);
                }
    };
    int k0 = wave * 128;
    for (; k0 + (U - 1) * 128 * NW + 128 <= a.K; k0 += U * 128 * NW) turns(std::true_type{}, k0);
    if (k0 < a.K) turns(std::false_type{}, k0);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) part[wave][rb * TB + tb][lane] = acc[rb][tb];
    __syncthreads();

    for (int block = wave; block < RB * TB; block += NW) {
        const int rb = block / TB, tb = block % TB, row = 16 * tb + l16, n = n0 + 16 * rb + 4 * g4;
        if (row >= b.count || n >= a.N) continue;
        const int m = token_of(a, b.place + row);
        const float scale = a.scale[m], sum = (float)a.sum[m];
        const float *alpha = a.alpha + (int64_t)b.expert * a.N, *zero = a.zero + (int64_t)b.expert * a.N;
        f32x4 al, ze, ka, kb;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            al[e] = alpha[min(n + e, a.N - 1)];
            ze[e] = zero[min(n + e, a.N - 1)];
        }
        channel_factors(al, ze, a.mult, a.offset, ka, kb);
        i32x4 dot = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < NW; ++w) dot += part[w][block][lane];
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = int8_output(dot[e], sum, scale, ka[e], kb[e]);
        if (a.gate) {
            uint16_t *out = a.Y + (int64_t)(b.place + row) * (a.N / 2) + n / 2;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (n + 2 * e < a.N) out[e] = (uint16_t)float_to_bf16_bits(gated_value(y[2 * e], y[2 * e + 1], a.gate));
        } else {
            uint16_t *out = a.Y + (int64_t)(b.place + row) * a.N + n;
            if (a.N % 4 == 0) {
                *reinterpret_cast<u32x2 *>(out) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < a.N) out[e] = (uint16_t)float_to_bf16_bits(y[e]);
            }
        }
    }
}

namespace {

template <bool R8, int RB, int TB, int NW, int U>
mq_status launch_few(const Int8Args &a, hipStream_t st) {
    const int64_t tiles_n = cdiv(a.N, 16 * RB), blocks = block_bound(a.T, a.E, a.offsets != nullptr, 16 * TB);
    if (tiles_n * blocks > 0x7FFFFF00) return MQ_ERR_SHAPE;
    int8_few_kernel<R8, RB, TB, NW, U><<<dim3((unsigned)(tiles_n * blocks)), dim3(64 * NW), 0, st>>>(a, (int)tiles_n, (int)blocks);
    return launch_status();
}

}  // namespace

mq_status launch_int8_few(const Int8Args &a, hipStream_t st) {
    return a.offset != 0.f ? launch_few<true, 1, 1, 8, 4>(a, st) : launch_few<false, 1, 1, 8, 4>(a, st);
}

}  // namespace mq
