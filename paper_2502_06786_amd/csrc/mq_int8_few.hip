// The product in 8-bit integers for few tokens.
#include "mq_int8.h"

namespace mq {

// Workgroup = 16 places x 64 channels, 16 channels to a wave, operands straight from memory.  Rows of the matrix-core product are
// channels, columns places: lane (l16, g4) ends up with channels 4 g4 .. 4 g4 + 3 of place l16.
template <bool R8>
__global__ __launch_bounds__(256) void int8_block_kernel(Int8Args a, int tiles_n) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g4 = lane >> 4, l16 = lane & 15;
    const Block b = find_block(a, blockIdx.x / tiles_n, 16);
    if (b.count <= 0) return;
    const int n0 = blockIdx.x % tiles_n * 64 + wave * 16;
    if (n0 >= a.N) return;
    const int place = b.place + min(l16, b.count - 1), m = token_of(a, place);
    const uint8_t *wrow = a.codes + ((int64_t)b.expert * a.N + min(n0 + l16, a.N - 1)) * a.K;
    const int8_t *xrow = a.Xq + (int64_t)m * a.K;
    i32x4 acc = {0, 0, 0, 0};
    for (int k0 = 0; k0 < a.K; k0 += 64) {
        const int k = k0 + 16 * g4;
        i32x4 w = {0, 0, 0, 0}, x = {0, 0, 0, 0};
        if (k < a.K) {
            w = *reinterpret_cast<const i32x4 *>(wrow + k);
            x = *reinterpret_cast<const i32x4 *>(xrow + k);
        }
        acc = mfma_i8(signed_codes<R8>(w), x, acc);
    }
    if (l16 >= b.count) return;
    const float s = a.scale[m], sum = (float)a.sum[m];
    const float *alpha = a.alpha + (int64_t)b.expert * a.N, *zero = a.zero + (int64_t)b.expert * a.N;
    float y[4];
    f32x4 al, ze, ka, kb;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        al[e] = alpha[min(n0 + 4 * g4 + e, a.N - 1)];
        ze[e] = zero[min(n0 + 4 * g4 + e, a.N - 1)];
    }
    channel_factors(al, ze, a.mult, a.offset, ka, kb);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = int8_output(acc[e], sum, s, ka[e], kb[e]);
    const int n = n0 + 4 * g4;
    if (a.gate) {
        uint16_t *out = a.Y + (int64_t)place * (a.N / 2) + n / 2;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (n + 2 * e < a.N) out[e] = (uint16_t)float_to_bf16_bits(gated_value(y[2 * e], y[2 * e + 1], a.gate));
    } else {
        uint16_t *out = a.Y + (int64_t)place * a.N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) out[e] = (uint16_t)float_to_bf16_bits(y[e]);
    }
}

mq_status launch_int8_blocks(const Int8Args &a, hipStream_t st) {
    const int64_t tiles_n = cdiv(a.N, 64), blocks = block_bound(a.T, a.E, a.offsets != nullptr, 16) * tiles_n;
    if (blocks > 0x7FFFFFFF) return MQ_ERR_SHAPE;
    if (a.offset != 0.f)
        int8_block_kernel<true><<<dim3((unsigned)blocks), dim3(256), 0, st>>>(a, (int)tiles_n);
    else
        int8_block_kernel<false><<<dim3((unsigned)blocks), dim3(256), 0, st>>>(a, (int)tiles_n);
    return launch_status();
}

}  // namespace mq
