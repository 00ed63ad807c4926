// The layer in 8-bit integers: tokens quantized to int8 with a scale each, times the codes of the weights as they are stored, on the
// matrix core's 8-bit product (twice the rate of the bf16 one, and nothing is converted).  Quantizer of tokens, entry points.
#include <algorithm>

#include "mq_int8.h"

namespace mq {

// ============================================================================================
// quantizer of tokens
// ============================================================================================
// scale = top / 127, code = the whole number nearest to x 127 / top (ties to even).  One read of the row into registers, so 2 bytes read and 1
// written per value, which bounds it: 8192 x 14336 64 us (5.5 TB/s; the codes fit the last-level cache), 8192 x 4096 21.7 us (4.6 TB/s); a single
// row 2.3 us, the launch.  TPR threads to a row, V chunks of 8 values in each.
// rows: null, or the row of X that row m of the result is made of (rows are data: whatever they hold, they stay below X_rows).
template <int TPR, int V, int BLOCK>
__global__ __launch_bounds__(BLOCK) void quantize_tokens_kernel(const uint16_t *__restrict__ X, int64_t M, int K, int64_t ldx,
                                                                const int32_t *__restrict__ rows, int X_rows, int8_t *__restrict__ Xq, int64_t ldq,
                                                                float *__restrict__ scale, int32_t *__restrict__ sum) {
    constexpr int WAVES = TPR / 64;  // to a row
    __shared__ uint32_t tops[BLOCK / 64];
    __shared__ int32_t sums[BLOCK / 64];
    const int t = threadIdx.x % TPR, wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
    const int64_t m = (int64_t)blockIdx.x * (BLOCK / TPR) + threadIdx.x / TPR;
    const bool live = m < M;
    int64_t from = live ? m : 0;
    if (rows) from = min(max(rows[from], 0), X_rows - 1);
    const u32x4 *src = reinterpret_cast<const u32x4 *>(X + from * ldx);
    u32x4 v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i] = u32x4{0u, 0u, 0u, 0u};
        const int c = t + i * TPR;
        if (live && c * 8 < K) v[i] = src[c];
    }
    uint32_t top2 = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) top2 = top_of(top2, v[i]);
    uint32_t top = top_of_wave(top2);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = max(top, tops[first + w]);
    }
    const TokenScale ts = token_scale(top);
    int total = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = t + i * TPR;
        const u32x2 codes = token_codes(v[i], ts, total);
        if (live && c * 8 < K) *reinterpret_cast<u32x2 *>(Xq + m * ldq + c * 8) = codes;
    }
    total = sum_of_wave(total);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) sums[wave] = total;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) total += sums[first + w];
    }
    if (live && t == 0) {
        scale[m] = ts.scale;
        sum[m] = total;
    }
}

namespace {

template <int TPR, int V, int BLOCK>
mq_status launch_tokens(const uint16_t *X, int64_t M, int64_t K, int64_t ldx, const int32_t *rows, int64_t X_rows, int8_t *Xq, int64_t ldq, float *scale,
                        int32_t *sum, hipStream_t st) {
    // (a launch has less than 2^32 threads)
    constexpr int64_t most = 0xFFFFFFFFll / BLOCK * (BLOCK / TPR);
    for (int64_t m = 0; m < M; m += most) {
        const int64_t n = std::min(M - m, most);
        quantize_tokens_kernel<TPR, V, BLOCK><<<dim3((unsigned)cdiv(n, BLOCK / TPR)), dim3(BLOCK), 0, st>>>(
            rows ? X : X + m * ldx, n, (int)K, ldx, rows ? rows + m : nullptr, (int)X_rows, Xq + m * ldq, ldq, scale + m, sum + m);
    }
    return launch_status();
}

// ---- workspace: the quantized tokens, then the partial sums of ranges of K, if there are any ---------------------------
struct Int8Layout {
    size_t codes, scale, sum, part;
};
Int8Layout int8_layout(int64_t M, int64_t K) {
    Int8Layout l;
    size_t off = 0;
    l.codes = off, off += align256((size_t)M * (cdiv(K, kInt8Line) * kInt8Line));
    l.scale = off, off += align256((size_t)M * 4);
    l.sum = off, off += align256((size_t)M * 4);
    l.part = off;
    return l;
}
Int8Plan int8_plan(int64_t T, int64_t N, int64_t K, int64_t E, size_t part_bytes) {
    return remembered<Int8Plan>(make_int8_plan, T, N, K, E, (int64_t)std::min(part_bytes, (size_t)kInt8PartBytes));
}

// `part`: room for the partial sums of the plan's ranges, 256-byte aligned
mq_status launch_int8(const Int8Args &a, const Int8Plan &plan, void *part, hipStream_t st) {
    switch (plan.form) {
        case kInt8Few: return launch_int8_few(a, st);
        case kInt8Mid32: return launch_int8_mid(a, 32, plan.splits, part, st);
        case kInt8Mid64: return launch_int8_mid(a, 64, plan.splits, part, st);
        case kInt8Mid96: return launch_int8_mid(a, 96, plan.splits, part, st);
        default: return launch_int8_tiles(a, (Int8Form)plan.form, plan.splits, part, st);
    }
}

// sizes, bits and flags of a product
bool int8_sizes(int64_t M, int64_t N, int64_t K) { return M >= 0 && N >= 0 && K >= 1 && M <= 0x7FFFFF00 && N <= 0x7FFFFF00 && K <= kInt8MaxK; }
mq_status check_int8(int64_t M, int64_t N, int64_t K, int r, uint32_t flags) {
    if (!int8_sizes(M, N, K)) return MQ_ERR_SHAPE;
    if (r < 1 || r > 8) return MQ_ERR_BITS;
    if ((flags & ~(uint32_t)(MQ_FLAG_GATED | MQ_FLAG_FFN_SILU)) || flags == MQ_FLAG_FFN_SILU) return MQ_ERR_BITS;
    if (K % 16 != 0 || ((flags & MQ_FLAG_GATED) && N % 2 != 0)) return MQ_ERR_ALIGN;
    return MQ_OK;
}

mq_status check_weights(const uint8_t *codes, const float *alpha, const float *zero, const uint16_t *Y) {
    if (!codes || !alpha || !zero || !Y) return MQ_ERR_NULL;
    if (!aligned16(codes) || !aligned16(alpha) || !aligned16(zero) || !aligned16(Y)) return MQ_ERR_ALIGN;
    return MQ_OK;
}

Int8Args int8_args(const uint8_t *codes, const float *alpha, const float *zero, int64_t M, int64_t T, int64_t N, int64_t K, int64_t E, int r,
                   uint32_t flags, uint16_t *Y) {
    Int8Args a{};
    a.codes = codes;
    a.alpha = alpha;
    a.zero = zero;
    a.Y = Y;
    a.M = (int)M;
    a.T = (int)T;
    a.N = (int)N;
    a.K = a.ldq = (int)K;
    a.E = (int)E;
    a.gate = !(flags & MQ_FLAG_GATED) ? 0 : (flags & MQ_FLAG_FFN_SILU) ? 2 : 1;
    a.mult = (float)(1 << (8 - r));
    a.offset = r == 8 ? 128.0f : 0.0f;
    return a;
}

// quantizes the tokens into the workspace and multiplies them
mq_status quantize_and_multiply(Int8Args a, const uint16_t *X, void *ws, size_t ws_bytes, hipStream_t st) {
    const Int8Layout l = int8_layout(a.M > a.T ? a.M : a.T, a.K);
    if (!ws || !aligned16(ws) || ws_bytes < l.part + 256) return MQ_ERR_WORKSPACE;
    const int64_t E = a.offsets ? a.E : 0;
    if (int8_single(a.T, a.N, a.K, E)) return launch_int8_single(a, X, st);
    const Int8Plan plan = int8_plan(a.T, a.N, a.K, E, ws_bytes - l.part - 256);
    if (!int8_launches(plan, a.T, a.N, E)) return MQ_ERR_SHAPE;
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
    int8_t *Xq = reinterpret_cast<int8_t *>(base + l.codes);
    a.ldq = (int)(cdiv(a.K, kInt8Line) * kInt8Line);
    float *scale = reinterpret_cast<float *>(base + l.scale);
    int32_t *sum = reinterpret_cast<int32_t *>(base + l.sum);
    // gathered tokens past 2 GiB are quantized in the order of the places: the kernels address those that they gather with 32 bits
    const bool placed = a.rows && (int64_t)a.M * a.ldq > 0x7FFFFFFF;
    const mq_status s = launch_quantize_tokens(X, placed ? a.T : a.M, a.K, a.K, placed ? a.rows : nullptr, a.M, Xq, a.ldq, scale, sum, st);
    if (s != MQ_OK) return s;
    if (placed) {
        a.rows = nullptr;
        a.M = a.T;
    }
    a.Xq = Xq;
    a.scale = scale;
    a.sum = sum;
    return launch_int8(a, plan, base + l.part, st);
}

}  // namespace

mq_status launch_quantize_tokens(const uint16_t *X, int64_t M, int64_t K, int64_t ldx, const int32_t *rows, int64_t X_rows, int8_t *Xq, int64_t ldq,
                                 float *scale, int32_t *sum, hipStream_t st) {
    // A lane holds two to eight pieces of a row in registers.  Short rows have a wave each (11127 of 496 values 8.2 us, with room for 4096 of them 14.2;
    // 8192 of 2048 13.4 and 15.7); a workgroup to each is done sooner where they are few or longer (600 of 4096 4.5 and 5.1 us, 16 of 4096 3.9
    // and 4.6; 1024 threads and 256: 256 of 14336 6.2 and 6.6, 2000 of 14336 21.6 and 20.8).
    if (K <= 1024) return launch_tokens<64, 2, 256>(X, M, K, ldx, rows, X_rows, Xq, ldq, scale, sum, st);
    if (K <= 2048 && M > 512) return launch_tokens<64, 4, 256>(X, M, K, ldx, rows, X_rows, Xq, ldq, scale, sum, st);
    if (K <= 4096) return launch_tokens<256, 2, 256>(X, M, K, ldx, rows, X_rows, Xq, ldq, scale, sum, st);
    if (K <= 16384 && M <= 256) return launch_tokens<1024, 2, 1024>(X, M, K, ldx, rows, X_rows, Xq, ldq, scale, sum, st);
    if (K <= 16384) return launch_tokens<256, 8, 256>(X, M, K, ldx, rows, X_rows, Xq, ldq, scale, sum, st);
    return launch_tokens<1024, 16, 1024>(X, M, K, ldx, rows, X_rows, Xq, ldq, scale, sum, st);
}

size_t int8_workspace_bytes(int64_t M, int64_t N, int64_t K, bool grouped) {
    if (!int8_sizes(M, N, K) || K % 16 != 0) return 0;
    size_t part = 0;
    if (!grouped && M > 0 && N > 0) {
        const Int8Plan plan = int8_plan(M, N, K, 0, kInt8PartBytes);
        part = (size_t)int8_part_bytes(kInt8Costs[plan.form], M, N, plan.splits);
    }
    return int8_layout(M, K).part + part + 256;
}

}  // namespace mq

extern "C" mq_status mq_quantize_tokens(const uint16_t *X, int64_t M, int64_t K, int64_t ldx, int8_t *Xq, float *scale, int32_t *sum,
                                        void *hip_stream) {
    using namespace mq;
    if (M < 0 || K < 1 || M > 0x7FFFFF00 || K > kInt8MaxK || ldx < K || ldx > ((int64_t)1 << 40)) return MQ_ERR_SHAPE;
    if (K % 16 != 0 || ldx % 8 != 0) return MQ_ERR_ALIGN;
    if (M == 0) return MQ_OK;
    if (!X || !Xq || !scale || !sum) return MQ_ERR_NULL;
    if (!aligned16(X) || !aligned16(Xq) || !aligned16(scale) || !aligned16(sum)) return MQ_ERR_ALIGN;
    return launch_quantize_tokens(X, M, K, ldx, nullptr, M, Xq, K, scale, sum, static_cast<hipStream_t>(hip_stream));
}

extern "C" mq_status mq_linear_fwd_int8_quantized(const int8_t *Xq, const float *scale, const int32_t *sum, const uint8_t *codes,
                                                  const float *alpha, const float *zero, int64_t M, int64_t N, int64_t K, int r,
                                                  uint32_t flags, uint16_t *Y, void *ws, size_t ws_bytes, void *hip_stream) {
    using namespace mq;
    mq_status s = check_int8(M, N, K, r, flags);
    if (s != MQ_OK || M == 0 || N == 0) return s;
    if (!Xq || !scale || !sum) return MQ_ERR_NULL;
    s = check_weights(codes, alpha, zero, Y);
    if (s != MQ_OK) return s;
    if (!aligned16(Xq) || !aligned16(scale) || !aligned16(sum)) return MQ_ERR_ALIGN;
    if (ws && !aligned16(ws)) return MQ_ERR_WORKSPACE;
    Int8Args a = int8_args(codes, alpha, zero, M, M, N, K, 1, r, flags, Y);
    a.Xq = Xq;
    a.scale = scale;
    a.sum = sum;
    const Int8Plan plan = int8_plan(M, N, K, 0, ws && ws_bytes > 256 ? ws_bytes - 256 : 0);
    if (!int8_launches(plan, M, N, 0)) return MQ_ERR_SHAPE;
    uint8_t *part = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
    return launch_int8(a, plan, part, static_cast<hipStream_t>(hip_stream));
}

extern "C" mq_status mq_linear_fwd_int8(const uint16_t *X, const uint8_t *codes, const float *alpha, const float *zero, int64_t M, int64_t N,
                                        int64_t K, int r, uint32_t flags, uint16_t *Y, void *ws, size_t ws_bytes, void *hip_stream) {
    using namespace mq;
    mq_status s = check_int8(M, N, K, r, flags);
    if (s != MQ_OK || M == 0 || N == 0) return s;
    if (!X) return MQ_ERR_NULL;
    s = check_weights(codes, alpha, zero, Y);
    if (s != MQ_OK) return s;
    if (!aligned16(X)) return MQ_ERR_ALIGN;
    return quantize_and_multiply(int8_args(codes, alpha, zero, M, M, N, K, 1, r, flags, Y), X, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
}

extern "C" mq_status mq_experts_fwd_int8(const uint16_t *X, int64_t M, const int32_t *rows, const int32_t *offsets, const uint8_t *codes,
                                         const float *alpha, const float *zero, int64_t T, int64_t E, int64_t N, int64_t K, int r,
                                         uint32_t flags, uint16_t *Y, void *ws, size_t ws_bytes, void *hip_stream) {
    using namespace mq;
    mq_status s = check_int8(M, N, K, r, flags);
    if (s != MQ_OK) return s;
    if (T < 0 || T > 0x7FFFFF00 || E < 1 || E > kMaxExperts || (!rows && T > M) || (T > 0 && M == 0)) return MQ_ERR_SHAPE;
    if (T == 0 || N == 0) return MQ_OK;
    if (!X || !offsets) return MQ_ERR_NULL;
    s = check_weights(codes, alpha, zero, Y);
    if (s != MQ_OK) return s;
    if (!aligned16(X) || !aligned16(offsets) || (rows && !aligned16(rows))) return MQ_ERR_ALIGN;
    Int8Args a = int8_args(codes, alpha, zero, M, T, N, K, E, r, flags, Y);
    a.rows = rows;
    a.offsets = offsets;
    return quantize_and_multiply(a, X, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
}
