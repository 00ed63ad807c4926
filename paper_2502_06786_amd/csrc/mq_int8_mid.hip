// The product in 8-bit integers between few and many tokens: small tiles through LDS, several workgroups to a compute unit, K split over
// workgroups where there are not enough tiles.  Bound by memory: three stages of 64 rows of codes and the tokens' (12 to 20 KB each) are on their
// way per workgroup, two or three of those to a compute unit, 36 to 60 KB times that.  16 tokens through 28672 x 4096 26.7 us (4.4 TB/s), 23 to each
// of 8 experts of that size 174 us (5.5 TB/s), 77 through 4096 x 14336 in four ranges 15.7 us and 4 for their sum.  Codes straight to registers
// were slower (every wave waits for its own).
#include "mq_int8.h"
#include "mq_linear.h"

namespace mq {

// NW waves, WR x WC of them, each with RB blocks of 16 channels times TB blocks of 16 places; stages of 128 k, NBUF of them in LDS.
template <int RB, int TB, int WR, int WC, int NBUF>
struct Int8Mid {
    static constexpr int NW = WR * WC, TN = 16 * RB * WR, TM = 16 * TB * WC;
    static constexpr int STAGE = (TN + TM) * 128, LDS = NBUF * STAGE;
};

template <bool R8, int RB, int TB, int WR, int WC, int NBUF>
__global__ __launch_bounds__(64 * WR * WC) void int8_mid_kernel(Int8Args a, int tiles_m, int tiles_n, Int8Ranges s) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass only needs the launch stub
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    typedef Int8Mid<RB, TB, WR, WC, NBUF> T;
    constexpr int NW = T::NW, CL = T::TN / (8 * NW), XL = T::TM / (8 * NW), LPS = CL + XL;
    static_assert(T::TN % (8 * NW) == 0 && T::TM % (8 * NW) == 0, "");
    const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave % WR, wc = wave / WR;
    const int tiles = tiles_m * tiles_n;
    const uint32_t wid = xcd_contiguous_id(blockIdx.x, gridDim.x);
    const int split = (int)(wid / (uint32_t)tiles), tile = (int)(wid % (uint32_t)tiles);
    const Block b = find_block(a, tile % tiles_m, T::TM);   // (tiles of the same channels follow each other)
    if (b.count <= 0) return;
    const int n0 = tile / tiles_m * T::TN;
    const int stages = (a.K + 127) / 128;
    const int s0 = (int)((int64_t)stages * split / s.splits), s1 = (int)((int64_t)stages * (split + 1) / s.splits);
    const int k_end = min(a.K, s1 * 128);

    const __amdgpu_buffer_rsrc_t rC = make_rsrc(a.codes + ((int64_t)b.expert * a.N + n0) * a.K, (uint64_t)(a.N - n0) * a.K);
    const int64_t base = a.rows ? 0 : b.place;   // (gathered tokens lie within 2 GiB)
    const __amdgpu_buffer_rsrc_t rX = make_rsrc(a.Xq + base * a.ldq, (uint64_t)(a.M - base) * a.ldq);
    uint32_t coff;
    int col;
    bf16_tile_lane<NW>(wave, lane, 0, (uint32_t)a.K, coff, col);   // (rows of eight 16-byte chunks as there)
    col *= 2;
    const uint32_t cstep = 8u * NW * (uint32_t)a.K;
    uint32_t xoff[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int row = wave * 8 + (lane >> 3) + 8 * NW * i;
        xoff[i] = row < b.count ? (uint32_t)(token_of(a, b.place + row) - (int)base) * (uint32_t)a.ldq + (uint32_t)col : kOOB;
    }
    auto issue = [&](int st, int buf) {   // past the end of the range: out of range, zeros
        const int k0 = st * 128;
        const bool in = k0 + col < k_end;
#pragma unroll
        for (int i = 0; i < LPS; ++i) {
            const uint32_t off = i < CL ? coff + (uint32_t)i * cstep : xoff[i < CL ? 0 : i - CL];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(i < CL ? rC : rX, (lds_ptr)(smem + buf * T::STAGE + (wave + i * NW) * 1024), 16,
                                                     in ? off + (uint32_t)k0 : kOOB, 0, 0, 0);   // (kOOB + k0 is out of range too)
        }
    };
    uint32_t ca[2], xa[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int sw = ((2 * group_chunk(g4) + t) ^ ((l16 >> 1) & 7)) << 4;
        ca[t] = (wr * 16 * RB + l16) * 128 + sw;
        xa[t] = T::TN * 128 + (wc * 16 * TB + l16) * 128 + sw;
    }
    i32x4 acc[RB][TB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = i32x4{0, 0, 0, 0};

    // what the outputs need, requested before the first stage
    float alpha[RB][4], zero[RB][4], scale[TB];
    int sum[TB];
    if (s.splits == 1) {
        const int64_t first = (int64_t)b.expert * a.N;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = min(n0 + (wr * RB + rb) * 16 + 4 * g4 + e, a.N - 1);
                alpha[rb][e] = a.alpha[first + n];
                zero[rb][e] = a.zero[first + n];
            }
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
            const int m = token_of(a, b.place + min((wc * TB + tb) * 16 + l16, b.count - 1));
            scale[tb] = a.scale[m];
            sum[tb] = a.sum[m];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NBUF - 1; ++i) issue(s0 + i, i);
    int buf = 0, free = NBUF - 1;
    for (int st = s0; st < s1; ++st) {
        // stage st has landed, every wave is done with stage st - 1, whose buffer is filled again
        stage_barrier<(NBUF - 2) * LPS, 0>();
        issue(st + NBUF - 1, free);
        const uint8_t *at = smem + buf * T::STAGE;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            i32x4 w[RB], x[TB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) w[rb] = signed_codes<R8>(*reinterpret_cast<const i32x4 *>(at + ca[t] + rb * 2048));
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) x[tb] = *reinterpret_cast<const i32x4 *>(at + xa[t] + tb * 2048);
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) acc[rb][tb] = mfma_i8(w[rb], x[tb], acc[rb][tb]);
        }
        free = buf;
        buf = buf + 1 == NBUF ? 0 : buf + 1;
    }
    wait_vm0();   // (no load may be on its way into LDS that another workgroup gets)
    if (s.splits > 1) {
        i32x4 *to = s.part + ((int64_t)wid * NW + wave) * (RB * TB * 64) + lane;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) to[(rb * TB + tb) * 64] = acc[rb][tb];
        return;
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int n = n0 + (wr * RB + rb) * 16 + 4 * g4;
        f32x4 ka, kb;
        channel_factors(f32x4{alpha[rb][0], alpha[rb][1], alpha[rb][2], alpha[rb][3]}, f32x4{zero[rb][0], zero[rb][1], zero[rb][2], zero[rb][3]}, a.mult,
                        ka, kb);
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
            const int row = (wc * TB + tb) * 16 + l16;
            if (row < b.count && n < a.N) store_four(a, b.place + row, n, acc[rb][tb], scale[tb], (float)sum[tb], ka, kb);
        }
    }
#else
    (void)a;
#endif
}

namespace {

template <bool R8, int RB, int TB, int WR, int WC, int NBUF>
mq_status launch_mid(const Int8Args &a, int splits, void *part, hipStream_t st) {
    typedef Int8Mid<RB, TB, WR, WC, NBUF> T;
    const int64_t tiles_n = cdiv(a.N, T::TN), grid = int8_grid(T::TM == 32 ? kInt8Mid32 : T::TM == 64 ? kInt8Mid64 : kInt8Mid96, a.T, a.N, a.offsets ? a.E : 0, splits);
    const int64_t tiles_m = grid / tiles_n / splits;
    static_assert(T::NW <= 4 && T::TN == 64 && (T::TM == 32 || T::TM == 64 || T::TM == 96), "the forms of mq_int8_plan.h");
    constexpr auto kernel = int8_mid_kernel<R8, RB, TB, WR, WC, NBUF>;
    if (!allow_lds<kernel>(T::LDS)) return MQ_ERR_DEVICE;
    const Int8Ranges s{static_cast<i32x4 *>(part), splits};
    kernel<<<dim3((unsigned)grid), dim3(64 * T::NW), T::LDS, st>>>(a, (int)tiles_m, (int)tiles_n, s);
    const mq_status status = launch_status();
    return status != MQ_OK || splits == 1 ? status : launch_int8_join<RB, TB, WR, WC>(a, s, st);
}

template <int RB, int TB, int WR, int WC, int NBUF>
mq_status launch_mid_form(const Int8Args &a, int splits, void *part, hipStream_t st) {
    return a.offset != 0.f ? launch_mid<true, RB, TB, WR, WC, NBUF>(a, splits, part, st) : launch_mid<false, RB, TB, WR, WC, NBUF>(a, splits, part, st);
}

}  // namespace

mq_status launch_int8_mid(const Int8Args &a, int places, int splits, void *part, hipStream_t st) {
    return places == 32   ? launch_mid_form<1, 2, 4, 1, 4>(a, splits, part, st)
           : places == 64 ? launch_mid_form<1, 4, 4, 1, 4>(a, splits, part, st)
                          : launch_mid_form<1, 6, 4, 1, 4>(a, splits, part, st);
}

}  // namespace mq
