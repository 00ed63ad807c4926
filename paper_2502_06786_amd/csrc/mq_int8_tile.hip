// The product in 8-bit integers for many tokens: tiles through LDS.
#include "mq_int8.h"
#include "mq_linear.h"

namespace mq {

// 16 zero bytes: what stands past the end of a token's row
__device__ u32x4 int8_zeros = {0u, 0u, 0u, 0u};

// In place in the accumulator file.  The compiler does not see a matrix product here (see mfma16_acc for why and for the waits that
// are ours then): an operand that a vector instruction has written is used two wait states later at the earliest, an accumulator
// read eight after its product.
__device__ __forceinline__ void mfma_i8_acc(i32x4 &acc, const i32x4 &a, const i32x4 &b) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}

// Four waves, WR x WC of them, each with RB blocks of 16 channels times TB blocks of 16 places; stages of 64 k, NBUF of them in LDS.
template <int RB, int TB, int WR, int WC, int NBUF>
struct Int8Tile {
    static constexpr int TN = 16 * RB * WR, TM = 16 * TB * WC;
    static constexpr int STAGE = (TN + TM) * 64;
    static constexpr int OS = TN * 2 + 16;   // bytes of a row of the staged outputs
    static constexpr int LDS = NBUF * STAGE > TM * OS ? NBUF * STAGE : TM * OS;
};

template <bool R8, int RB, int TB, int WR, int WC, int NBUF, int WGS>
__global__ __launch_bounds__(256, WGS) void int8_tile_kernel(Int8Args a, int tiles_m, int tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass only needs the launch stub
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    typedef Int8Tile<RB, TB, WR, WC, NBUF> T;
    constexpr int CL = T::TN / 64, XL = T::TM / 64, LPS = CL + XL, NM = RB * TB;
    static_assert(WR * WC == 4 && T::TN % 64 == 0 && T::TM % 64 == 0, "");
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g4 = lane >> 4, l16 = lane & 15, wr = wave / WC, wc = wave % WC;

    const uint32_t lid = xcd_contiguous_id(blockIdx.x, gridDim.x);
    constexpr int GROUP = 4;
    const int width = GROUP * tiles_n;
    const int first_m = (int)(lid / width) * GROUP;
    const int gsz = min(tiles_m - first_m, GROUP);
    const Block b = find_block(a, first_m + (int)(lid % width) % gsz, T::TM);
    if (b.count <= 0) return;
    const int n0 = (int)(lid % width) / gsz * T::TN;

    const __amdgpu_buffer_rsrc_t rC = make_rsrc(a.codes + ((int64_t)b.expert * a.N + n0) * a.K, (uint64_t)(a.N - n0) * a.K);
    uint32_t coff;
    int col;
    u8_tile_lane<4>(wave, lane, 0, (uint32_t)a.K, coff, col);
    const uint32_t cstep = 64u * (uint32_t)a.K;
    const int8_t *xrow[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int row = wave * 16 + (lane >> 2) + 64 * i;
        xrow[i] = a.Xq + (int64_t)token_of(a, b.place + min(row, b.count - 1)) * a.K + col;
    }

    // load i of stage kt; past the end of the rows zeros, so that every stage has as many loads in flight
    auto issue_one = [&](int kt, int i) {
        const int k0 = kt * 64;
        uint8_t *to = smem + kt % NBUF * T::STAGE + (wave + (i < CL ? i : i - CL) * 4) * 1024;
        if (i < CL) {
            const uint32_t off = k0 + col < a.K ? coff + (uint32_t)k0 : kOOB;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rC, (lds_ptr)to, 16, off + (uint32_t)i * cstep, 0, 0, 0);
        } else {
            const void *from = k0 + col < a.K ? (const void *)(xrow[i - CL] + k0) : (const void *)&int8_zeros;
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)from, (lds_ptr)(to + T::TN * 64), 16, 0, 0);
        }
    };

    const int sw = (group_chunk(g4) ^ ((l16 >> 2) & 3)) << 4;
    const uint32_t ca = (wr * 16 * RB + l16) * 64 + sw, xa = T::TN * 64 + (wc * 16 * TB + l16) * 64 + sw;  // + 1024 per block of 16

    i32x4 acc[RB][TB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = i32x4{0, 0, 0, 0};

#pragma unroll
    for (int s = 0; s < NBUF; ++s)
#pragma unroll
        for (int i = 0; i < LPS; ++i) issue_one(s, i);
    stage_barrier<(NBUF - 1) * LPS, 0>();

    i32x4 wf[2][RB], xf[TB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) wf[0][rb] = signed_codes<R8>(*reinterpret_cast<const i32x4 *>(smem + ca + rb * 1024));
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) xf[tb] = *reinterpret_cast<const i32x4 *>(smem + xa + tb * 1024);

    auto stage = [&](auto set_tag, int kt) {
        constexpr int S = decltype(set_tag)::value;
        // stage kt + 1 has landed, every wave has read stage kt; stages kt + 2 .. may be on their way
        stage_barrier<(NBUF - 2) * LPS, 0>();
        const uint8_t *nxt = smem + (kt + 1) % NBUF * T::STAGE;
        static_for<NM>([&](auto q_tag) {
            constexpr int q = decltype(q_tag)::value, tb = q / RB, rb = q % RB;
            mfma_i8_acc(acc[rb][tb], wf[S][rb], xf[tb]);
            static_for<RB>([&](auto j_tag) {
                constexpr int j = decltype(j_tag)::value;
                if constexpr (q == j * (NM / (4 * RB) > 1 ? NM / (4 * RB) : 1)) wf[1 - S][j] = *reinterpret_cast<const i32x4 *>(nxt + ca + j * 1024);
                if constexpr (R8 && q == NM / 2 + j * (NM / 2 - 3) / RB) {
                    wf[1 - S][j] = signed_codes<R8>(wf[1 - S][j]);
                    asm volatile("" : "+v"(wf[1 - S][j]));   // here and not where it is used
                }
            });
            if constexpr (rb == RB - 1) xf[tb] = *reinterpret_cast<const i32x4 *>(nxt + xa + tb * 1024);
            static_for<LPS>([&](auto l_tag) {
                constexpr int l = decltype(l_tag)::value;
                if constexpr (q == NM / 4 + l * (NM / 2) / LPS) issue_one(kt + NBUF, l);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    const int nkt = (a.K + 63) / 64;
    for (int kt = 0; kt < nkt; kt += 2) {   // (after an odd number of stages one of zeros)
        stage(std::integral_constant<int, 0>{}, kt);
        stage(std::integral_constant<int, 1>{}, kt + 1);
    }
    mfma16_settle();
    wait_vm0();  // (loads past the end must not land in the staged outputs)
    __syncthreads();

    // ---- outputs: staged as rows of bf16, stored as whole rows -------------------------------------------
    const float *alpha = a.alpha + (int64_t)b.expert * a.N, *zero = a.zero + (int64_t)b.expert * a.N;
    float sc[TB], sm[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) {
        const int m = token_of(a, b.place + min(wc * 16 * TB + tb * 16 + l16, b.count - 1));
        sc[tb] = a.scale[m];
        sm[tb] = (float)a.sum[m];
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int nloc = (wr * RB + rb) * 16 + 4 * g4;
        float al[4], ze[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = min(n0 + nloc + e, a.N - 1);
            al[e] = alpha[n];
            ze[e] = zero[n];
        }
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = int8_output(acc[rb][tb][e], sm[tb], sc[tb], al[e], ze[e], a.mult, a.offset);
            uint8_t *to = smem + (wc * 16 * TB + tb * 16 + l16) * T::OS;
            if (a.gate)
                *reinterpret_cast<uint32_t *>(to + nloc) = pack_bf16x2(gated_value(y[0], y[1], a.gate), gated_value(y[2], y[3], a.gate));
            else
                *reinterpret_cast<u32x2 *>(to + nloc * 2) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        }
    }
    __syncthreads();
    const int shift = a.gate ? 1 : 0, cols = T::TN >> shift, first = n0 >> shift, n_out = a.N >> shift;
    if (n_out % 8 == 0) {
        const int per = cols / 8;
        for (int c = threadIdx.x; c < b.count * per; c += 256) {
            const int row = c / per, ch = c % per;
            if (first + ch * 8 < n_out)
                __builtin_nontemporal_store(*reinterpret_cast<const u32x4 *>(smem + row * T::OS + ch * 16),
                                            reinterpret_cast<u32x4 *>(a.Y + (int64_t)(b.place + row) * n_out + first + ch * 8));
        }
    } else {
        for (int c = threadIdx.x; c < b.count * cols; c += 256) {
            const int row = c / cols, ch = c % cols;
            if (first + ch < n_out) a.Y[(int64_t)(b.place + row) * n_out + first + ch] = *reinterpret_cast<const uint16_t *>(smem + row * T::OS + ch * 2);
        }
    }
#else
    (void)a;
#endif
}

namespace {

template <bool R8, int RB, int TB, int WR, int WC, int NBUF, int WGS>
mq_status launch_tile(const Int8Args &a, hipStream_t st) {
    typedef Int8Tile<RB, TB, WR, WC, NBUF> T;
    const int64_t tiles_n = cdiv(a.N, T::TN), tiles_m = block_bound(a.T, a.E, a.offsets != nullptr, T::TM);
    if (tiles_n * tiles_m > 0x7FFFFFFF) return MQ_ERR_SHAPE;
    constexpr auto kernel = int8_tile_kernel<R8, RB, TB, WR, WC, NBUF, WGS>;
    if (!allow_lds<kernel>(T::LDS)) return MQ_ERR_DEVICE;
    kernel<<<dim3((unsigned)(tiles_n * tiles_m)), dim3(256), T::LDS, st>>>(a, (int)tiles_m, (int)tiles_n);
    return launch_status();
}

}  // namespace

#ifndef MQ_TILE
#define MQ_TILE 8, 8, 2, 2, 4, 1
#endif
mq_status launch_int8_tiles(const Int8Args &a, hipStream_t st) {
    return a.offset != 0.f ? launch_tile<true, MQ_TILE>(a, st) : launch_tile<false, MQ_TILE>(a, st);
}

}  // namespace mq
